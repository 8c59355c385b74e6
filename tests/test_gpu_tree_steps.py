"""kvarn_tree_attention over caches whose tiles hold steps far apart, through the C ABI against 64 bits.

The tolerance is that of the other caches (2e-3 of a row's largest value for a bf16 out beside its rounding, 2e-5 for
an fp32 one): each product and sum is as exact relative to its own operands, whatever else a tile holds.
"""
import pytest
import torch

from steps_util import cache_of, check_tree, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    torch.cuda.set_device(0)
    return kvarn


# Batch, kv heads, heads of each, drafts: 16 query rows in a workgroup, and 32.
FORMS = [(2, 2, 4, 5), (64, 8, 4, 5)]


def _drafts(form, dtype, gain_v=1.0):
    B, H, g, T = form
    return (normal((B, T, H * g, 128), 1).to(dtype), normal((B, T, H, 128), 2).to(dtype), (gain_v * normal((B, T, H, 128), 3)).to(dtype))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("bits,aux", [(2, 0), (4, 0), (4, 1)])
@pytest.mark.parametrize("what", ["small", "zero"])
def test_one_token_among_values(K, form, bits, aux, what):
    """A value token of 1e-5 times the others, or of zeros among small ones, at every place of the format."""
    B, H, _, _ = form
    for token in (20, 5, 127):
        k, v = normal((B * 300, H, 128), 4), normal((B * 300, H, 128), 5)
        gain = 1e-4 if what == "zero" else 1.0
        v *= gain
        v.view(B, 300, H, 128)[:, token] *= {"small": 1e-5, "zero": 0.0}[what]
        p, cache, hc = cache_of(K, k.bfloat16(), v.bfloat16(), [300] * B, bits, aux)
        q, dk, dv = _drafts(form, torch.bfloat16, gain)
        check_tree(K, p, cache, hc, q, dk, dv, torch.bfloat16, 300, first=2)
