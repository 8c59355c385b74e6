"""kvarn_tree_attention's workspace: no call relies on its contents, and all that the merge reads is written."""
import numpy as np
import pytest
import torch

from serving_util import SCALE, dt, random_masks
from steps_util import cache_of, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    torch.cuda.set_device(0)
    return kvarn


# Several parts with sets of 16 and of 32 rows, with workgroups of four and of eight waves.
@pytest.mark.parametrize("B,H,g,T,long", [(66, 8, 5, 6, 16500), (70, 8, 3, 9, 16500), (2, 8, 4, 16, 8245), (3, 2, 4, 30, 2100), (1, 1, 4, 16, 33000)])
@pytest.mark.parametrize("bits,aux", [(2, 0), (2, 1), (4, 0), (4, 1)])
@pytest.mark.parametrize("gain", [1.0, 3e-6])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_contents_do_not_matter(K, B, H, g, T, long, bits, aux, gain, dtype):
    lens = [long if b % 11 == 0 else 100 + (150 * b) % 9000 for b in range(B)]
    p, cache, _ = cache_of(K, normal((sum(lens), H, 128), 1).bfloat16(), (gain * normal((sum(lens), H, 128), 2).abs()).bfloat16(), lens, bits, aux)
    gen = torch.Generator(device="cuda").manual_seed(B)
    q, k, v = (torch.randn((B, T, n, 128), generator=gen, device="cuda").to(dtype) for n in (H * g, H, H))
    mask = random_masks(B, T, np.random.default_rng(bits))
    live = torch.tensor([1 + (T - 1 + b) % T for b in range(B)], dtype=torch.int32, device="cuda")
    n = K.kvarn_tree_workspace_bytes(p, cache, H * g, T, long)
    assert n > 0
    outs = []
    for fill in (0.0, float("nan"), 1e30, -1e30):
        ws = torch.full((n // 4,), fill, device="cuda")
        out = torch.zeros(q.shape, dtype=dtype, device="cuda")
        K.kvarn_tree_attention(p, cache, H * g, T, q, H * g * 128, dt(K, q), k, v, H * 128, dt(K, k), mask, live, out, H * g * 128,
                               dt(K, out), SCALE, long, ws, n)
        torch.cuda.synchronize()
        outs.append(out)
    for out in outs:
        assert bool(torch.isfinite(out).all()) and torch.equal(out, outs[0])
