"""kvarn_tree_attention over infinities and NaN among the values of the sink, the residual and seen drafts: the channel
that holds one, and no other, is one in every row that sees it."""
import numpy as np
import pytest
import torch

from gpu_util import check_output
from serving_util import f64, make_cache, tree, tree_reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    torch.cuda.set_device(0)
    return kvarn


@pytest.mark.parametrize("B,T,n", [(2, 5, 300), (2, 5, 7 + 128 + 64), (140, 9, 300), (1, 4, 33000)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("where", ["sink", "residual", "last", "draft"])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
def test_one_channel(K, B, T, n, dtype, where, value):
    n_sink = 7
    p, cache, hc = make_cache(K, [n] * B, 2, n_sink=n_sink, seed=T)
    gen = torch.Generator(device="cuda").manual_seed(T)
    q, k, v = (torch.randn((B, T, m, 128), generator=gen, device="cuda").to(dtype) for m in (8, 2, 2))
    ref = tree_reference(hc, q[:1], k[:1], v[:1], None, None)[0]
    rest, channel, head = (n - n_sink) % 128, 77, 1
    if where == "draft":
        v[0, 0, head, channel] = value
    elif where == "sink":
        cache.v_sink[0, head, 3, channel] = value
    else:
        cache.v_resid[0, head, rest - 1 if where == "last" else 2, channel] = value
    out = torch.zeros_like(q)
    tree(K, p, cache, q, k, v, None, None, out, n)
    torch.cuda.synchronize()
    got = f64(out[0])
    hit = got[:, 4 * head:4 * head + 4, channel]
    assert np.isnan(hit).all() if value != value else (hit == value).all()
    got[:, 4 * head:4 * head + 4, channel] = ref[:, 4 * head:4 * head + 4, channel]
    check_output(got, ref, dtype == torch.bfloat16, 2e-3 if dtype == torch.bfloat16 else 2e-5)


@pytest.mark.parametrize("B,T,n", [(2, 5, 300), (140, 9, 300), (1, 4, 33000)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("side", ["k_body", "v_body"])
def test_a_tile_of_nan(K, B, T, n, dtype, side):
    """A step that is no number makes every row of its kv head none, and leaves the others as they are."""
    p, cache, hc = make_cache(K, [n] * B, 2, seed=T)
    gen = torch.Generator(device="cuda").manual_seed(T)
    q, k, v = (torch.randn((B, T, m, 128), generator=gen, device="cuda").to(dtype) for m in (8, 2, 2))
    good, out = torch.zeros_like(q), torch.zeros_like(q)
    tree(K, p, cache, q, k, v, None, None, good, n)
    getattr(cache, side)[0, 1, 1, 4096:].view(torch.float32)[5] = float("nan")
    tree(K, p, cache, q, k, v, None, None, out, n)
    torch.cuda.synchronize()
    assert bool(torch.isnan(out[0, :, 4:]).all()) and torch.equal(out[0, :, :4], good[0, :, :4]) and torch.equal(out[1:], good[1:])
