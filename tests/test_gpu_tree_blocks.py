"""kvarn_tree_attention over a sequence with a block id outside the pool: its sink, residual and drafts alone, whatever
the plan."""
import numpy as np
import pytest
import torch

from gpu_util import check_output
from serving_util import SCALE, f64, make_cache, tree

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    torch.cuda.set_device(0)
    return kvarn


# One wave per tile, several parts, workgroups of eight waves, sets of 32 rows.
@pytest.mark.parametrize("B,T,lens", [(3, 5, [512, 300, 700]), (2, 16, [8245, 3000]), (1, 4, [33000]), (3, 30, [2100, 1200, 0]), (140, 9, None)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("which", ["first", "last", "middle"])
def test_the_body_is_left_out_as_a_whole(K, B, T, lens, dtype, which):
    n_sink = 7
    lens = lens or [n_sink + (b * 37) % 600 + 128 for b in range(B)]
    p, cache, hc = make_cache(K, lens, 2, n_sink=n_sink, paged=True, seed=T)
    gen = torch.Generator(device="cuda").manual_seed(T)
    q, k, v = (torch.randn((B, T, n, 128), generator=gen, device="cuda").to(dtype) for n in (8, 2, 2))
    good = torch.zeros_like(q)
    tree(K, p, cache, q, k, v, None, None, good, max(lens))
    torch.cuda.synchronize()
    assert int(cache.err_word[0]) == 0
    nb = (lens[0] - n_sink) // 128
    cache.block_table[0, {"first": 0, "last": nb - 1, "middle": nb // 2}[which]] = (cache.n_phys, -1)[T % 2]
    out = torch.zeros_like(q)
    tree(K, p, cache, q, k, v, None, None, out, max(lens))
    torch.cuda.synchronize()
    assert int(cache.err_word[0]) == 2 and torch.equal(out[1:], good[1:])
    for h in range(2):
        bf = [x.to(torch.bfloat16) for x in (k, v)]
        rest = (lens[0] - n_sink) % 128
        own = [np.concatenate([(f64(s[0, h])), f64(r[0, h, :rest])]) for s, r in ((cache.k_sink, cache.k_resid), (cache.v_sink, cache.v_resid))]
        for i in range(T):
            keys, values = (np.concatenate([own[j], f64(bf[j][0, :i + 1, h])]) for j in (0, 1))
            z = f64(q[0, i, 4 * h:4 * h + 4]) @ keys.T * SCALE
            e = np.exp(z - z.max(1, keepdims=True))
            check_output(f64(out[0, i, 4 * h:4 * h + 4]), (e / e.sum(1, keepdims=True)) @ values, dtype == torch.bfloat16,
                         2e-3 if dtype == torch.bfloat16 else 2e-5)
