"""kvarn_tree_attention through the C ABI against attention in 64 bits over the oracle's view of the cache.

Tolerance, normwise and against a row's largest value (check_output): for a bf16 out the library's bar of 2e-3
beside the rounding of the stored value (queries and probabilities are held to 2^-11, which moves a logit by about
2^-11 / sqrt(3) * |q| |k| / sqrt(128) < 1e-3 for the logits of a few units used here).  For an fp32 out 2e-5: the 22
bits are below the roundings of the sums, about sqrt(130) * 2^-25 * 4 = 1.4e-6 in a logit and as much in an output.
"""
import numpy as np
import pytest
import torch

from gpu_util import check_output
from serving_util import SCALE, f64, make_cache, random_masks, tree, tree_reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    torch.cuda.set_device(0)
    return kvarn


def _drafts(B, T, n_kv, g, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn((B, T, n_kv * g, 128), generator=gen, device="cuda").to(dtype)
    k = torch.randn((B, T, n_kv, 128), generator=gen, device="cuda").to(dtype)
    v = torch.randn((B, T, n_kv, 128), generator=gen, device="cuda").to(dtype)
    return q, k, v


def _check(K, p, cache, hc, q, k, v, mask, live, out_dtype, max_len, scale=SCALE):
    out = torch.full(q.shape, 7.0, device="cuda").to(out_dtype)
    lv = None if live is None else torch.tensor(live, dtype=torch.int32, device="cuda")
    ws = tree(K, p, cache, q, k, v, mask, lv, out, max_len, scale)
    torch.cuda.synchronize()
    ref = tree_reference(hc, q, k, v, mask, live, scale)
    got = f64(out)
    for b in range(q.shape[0]):
        n = q.shape[1] if live is None else min(max(live[b], 0), q.shape[1])
        assert np.all(got[b, n:] == 7.0)
        if n:
            check_output(got[b, :n], ref[b, :n], out_dtype == torch.bfloat16, 2e-3 if out_dtype == torch.bfloat16 else 2e-5)
    return out, ws


@pytest.mark.parametrize("bits,aux,n_sink,rotate,paged", [(2, 0, 0, 1, False), (2, 1, 128, 1, True), (4, 0, 5, 1, True),
                                                         (4, 1, 0, 1, False), (2, 0, 0, 0, False), (4, 1, 33, 0, True)])
@pytest.mark.parametrize("g,T", [(1, 1), (4, 5), (5, 64), (16, 3), (8, 17)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_matches_reference(K, bits, aux, n_sink, rotate, paged, g, T, dtype):
    lens = [n_sink + 3 * 128 + 29, 0, 1, n_sink + 128, n_sink + 127, 5 * 128 + 65]
    p, cache, hc = make_cache(K, lens, 2, bits, aux, n_sink, rotate, paged, seed=bits + n_sink + g)
    q, k, v = _drafts(6, T, 2, g, dtype, g + T)
    rng = np.random.default_rng(T)
    live = [T, max(T - 1, 1), T, 1, 0, (T + 1) // 2]
    _check(K, p, cache, hc, q, k, v, random_masks(6, T, rng), live, dtype, max(lens))
    assert int(cache.err_word[0]) == 0


@pytest.mark.parametrize("n", [0, 1, 31, 32, 33, 127, 128, 129, 255, 256, 1000, 4096 + 77])
def test_lengths_and_chain(K, n):
    """Every region empty, one token long, full and partly full; the chain is the mask of all drafts before."""
    p, cache, hc = make_cache(K, [n], 1, seed=n)
    q, k, v = _drafts(1, 9, 1, 4, torch.bfloat16, n)
    a, _ = _check(K, p, cache, hc, q, k, v, None, None, torch.bfloat16, n)
    mask = torch.tensor([[(2 << i) - 1 for i in range(9)]], dtype=torch.int64, device="cuda")
    b, _ = _check(K, p, cache, hc, q, k, v, mask, [9], torch.bfloat16, n + 300)  # a hint above the length
    c, _ = _check(K, p, cache, hc, q.float(), k.float(), v.float(), mask, None, torch.float32, n)
    if n == 0:
        assert torch.equal(a, b)


def test_chain_of_64(K):
    p, cache, hc = make_cache(K, [130, 70], 2, n_sink=64, seed=2)
    q, k, v = _drafts(2, 64, 2, 2, torch.bfloat16, 5)
    _check(K, p, cache, hc, q, k, v, None, None, torch.bfloat16, 130)


def test_rows_that_see_nothing(K):
    """Empty masks over an empty cache give zeros; over a cache, the cache alone; bits of drafts that are not there
    count for nothing."""
    p, cache, hc = make_cache(K, [0, 200], 2, seed=1)
    q, k, v = _drafts(2, 6, 2, 4, torch.bfloat16, 1)
    mask = torch.zeros((2, 6), dtype=torch.int64, device="cuda")
    out, _ = _check(K, p, cache, hc, q, k, v, mask, [6, 6], torch.bfloat16, 200)
    assert bool((out[0] == 0).all()) and not bool((out[1] == 0).all())
    mask[:] = -1 << 4  # drafts 4 .. 63, of which none is there
    _check(K, p, cache, hc, q, k, v, mask, [4, 3], torch.bfloat16, 200)


def test_masked_values_do_not_reach_others(K):
    """NaN and infinities in drafts that a row may not see, behind n_live, and in rows of the cache behind the length
    (make_cache fills them with NaN)."""
    p, cache, hc = make_cache(K, [300, 0, 20], 2, n_sink=16, seed=7)
    q, k, v = _drafts(3, 40, 2, 4, torch.bfloat16, 7)
    rng = np.random.default_rng(7)
    mask = random_masks(3, 40, rng)
    live = [40, 35, 2]
    ref = tree_reference(hc, q, k, v, mask, live)
    bad = [5, 17, 36]
    for j, (x, y) in zip(bad, [(float("nan"), float("inf")), (-float("inf"), float("nan")), (float("inf"), -float("inf"))]):
        k[:, j], v[:, j] = x, y
    k[2, 2:], v[2, 2:] = float("nan"), float("nan")
    out = torch.full(q.shape, 7.0, device="cuda").to(torch.bfloat16)
    tree(K, p, cache, q, k, v, mask, torch.tensor(live, dtype=torch.int32, device="cuda"), out, 300)
    torch.cuda.synchronize()
    m = mask.cpu().numpy().view(np.uint64)
    for b in range(3):
        rows = [i for i in range(live[b]) if not any((int(m[b, i]) >> j) & 1 for j in bad if j < live[b])]
        assert rows
        check_output(f64(out)[b, rows], ref[b, rows], True)


def test_strides(K):
    """Rows inside wider rows of a fused projection, fp32 queries with bf16 drafts and the other way round."""
    p, cache, hc = make_cache(K, [150, 513], 2, seed=9)
    q, k, v = _drafts(2, 7, 2, 3, torch.float32, 9)
    wide = torch.full((2, 7, 6 + 2 + 2 + 1, 128), 3.0, device="cuda")
    wide[:, :, :6], wide[:, :, 6:8], wide[:, :, 8:10] = q, k, v
    for qt, kt in ((torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)):
        wq, wk = wide.to(qt), wide.to(kt)
        out = torch.full((2, 7, 9, 128), 7.0, device="cuda").to(torch.bfloat16)
        n = K.kvarn_tree_workspace_bytes(p, cache, 6, 7, 513)
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        c = {torch.float32: 0, torch.bfloat16: 1}
        K.kvarn_tree_attention(p, cache, 6, 7, wq, 11 * 128, c[qt], wk[:, :, 6:], wk[:, :, 8:], 11 * 128, c[kt], None, None,
                               out, 9 * 128, 1, SCALE, 513, ws, n)
        torch.cuda.synchronize()
        check_output(f64(out[:, :, :6]), tree_reference(hc, q.to(qt), k.to(kt), v.to(kt), None, None), True)
        assert bool((out[:, :, 6:] == 7.0).all())


@pytest.mark.parametrize("scale", [4 * SCALE, 40 * SCALE, 0.0, -SCALE])
def test_scales(K, scale):
    """Peaked softmaxes, a flat one and a negative scale; logits in the hundreds are held to the fp32 bar only as far
    as their own fp32 rounding: 2^-24 of 500 moves a probability by 3e-5."""
    p, cache, hc = make_cache(K, [900, 64], 1, bits=4, seed=11)
    q, k, v = _drafts(2, 12, 1, 4, torch.float32, 11)
    out = torch.empty_like(q)
    tree(K, p, cache, q, k, v, None, None, out, 900, scale)
    torch.cuda.synchronize()
    check_output(f64(out), tree_reference(hc, q, k, v, None, None, scale), False, 2e-3)


def test_one_draft_is_a_decode(K):
    """A single draft that sees itself is the token that kvarn_append_decode appends and attends."""
    for n in (5, 300, 3000):
        p, cache, hc = make_cache(K, [n, n], 2, n_sink=4, seed=n)
        q, k, v = _drafts(2, 1, 2, 4, torch.bfloat16, n)
        a, _ = _check(K, p, cache, hc, q, k, v, None, None, torch.bfloat16, n)
        out = torch.empty((2, 8, 128), dtype=torch.bfloat16, device="cuda")
        wb = K.kvarn_decode_workspace_bytes(p, cache, 8, n + 1)
        ws = torch.empty(max(wb, 16), dtype=torch.uint8, device="cuda")
        K.kvarn_append_decode(p, cache, k[:, 0].contiguous(), v[:, 0].contiguous(), 1, n, 8, q[:, 0].contiguous(), 1, out, 1,
                              SCALE, ws, wb)
        torch.cuda.synchronize()
        check_output(f64(a[:, 0]), f64(out), True, 2e-3 + 2.0 ** -8)  # both are rounded to bf16


def test_large_values(K):
    """Keys and values far from 1: scales of the tiles beyond what 16 bits hold."""
    for gain in (1e6, 1e-6):
        p, cache, hc = make_cache(K, [400], 1, seed=13, gain=gain)
        q, k, v = _drafts(1, 5, 1, 4, torch.float32, 13)
        _check(K, p, cache, hc, q / gain, k * gain, v, None, None, torch.float32, 400)
        _check(K, p, cache, hc, (q / gain).bfloat16(), (k * gain).bfloat16(), v.bfloat16(), None, None, torch.bfloat16, 400)


def test_bad_block_ids(K):
    """An id outside the pool sets bit 1 and the sequence's body is skipped; the other sequences are as they were."""
    lens = [512, 300, 700]
    p, cache, hc = make_cache(K, lens, 2, paged=True, seed=3)
    q, k, v = _drafts(3, 5, 2, 4, torch.bfloat16, 3)
    good, _ = _check(K, p, cache, hc, q, k, v, None, None, torch.bfloat16, 700)
    cache.block_table[1, 1] = cache.n_phys
    out = torch.empty_like(good)
    tree(K, p, cache, q, k, v, None, None, out, 700)
    torch.cuda.synchronize()
    assert int(cache.err_word[0]) == 2
    assert torch.equal(out[0], good[0]) and torch.equal(out[2], good[2])


@pytest.mark.parametrize("B,n_kv,g,T,lens", [(1, 1, 4, 16, 33000), (2, 8, 4, 16, 8245), (1, 8, 16, 64, 4100), (70, 2, 2, 3, 1500)])
def test_long_contexts(K, B, n_kv, g, T, lens):
    """Work split over a long axis and joined; ragged lengths in one call; the same result on every run."""
    ll = [max(lens - 317 * b, 3) for b in range(B)]
    p, cache, hc = make_cache(K, ll, n_kv, seed=B)
    q, k, v = _drafts(B, T, n_kv, g, torch.bfloat16, T)
    mask = random_masks(B, T, np.random.default_rng(B))
    out, _ = _check(K, p, cache, hc, q, k, v, mask, None, torch.bfloat16, max(ll))
    again = torch.empty_like(out)
    tree(K, p, cache, q, k, v, mask, None, again, max(ll))
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    f32 = torch.empty(q.shape, device="cuda")
    tree(K, p, cache, q, k, v, mask, None, f32, max(ll))
    torch.cuda.synchronize()
    check_output(f64(out), f64(f32), True)


@pytest.mark.parametrize("bits,aux,n_sink,rotate,paged", [(2, 0, 0, 1, False), (2, 1, 40, 1, True), (4, 0, 40, 1, True), (4, 1, 0, 1, False),
                                                         (2, 1, 0, 0, False), (4, 0, 0, 0, True)])
def test_many_rows(K, bits, aux, n_sink, rotate, paged):
    """Enough sequences that 32 query rows go together: ragged lengths and trees, the last set of rows partly full."""
    B, T, g = 140, 9, 4
    lens = [n_sink + (b * 37) % 300 if b % 9 else 0 for b in range(B)]
    lens[5], lens[77] = n_sink + 1100, n_sink + 128
    p, cache, hc = make_cache(K, lens, 2, bits, aux, n_sink, rotate, paged, seed=bits)
    q, k, v = _drafts(B, T, 2, g, torch.bfloat16, bits + 1)
    mask = random_masks(B, T, np.random.default_rng(bits))
    live = [(b * 5) % (T + 1) for b in range(B)]
    _check(K, p, cache, hc, q, k, v, mask, live, torch.bfloat16, max(lens))
    # non-finite values of drafts that others may not see, with these kernels
    ref = tree_reference(hc, q[:4], k[:4], v[:4], mask[:4], live[:4])
    v[:, 2], k[:, 2] = float("inf"), float("nan")
    out = torch.empty_like(q)
    tree(K, p, cache, q, k, v, mask, torch.tensor(live, dtype=torch.int32, device="cuda"), out, max(lens))
    torch.cuda.synchronize()
    m = mask.cpu().numpy().view(np.uint64)
    for b in range(4):
        rows = [i for i in range(live[b]) if live[b] <= 2 or not int(m[b, i]) >> 2 & 1]
        if rows:
            check_output(f64(out)[b, rows], ref[b, rows], True)


@pytest.mark.parametrize("T", [7, 6])
@pytest.mark.parametrize("bits,aux", [(2, 0), (4, 1)])
def test_many_rows_of_long_sequences(K, bits, aux, T):
    """The same with long sequences, in order of length (7 drafts: two sets of rows) and in several parts (6: one), against the fp32 out's kernels (which the oracle holds to 2e-5)."""
    B, H, g = 66, 8, 5
    lens = [16500 if b % 11 == 0 else 100 + 150 * b for b in range(B)]
    p, cache, hc = make_cache(K, lens, H, bits, aux, seed=bits)
    q, k, v = _drafts(B, T, H, g, torch.bfloat16, bits)
    mask = random_masks(B, T, np.random.default_rng(bits))
    live = torch.tensor([1 + b % T for b in range(B)], dtype=torch.int32, device="cuda")
    out, f32 = torch.zeros_like(q), torch.zeros(q.shape, device="cuda")
    ws = tree(K, p, cache, q, k, v, mask, live, out, max(lens))
    tree(K, p, cache, q, k, v, mask, live, f32, max(lens))
    torch.cuda.synchronize()
    assert (ws.numel() > 16) == (T == 6)
    check_output(f64(out), f64(f32), True)


@pytest.mark.parametrize("B,g,T,n,bits,aux", [(1, 1, 4, 33000, 2, 1), (8, 4, 16, 4200, 4, 0), (3, 2, 30, 2100, 2, 0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_workgroups_of_eight_waves(K, B, g, T, n, bits, aux, dtype):
    """Few sets of rows over sequences of some length: eight waves share a set, one part or several; ragged down to
    nothing, so that waves and whole parts stay without work."""
    lens = [n if b == 0 else max(n - 900 * b, 0) for b in range(B)]
    p, cache, hc = make_cache(K, lens, 4, bits, aux, n_sink=7, seed=B)
    q, k, v = _drafts(B, T, 4, g, dtype, T)
    mask = random_masks(B, T, np.random.default_rng(B))
    _check(K, p, cache, hc, q, k, v, mask, [max(T - b, 1) for b in range(B)], dtype, n)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_zero_queries(K, dtype):
    """Queries of zeros attend evenly, also over keys that are tiny or large; one such row among others."""
    for gain in (1e-12, 1.0, 1e6):
        p, cache, hc = make_cache(K, [520, 0], 2, seed=17, gain=gain)
        q, k, v = _drafts(2, 6, 2, 4, dtype, 17)
        for rows in (slice(None), slice(2, 3)):
            x = q / gain
            x[:, rows] = 0
            _check(K, p, cache, hc, x, k * gain, v, None, None, dtype, 520)


def test_a_row_of_nan_stays_alone(K):
    """A query that is not a number gives a row that is none, and leaves the others as they are."""
    p, cache, hc = make_cache(K, [700], 2, seed=19)
    q, k, v = _drafts(1, 8, 2, 4, torch.bfloat16, 19)
    good, _ = _check(K, p, cache, hc, q, k, v, None, None, torch.bfloat16, 700)
    for bad in (float("nan"), float("inf")):
        x = q.clone()
        x[0, 3, 2, 5] = bad
        out = torch.empty_like(q)
        tree(K, p, cache, x, k, v, None, None, out, 700)
        torch.cuda.synchronize()
        rest = torch.ones((8, 8), dtype=torch.bool)
        rest[3, 2] = False
        assert not bool(torch.isfinite(out[0, 3, 2]).all())
        check_output(f64(out[0][rest.cuda()]), f64(good[0][rest.cuda()]), True, 2e-3 + 2.0 ** -8)


@pytest.mark.parametrize("B,n_kv,g,T,bits,aux,paged,dtype", [(128, 4, 1, 3, 2, 0, True, torch.bfloat16), (65, 8, 2, 2, 4, 1, False, torch.bfloat16),
                                                          (37, 7, 4, 9, 2, 1, True, torch.bfloat16), (128, 4, 2, 1, 2, 0, False, torch.float32)])
def test_the_longest_first(K, B, n_kv, g, T, bits, aux, paged, dtype):
    """Batches whose sequences are taken by length: lengths in no order, equal ones and empty ones among them, drafts of
    all numbers, down to none; the rows of drafts that are not there stay as they were."""
    rng = np.random.default_rng(B + g)
    lens = [int(x) for x in rng.choice([0, 1, 40, 127, 128, 200, 200, 389], B)]
    lens[B // 3], lens[B - 1] = 3100, 700
    p, cache, hc = make_cache(K, lens, n_kv, bits, aux, 5, 1, paged, seed=B)
    q, k, v = _drafts(B, T, n_kv, g, dtype, B)
    mask = random_masks(B, T, rng)
    _check(K, p, cache, hc, q, k, v, mask, [int(x) for x in rng.integers(0, T + 1, B)], dtype, 3100)
    # equally long, where the order is the index
    lens = [300] * B
    p, cache, hc = make_cache(K, lens, n_kv, bits, aux, 5, 1, paged, seed=B, extra_blocks=24)
    _check(K, p, cache, hc, q, k, v, None, None, dtype, 3100)
