"""kvarn_read_tokens through the C ABI against the oracle's dequantized tiles.

Tolerance in 32 bits: a rotated element (code a + b) s2 has three roundings of |code a| + |b| at most, and each of
the seven butterfly stages rounds a partial sum of them, so |error| <= 11 * 2^-24 * sum_c (|code a| + |b|) s2 / sqrt(128);
without rotation three roundings of the element's own.  bf16 adds its rounding, 2^-8 of the value.
"""
import numpy as np
import pytest
import torch

import oracle
from serving_util import f64, make_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    torch.cuda.set_device(0)
    return kvarn


def _bound(hc, b, h, kind, n):
    """Error bound of each token's rows [n, 128] in 32 bits."""
    out = np.zeros((n, 128))
    ns = min(n, hc.n_sink)
    for j in range(max(n - hc.n_sink, 0) // 128):
        tile = (hc.k_body if kind == 0 else hc.v_body)[b, h, j]
        codes, a, off, s2 = oracle.unpack_tile(tile, kind, hc.bits, hc.aux)
        a, off, s2 = (x.astype(np.float64) for x in (a, off, s2))
        z = (codes * a + np.abs(off)) * s2[:, None] if kind == 0 else (codes * a[:, None] + np.abs(off)[:, None]) * s2
        e = 11 * 2.0 ** -24 * z.sum(1, keepdims=True) / np.sqrt(128) if hc.rotate else 3 * 2.0 ** -24 * z
        out[ns + j * 128:ns + (j + 1) * 128] = e
    return out


def _check(hc, got, first, n, head_major):
    """got: the K and V rows [batch, ...], 7 where nothing may be written."""
    for b in range(hc.batch):
        length, f = int(hc.seq_len[b]), first[b]
        for h in range(hc.n_kv):
            ref = oracle.gather_stream(hc, b, h)
            for kind in (0, 1):
                rows = f64(got[kind][b, h] if head_major else got[kind][b, :, h])
                inside = [(i, f + i) for i in range(n) if 0 <= f + i < length]
                outside = [i for i in range(n) if not 0 <= f + i < length]
                assert np.all(rows[outside] == 7.0)
                if inside:
                    i, t = np.array(inside).T
                    tol = _bound(hc, b, h, kind, length)[t]
                    if got[kind].dtype == torch.bfloat16:
                        tol = tol * 1.01 + 2.0 ** -8 * np.abs(ref[kind][t])
                    assert np.all(np.abs(rows[i] - ref[kind][t]) <= tol), (b, h, kind)


@pytest.mark.parametrize("bits,aux,n_sink,rotate,paged", [(2, 0, 0, 1, False), (2, 1, 128, 1, True), (4, 0, 5, 1, True),
                                                         (4, 1, 0, 1, False), (2, 0, 0, 0, False), (4, 0, 0, 0, True)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_matches_oracle(K, bits, aux, n_sink, rotate, paged, dtype):
    lens = [n_sink + 3 * 128 + 29, 0, 1, n_sink + 128, n_sink + 127, 2 * 128 + 1]
    p, cache, hc = make_cache(K, lens, 2, bits, aux, n_sink, rotate, paged, seed=bits + n_sink)
    code = K.KVARN_F32 if dtype == torch.float32 else K.KVARN_BF16
    for n, first in ((600, None), (130, [127 + n_sink, 0, 0, 1, 126, 200]), (1, [300, -1, 0, n_sink, 5, 255]), (128, [-64] * 6)):
        f = None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda")
        k, v = (torch.full((6, n, 2, 128), 7.0, device="cuda").to(dtype) for _ in range(2))
        K.kvarn_read_tokens(p, cache, f, n, k, v, code, n * 256, 128, 256)
        torch.cuda.synchronize()
        _check(hc, (k, v), first or [0] * 6, n, False)
        # another layout, one side at a time
        k2, v2 = (torch.full((6, 2, n, 136), 7.0, device="cuda").to(dtype) for _ in range(2))
        K.kvarn_read_tokens(p, cache, f, n, k2, None, code, 2 * n * 136, n * 136, 136)
        K.kvarn_read_tokens(p, cache, f, n, None, v2, code, 2 * n * 136, n * 136, 136)
        torch.cuda.synchronize()
        assert torch.equal(k2[..., :128].transpose(1, 2), k) and torch.equal(v2[..., :128].transpose(1, 2), v)
        assert bool((k2[..., 128:] == 7.0).all()) and bool((v2[..., 128:] == 7.0).all())
    assert int(cache.err_word[0]) == 0


def test_bad_block_ids(K):
    """A tile whose id lies outside the pool is flagged and its rows are left; the others come."""
    lens = [512, 300]
    p, cache, hc = make_cache(K, lens, 2, paged=True, seed=3)
    cache.block_table[0, 2] = cache.n_phys
    cache.block_table[1, 0] = -1
    k = torch.full((2, 512, 2, 128), 7.0, device="cuda")
    v = k.clone()
    K.kvarn_read_tokens(p, cache, None, 512, k, v, K.KVARN_F32, 512 * 256, 128, 256)
    torch.cuda.synchronize()
    assert int(cache.err_word[0]) == 2
    for x in (k, v):
        assert bool((x[0, 256:384] == 7.0).all()) and bool((x[1, :128] == 7.0).all()) and bool((x[1, 300:] == 7.0).all())
        assert not bool((x[0, :256] == 7.0).any()) and not bool((x[1, 128:300] == 7.0).any())


def test_long_offsets(K):
    """Rows behind 2^31 elements, and first + n_tokens behind 2^31."""
    p, cache, hc = make_cache(K, [200, 130], 1, seed=5)
    stride = (1 << 31) + 64
    flat = torch.empty(stride + 256 * 128, dtype=torch.bfloat16, device="cuda")
    flat[:256 * 128] = 7.0
    flat[stride:] = 7.0
    K.kvarn_read_tokens(p, cache, None, 256, flat, None, K.KVARN_BF16, stride, 128, 128)
    got = torch.stack([flat[:256 * 128].view(256, 1, 128), flat[stride:].view(256, 1, 128)])
    want = torch.full((2, 256, 1, 128), 7.0, device="cuda").to(torch.bfloat16)
    K.kvarn_read_tokens(p, cache, None, 256, want, None, K.KVARN_BF16, 256 * 128, 128, 128)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    before = want.clone()
    first = torch.tensor([2**31 - 1, 2**31 - 3], dtype=torch.int32, device="cuda")
    K.kvarn_read_tokens(p, cache, first, 256, want, None, K.KVARN_BF16, 256 * 128, 128, 128)
    torch.cuda.synchronize()
    assert torch.equal(want, before)


# Rotated rows as bf16 are matrix products: a (of values s2) as two halves is off by 2^-22, each of two sums of 32 products
# and what came before cuts off 2^-22 of the largest at most, and the sums and the offset round three times more, together
# below 2^-20 of sum_c (|code a| + |b|) s2 / sqrt(128).  The bound above, 11 * 2^-24 * 1.01, is 0.7 of that, so it is taken here
# as 1.44 of it, and 2^-8 of the value for bf16.
def _bound_products(hc, b, h, kind, n, ref):
    return 1.44 * _bound(hc, b, h, kind, n) + 2.0 ** -8 * np.abs(ref)


@pytest.mark.parametrize("bits,aux,n_sink,paged", [(2, 0, 5, True), (2, 1, 0, False), (4, 0, 0, True), (4, 1, 128, False)])
def test_many_tiles(K, bits, aux, n_sink, paged):
    """Enough tiles that a wave takes a whole one; lengths, ranges and lost pages that end among a workgroup's four."""
    lens = [0, 1, 127 + n_sink, 128 + n_sink, 300, 900, 513 + n_sink, 4200] + [130 + 7 * i for i in range(24)]
    B, n = len(lens), 4100
    p, cache, hc = make_cache(K, lens, 2, bits, aux, n_sink, 1, paged, seed=40 + bits + aux)
    assert B * 2 * 2 * ((n + 126) // 128 + 1) >= 1536
    first = [0] * B
    first[5], first[6], first[7] = 130, 383 + n_sink, 77
    lost = None
    if paged:
        lost = (7, 6)
        cache.block_table[lost] = cache.n_phys + 3
    k, v = (torch.full((B, n, 2, 128), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    f = torch.tensor(first, dtype=torch.int32, device="cuda")
    K.kvarn_read_tokens(p, cache, f, n, k, v, K.KVARN_BF16, n * 256, 128, 256)
    torch.cuda.synchronize()
    assert int(cache.err_word[0]) == (2 if lost else 0)
    for b in range(B):
        for h in range(2):
            ref = oracle.gather_stream(hc, b, h)
            for kind, got in ((0, k), (1, v)):
                rows, m = f64(got[b, :, h]), max(lens[b] - first[b], 0)
                m = min(m, n)
                assert np.all(rows[m:] == 7.0)
                off = np.abs(rows[:m] - ref[kind][first[b]:first[b] + m])
                tol = _bound_products(hc, b, h, kind, lens[b], ref[kind])[first[b]:first[b] + m]
                if lost and b == lost[0]:
                    t0 = n_sink + 128 * lost[1] - first[b]
                    assert np.all(rows[t0:t0 + 128] == 7.0)
                    off[t0:t0 + 128] = 0.0
                assert np.all(off <= tol), (b, h, kind)


@pytest.mark.parametrize("gain", [2.0 ** -60, 2.0 ** 30])
def test_far_scales(K, gain):
    """Keys far from 1: the halves carry them by a power of two of their tile."""
    lens = [700, 260]
    p, cache, hc = make_cache(K, lens, 2, seed=9, gain=gain)
    k = torch.full((2, 700, 2, 128), 7.0, device="cuda", dtype=torch.bfloat16)
    K.kvarn_read_tokens(p, cache, None, 700, k, None, K.KVARN_BF16, 700 * 256, 128, 256)
    torch.cuda.synchronize()
    for b in range(2):
        for h in range(2):
            ref = oracle.gather_stream(hc, b, h)[0]
            assert np.all(np.abs(f64(k[b, :lens[b], h]) - ref) <= _bound_products(hc, b, h, 0, lens[b], ref))


def test_a_tile_of_nan_stays_alone(K):
    """A tile whose step is no number gives rows that are none; its neighbours come as ever, also in one workgroup."""
    for n_kv, n, more in ((1, 700, 0), (8, 8300, 60)):
        p, cache, hc = make_cache(K, [700] * 2, n_kv, extra_blocks=more, seed=4)
        for side in (cache.k_body, cache.v_body):
            side[0, 0, 1, 4096:].view(torch.float32)[5] = float("nan")
        out = []
        for code, dtype in ((K.KVARN_BF16, torch.bfloat16), (K.KVARN_F32, torch.float32)):
            k, v = (torch.zeros((2, n, n_kv, 128), device="cuda", dtype=dtype) for _ in range(2))
            K.kvarn_read_tokens(p, cache, None, n, k, v, code, n * n_kv * 128, 128, n_kv * 128)
            torch.cuda.synchronize()
            out.append((k, v))
        for x, y in zip(*out):
            assert torch.equal(torch.isnan(x), torch.isnan(y))
            assert bool(torch.isnan(x[0, 128:256, 0]).any()) and not bool(torch.isnan(x[1]).any())
