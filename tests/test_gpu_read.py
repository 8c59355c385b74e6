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
