"""kvarn_read_tokens as bf16 over rotated tiles whose steps lie far apart, against the oracle's dequantized tiles.

Tolerance: the 32-bit bound of the other tests, 11 * 2^-24 * sum_c (|code a| + |b|) s2 / sqrt(128), taken at 1.44 for the matrix
products, and 2^-8 of the value for bf16."""
import numpy as np
import pytest
import torch

import oracle
from serving_util import f64
from steps_util import cache_of, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    torch.cuda.set_device(0)
    return kvarn


def _check(K, k, v, lens, bits, aux, **params):
    p, cache, hc = cache_of(K, k, v, lens, bits, aux, **params)
    B, H, n = len(lens), k.shape[1], max(lens)
    got = [torch.full((B, n, H, 128), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    K.kvarn_read_tokens(p, cache, None, n, got[0], got[1], K.KVARN_BF16, n * H * 128, 128, H * 128)
    torch.cuda.synchronize()
    for b in range(min(B, 4)):
        for h in range(H):
            ref = oracle.gather_stream(hc, b, h)
            for kind in (0, 1):
                rows, tol = f64(got[kind][b, :, h]), 2.0 ** -8 * np.abs(ref[kind])
                for j in range(lens[b] // 128):
                    codes, a, off, s2 = (x.astype(np.float64) for x in oracle.unpack_tile((hc.k_body, hc.v_body)[kind][b, h, j], kind, bits, aux))
                    z = (codes * a + np.abs(off)) * s2[:, None] if kind == 0 else (codes * a[:, None] + np.abs(off)[:, None]) * s2
                    tol[128 * j:128 * j + 128] += 1.44 * 11 * 2.0 ** -24 * z.sum(1, keepdims=True) / np.sqrt(128)
                assert np.all(np.abs(rows[:lens[b]] - ref[kind]) <= tol), (b, h, kind)


# A workgroup for each tile, and a wave.
@pytest.mark.parametrize("B", [2, 200])
@pytest.mark.parametrize("bits,aux", [(2, 0), (4, 0), (2, 1), (4, 1)])
@pytest.mark.parametrize("gain", [1.0, 1e-4, 1e-6, 1e-9, 1e-12])
def test_keys_along_one_direction(K, B, bits, aux, gain):
    """Keys that are multiples of one row: every rotated channel but one has no range, and step 1."""
    k = gain * normal((B * 300, 2, 1), 1).expand(-1, -1, 128)
    _check(K, k.contiguous(), normal((B * 300, 2, 128), 2), [300] * B, bits, aux)


@pytest.mark.parametrize("B", [2, 200])
@pytest.mark.parametrize("bits,aux", [(2, 0), (4, 0), (4, 1)])
@pytest.mark.parametrize("gain", [1e-3, 1e-9])
def test_zero_and_large_tokens(K, B, bits, aux, gain):
    """Tokens of zeros and of 10^5 times the others, in keys and values."""
    k, v = (gain * normal((B * 300, 2, 128), s) for s in (3, 4))
    for x in (k, v):
        x.view(B, 300, 2, 128)[:, [3, 40, 127, 200]] = 0
        x.view(B, 300, 2, 128)[:, [20, 255]] *= 1e5
    _check(K, k, v, [300] * B, bits, aux)
