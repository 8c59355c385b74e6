"""Rotary positions through the C ABI against the formula in 64 bits.

Tolerance: the angle in half turns is rounded to 32 bits (2^-25, times pi) and sincospi is good to 2 units (2^-23), together
under 4e-7 in cos and sin; the two products and the sum round to 2^-24 each.  So |error| <= 7e-7 A (|x| + |y|), and a bf16 result
adds its own rounding, 2^-8 of the value.
"""
import numpy as np
import pytest
import torch

from serving_util import dt, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    torch.cuda.set_device(0)
    return kvarn


def _reference(x, pos, freq, amp, rot, half, inverse):
    """[n, heads, 128] in 64 bits, and |x| + |y| of each element's pair."""
    x = f64(x)
    ang = pos.astype(np.longdouble)[:, None, None] * freq * (-1 if inverse else 1)  # at 2^31 64 bits are good to 2e-7
    c, s, h = (amp * np.cos(ang)).astype(np.float64), (amp * np.sin(ang)).astype(np.float64), rot // 2
    i0 = np.arange(h) if half else 2 * np.arange(h)
    i1 = i0 + h if half else i0 + 1
    y, size = x.copy(), np.zeros_like(x)
    y[..., i0], y[..., i1] = x[..., i0] * c - x[..., i1] * s, x[..., i0] * s + x[..., i1] * c
    size[..., i0] = size[..., i1] = np.abs(x[..., i0]) + np.abs(x[..., i1])
    return y, size


def _check(got, x, pos, rope, rot, half, inverse):
    y, size = _reference(x, pos, rope.freq.cpu().numpy(), np.float64(np.float32(rope.amplitude)), rot, half, inverse)
    tol = 7e-7 * rope.amplitude * size + (2.0 ** -8 * np.abs(y) if got.dtype == torch.bfloat16 else 0.0)
    assert np.all(np.abs(f64(got) - y) <= tol)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("rot", [128, 64, 16, 48, 2, 90])
@pytest.mark.parametrize("n,n_q,n_kv", [(1, 1, 1), (3, 4, 1), (37, 10, 2), (261, 3, 3), (4, 0, 5), (5, 7, 0)])
def test_matches_formula(K, dtype, half, rot, n, n_q, n_kv):
    g = torch.Generator(device="cuda").manual_seed(rot + n)
    rope = K.Rope(rot, 10000.0, K.KVARN_ROPE_HALF if half else K.KVARN_ROPE_INTERLEAVED,
                  K.kvarn_rope_scaling(K.KVARN_ROPE_RAMP, 4.0, 4096.0, 1.0, 32.0))
    x = torch.randn((n, n_q + 2 * n_kv, 128), generator=g, device="cuda").to(dtype)  # rows of a fused projection
    q, k = x[:, :n_q], x[:, n_q:n_q + n_kv]
    pos = torch.randint(0, 1 << 20, (n,), generator=g, device="cuda", dtype=torch.int32)
    qo, ko = torch.full((n, n_q, 128), 7.0, device="cuda").to(dtype), torch.full((n, n_kv + 1, 128), 7.0, device="cuda").to(dtype)
    K.kvarn_rotary(rope, q, n_q, x.shape[1] * 128, qo, n_q * 128, k, n_kv, x.shape[1] * 128, ko, (n_kv + 1) * 128,
                   dt(K, x), n, pos, None, 1)
    torch.cuda.synchronize()
    pos = pos.cpu().numpy()
    _check(qo, q, pos, rope, rot, half, False)
    _check(ko[:, :n_kv], k, pos, rope, rot, half, False)
    assert bool((ko[:, n_kv:] == 7.0).all())  # heads that are not the call's
    # in place, and off again
    y = x.clone()
    args = (y, n_q, x.shape[1] * 128, y, x.shape[1] * 128, y[:, n_q:], n_kv, x.shape[1] * 128, y[:, n_q:], x.shape[1] * 128,
            dt(K, x), n, torch.from_numpy(pos).cuda(), None, 1)
    K.kvarn_rotary(rope, *args)
    torch.cuda.synchronize()
    assert torch.equal(y[:, :n_q], qo) and torch.equal(y[:, n_q:n_q + n_kv], ko[:, :n_kv]) and torch.equal(y[:, n_q + n_kv:], x[:, n_q + n_kv:])
    K.kvarn_rotary(rope, *args, 1)
    torch.cuda.synchronize()
    _check(y[:, :n_q], qo, pos, rope, rot, half, True)


@pytest.mark.parametrize("offset", [1, 2, 4])
def test_alignment(K, offset):
    """Pointers and strides that are multiples of an element only."""
    rope = K.Rope(128, 10000.0)
    g = torch.Generator(device="cuda").manual_seed(3)
    flat = torch.randn(9 * 261 + 8, generator=g, device="cuda").to(torch.bfloat16)
    out = torch.full_like(flat, 5.0)
    x, y = flat[offset:offset + 9 * 261].view(9, 261), out[offset:offset + 9 * 261].view(9, 261)
    K.kvarn_rotary(rope, x, 2, 261, y, 261, None, 0, 0, None, 0, K.KVARN_BF16, 9, None, None, 9)
    torch.cuda.synchronize()
    _check(y[:, :256].reshape(9, 2, 128), x[:, :256].reshape(9, 2, 128), np.arange(9), rope, 128, True, False)
    assert bool((y[:, 256:] == 5.0).all()) and bool((out[:offset] == 5.0).all())


def test_positions_of_sequences(K):
    """Lengths on the device, with and without depths; the last position an int32 start allows, and negative ones."""
    rope = K.Rope(128, 500000.0)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((4 * 6, 3, 128), generator=g, device="cuda")
    start = torch.tensor([0, 77, 2**31 - 1, -5], dtype=torch.int32, device="cuda")
    depth = torch.randint(0, 5, (24,), generator=g, device="cuda", dtype=torch.int32)
    for positions in (None, depth):
        y = torch.empty_like(x)
        K.kvarn_rotary(rope, x, 3, 384, y, 384, None, 0, 0, None, 0, K.KVARN_F32, 24, positions, start, 6)
        torch.cuda.synchronize()
        own = np.tile(np.arange(6), 4) if positions is None else depth.cpu().numpy()
        _check(y, x, own.astype(np.int64) + np.repeat(start.cpu().numpy().astype(np.int64), 6), rope, 128, True, False)
    # the token's index alone
    K.kvarn_rotary(rope, x, 3, 384, y, 384, None, 0, 0, None, 0, K.KVARN_F32, 24, None, None, 24)
    torch.cuda.synchronize()
    _check(y, x, np.arange(24), rope, 128, True, False)


def test_inverse_is_the_gradient(K):
    """<R x, w> has the gradient R^T w, against differences along random directions (the map is linear, so a whole
    step is exact but for its rounding)."""
    rope = K.Rope(96, 10000.0, K.KVARN_ROPE_INTERLEAVED, K.kvarn_rope_scaling(K.KVARN_ROPE_RAMP, 8.0, 2048.0, 1.0, 32.0))
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w, d = (torch.randn((50, 4, 128), generator=g, device="cuda") for _ in range(3))

    def turn(t, inverse):
        y = torch.empty_like(t)
        K.kvarn_rotary(rope, t, 4, 512, y, 512, None, 0, 0, None, 0, K.KVARN_F32, 50, None, None, 50, inverse)
        torch.cuda.synchronize()
        return y.double()

    change = ((turn(x + d, 0) - turn(x, 0)) * w.double()).sum()
    grad = (turn(w, 1) * d.double()).sum()
    # 25600 products, each off by at most 1e-6 of numbers of a few units, in random signs
    assert abs(float(change - grad)) <= 1e-6 * 4 * 25600 ** 0.5 * 4


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_long_calls(K, dtype, half):
    """Four heads per thread, an odd number of heads: rows that fill whole lines, and rows that do not, give the same."""
    rope = K.Rope(64, 10000.0, K.KVARN_ROPE_HALF if half else K.KVARN_ROPE_INTERLEAVED)
    n, n_q, n_kv = 2111, 31, 2
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((n, (n_q + n_kv) * 128), generator=g, device="cuda").to(dtype)
    outs = []
    for pad, offset in ((0, 0), (8, 0), (64, 8)):
        st = x.shape[1] + pad
        flat = torch.full((n * st + offset,), 5.0, device="cuda").to(dtype)
        y = flat[offset:].view(n, st)
        K.kvarn_rotary(rope, x, n_q, x.shape[1], y, st, x[:, n_q * 128:], n_kv, x.shape[1], y[:, n_q * 128:], st, dt(K, x), n,
                       None, None, n)
        torch.cuda.synchronize()
        assert bool((y[:, x.shape[1]:] == 5.0).all()) and bool((flat[:offset] == 5.0).all())
        outs.append(y[:, :x.shape[1]].clone())
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    rows = outs[0].view(n, n_q + n_kv, 128)[1900:2000]
    _check(rows, x.view(n, n_q + n_kv, 128)[1900:2000], np.arange(1900, 2000), rope, 64, half, False)
