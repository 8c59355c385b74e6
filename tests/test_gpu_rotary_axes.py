"""Rotary positions with several axes through the C ABI against the formula in 64 bits.

Tolerance as in test_gpu_rotary.py: |error| <= 7e-7 A (|x| + |y|) for a pair (x, y), and a bf16 result adds its own
rounding, 2^-8 of the value."""
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


def _check(got, x, pos, axis, freq, amp, rot, half, inverse):
    """pos: [n_axes, n] int64."""
    h = rot // 2
    ang = pos.astype(np.longdouble)[axis].T[:, None, :] * freq * (-1 if inverse else 1)
    c, s = (amp * np.cos(ang)).astype(np.float64), (amp * np.sin(ang)).astype(np.float64)
    i0 = np.arange(h) if half else 2 * np.arange(h)
    i1 = i0 + h if half else i0 + 1
    x = f64(x)
    y, size = x.copy(), np.zeros_like(x)
    y[..., i0], y[..., i1] = x[..., i0] * c - x[..., i1] * s, x[..., i0] * s + x[..., i1] * c
    size[..., i0] = size[..., i1] = np.abs(x[..., i0]) + np.abs(x[..., i1])
    tol = 7e-7 * amp * size + (2.0 ** -8 * np.abs(y) if got.dtype == torch.bfloat16 else 0.0)
    assert np.all(np.abs(f64(got) - y) <= tol)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("rot,sections", [(128, (24, 20, 20)), (128, (16, 16, 16, 16)), (64, (16, 16)), (48, (0, 24)), (90, (15, 14, 16)), (2, (1,))])
@pytest.mark.parametrize("n,n_q,n_kv", [(1, 1, 1), (37, 10, 2), (261, 3, 3), (4, 0, 5), (2111, 31, 2)])
def test_matches_formula(K, dtype, half, order, rot, sections, n, n_q, n_kv):
    g = torch.Generator(device="cuda").manual_seed(rot + n)
    rope = K.AxesRope(rot, sections, order, 10000.0, K.KVARN_ROPE_HALF if half else K.KVARN_ROPE_INTERLEAVED,
                      K.kvarn_rope_scaling(K.KVARN_ROPE_RAMP, 4.0, 4096.0, 1.0, 32.0))
    axis, freq, amp = np.array(list(rope.axes.axis)[:rot // 2]), rope.freq.cpu().numpy(), float(np.float32(rope.amplitude))
    x = torch.randn((n, n_q + 2 * n_kv, 128), generator=g, device="cuda").to(dtype)  # rows of a fused projection
    q, k = x[:, :n_q], x[:, n_q:n_q + n_kv]
    pos = torch.randint(0, 1 << 20, (len(sections), n), generator=g, device="cuda", dtype=torch.int32)
    qo, ko = torch.full((n, n_q, 128), 7.0, device="cuda").to(dtype), torch.full((n, n_kv + 1, 128), 7.0, device="cuda").to(dtype)
    K.kvarn_rotary_axes(rope, rope.axes, q, n_q, x.shape[1] * 128, qo, n_q * 128, k, n_kv, x.shape[1] * 128, ko, (n_kv + 1) * 128,
                        dt(K, x), n, pos, 1, n, None, 1)
    torch.cuda.synchronize()
    p = pos.cpu().numpy()
    _check(qo, q, p, axis, freq, amp, rot, half, False)
    _check(ko[:, :n_kv], k, p, axis, freq, amp, rot, half, False)
    assert bool((ko[:, n_kv:] == 7.0).all())
    # in place, positions token by token, and off again
    y, tpos = x.clone(), pos.t().contiguous()
    args = (rope, rope.axes, y, n_q, x.shape[1] * 128, y, x.shape[1] * 128, y[:, n_q:], n_kv, x.shape[1] * 128, y[:, n_q:],
            x.shape[1] * 128, dt(K, x), n, tpos, len(sections), 1, None, 1)
    K.kvarn_rotary_axes(*args)
    torch.cuda.synchronize()
    assert torch.equal(y[:, :n_q], qo) and torch.equal(y[:, n_q:n_q + n_kv], ko[:, :n_kv]) and torch.equal(y[:, n_q + n_kv:], x[:, n_q + n_kv:])
    K.kvarn_rotary_axes(*args, 1)
    torch.cuda.synchronize()
    _check(y[:, :n_q], qo, p, axis, freq, amp, rot, half, True)


@pytest.mark.parametrize("rot", [128, 40])
def test_equal_axes_are_one_position(K, rot):
    """A text token: bit for bit what kvarn_rotary gives."""
    rope = K.AxesRope(rot, (rot // 2 - 8, 5, 3), 1)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((300, 5, 128), generator=g, device="cuda")
    start = torch.tensor([7, 2**31 - 1, -3], dtype=torch.int32, device="cuda")
    pos = torch.randint(-50, 5000, (300,), generator=g, device="cuda", dtype=torch.int32)
    y, z = torch.empty_like(x), torch.empty_like(x)
    K.kvarn_rotary(rope, x, 5, 640, y, 640, None, 0, 0, None, 0, K.KVARN_F32, 300, pos, start, 100)
    K.kvarn_rotary_axes(rope, rope.axes, x, 5, 640, z, 640, None, 0, 0, None, 0, K.KVARN_F32, 300, pos, 1, 0, start, 100)
    torch.cuda.synchronize()
    assert torch.equal(y, z)


def test_starts_of_sequences(K):
    rope = K.AxesRope(128, (16, 24, 24), 0, 500000.0)
    axis, freq = np.array(list(rope.axes.axis)), rope.freq.cpu().numpy()
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((24, 3, 128), generator=g, device="cuda")
    start = torch.tensor([0, 77, 2**31 - 1, -5], dtype=torch.int32, device="cuda")
    pos = torch.randint(0, 90, (3, 30), generator=g, device="cuda", dtype=torch.int32)  # rows longer than the call's
    y = torch.empty_like(x)
    K.kvarn_rotary_axes(rope, rope.axes, x, 3, 384, y, 384, None, 0, 0, None, 0, K.KVARN_F32, 24, pos, 1, 30, start, 6)
    torch.cuda.synchronize()
    p = pos[:, :24].cpu().numpy().astype(np.int64) + np.repeat(start.cpu().numpy().astype(np.int64), 6)
    _check(y, x, p, axis, freq, 1.0, 128, True, False)


def test_own_frequencies(K):
    """An image's rope: height and width each with the frequencies of half a head."""
    rope = K.AxesRope(128, (32, 32), K.KVARN_AXES_SECTIONS, 10000.0, own_frequencies=True)
    f = rope.freq.cpu().numpy()
    want = 10000.0 ** (-2.0 * np.arange(32) / 64)
    np.testing.assert_allclose(f, np.concatenate([want, want]), rtol=1e-14)
    rope = K.AxesRope(128, (32, 32), K.KVARN_AXES_IN_TURN, 10000.0, own_frequencies=True)
    np.testing.assert_allclose(rope.freq.cpu().numpy(), np.repeat(want, 2), rtol=1e-14)


def test_inverse_is_the_gradient(K):
    """<R x, w> has the gradient R^T w, against differences along random directions (the map is linear, so a whole
    step is exact but for its rounding)."""
    rope = K.AxesRope(96, (20, 14, 14), 1, 10000.0, K.KVARN_ROPE_INTERLEAVED, K.kvarn_rope_scaling(K.KVARN_ROPE_RAMP, 8.0, 2048.0, 1.0, 32.0))
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w, d = (torch.randn((50, 4, 128), generator=g, device="cuda") for _ in range(3))
    pos = torch.randint(0, 4000, (3, 50), generator=g, device="cuda", dtype=torch.int32)

    def turn(t, inverse):
        y = torch.empty_like(t)
        K.kvarn_rotary_axes(rope, rope.axes, t, 4, 512, y, 512, None, 0, 0, None, 0, K.KVARN_F32, 50, pos, 1, 50, None, 50, inverse)
        torch.cuda.synchronize()
        return y.double()

    change = ((turn(x + d, 0) - turn(x, 0)) * w.double()).sum()
    grad = (turn(w, 1) * d.double()).sum()
    # 25600 products, each off by at most 1e-6 of numbers of a few units, in random signs
    assert abs(float(change - grad)) <= 1e-6 * 4 * 25600 ** 0.5 * 4
