"""Host-only tests of the entry points for rotary positions, drafted tokens and reading back: refusals with
status codes before the GPU is touched, and the rotary frequencies."""
import ctypes
import math

import numpy as np
import pytest


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    return kvarn


def _fake(n=1 << 16, align=256):
    buf = (ctypes.c_uint8 * (n + align))()
    addr = ctypes.addressof(buf)
    return buf, addr + (-addr) % align


class FakeCache:
    """Host addresses in the place of device buffers: only checked, never used."""

    def __init__(self, K, batch=2, n_kv=2, max_blocks=4, n_sink=0):
        self.keep, at = _fake()
        self.n_kv = n_kv
        self.d = K.kvarn_cache(batch, n_kv, max_blocks, at, at, at, at, at if n_sink else None, at if n_sink else None, at,
                               None, None, 0)

    def desc(self):
        return self.d


def _refused(K, call, ok, bad, status=-1):
    for kw in bad:
        with pytest.raises(K.KVarNError) as e:
            call(**{**ok, **kw}, stream=0)
        assert e.value.status == status, kw


def test_rotary_refusals(K):
    keep, x = _fake()
    rope = lambda rot=128, layout=0, amp=1.0, freq=x: K.kvarn_rope(rot, layout, amp, freq)  # noqa: E731
    ok = dict(rope=rope(), q=x, n_q=4, q_stride=512, q_out=x, q_out_stride=512, k=x, n_kv=2, k_stride=256, k_out=x,
              k_out_stride=256, dtype=1, n_tokens=6, positions=None, seq_start=None, tokens_per_seq=3, inverse=0)
    bad = [dict(rope=rope(rot=r)) for r in (0, 1, 7, 130, -2)]
    bad += [dict(rope=rope(layout=2)), dict(rope=rope(amp=float("nan"))), dict(rope=rope(amp=float("inf"))),
            dict(rope=rope(freq=None)), dict(rope=rope(freq=x + 4)), dict(q=None), dict(q_out=None), dict(k=None),
            dict(q=x + 1), dict(dtype=2), dict(n_q=0, n_kv=0), dict(n_q=-1), dict(n_kv=-1), dict(q_stride=511),
            dict(q_out_stride=500), dict(k_stride=-256), dict(k_stride=255), dict(q_out_stride=640), dict(n_tokens=-1),
            dict(tokens_per_seq=0), dict(tokens_per_seq=4), dict(inverse=2), dict(positions=x + 2), dict(seq_start=x + 1),
            dict(q_stride=1 << 62, q_out_stride=1 << 62)]
    _refused(K, K.kvarn_rotary, ok, bad)
    K.kvarn_rotary(**{**ok, "n_tokens": 0, "q": None}, stream=0)  # nothing to do


def test_frequencies(K):
    def plain(rot, base):
        return np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])

    S = K.kvarn_rope_scaling
    for rot, base in ((128, 10000.0), (64, 500000.0), (2, 10000.0)):
        f, amp = K.kvarn_rope_frequencies(rot, base)
        assert amp == 1.0
        np.testing.assert_allclose(f.numpy()[:rot // 2], plain(rot, base), rtol=1e-14)
    f, amp = K.kvarn_rope_frequencies(128, 1e4, S(K.KVARN_ROPE_LINEAR, 4.0, 0, 0, 0))
    assert amp == 1.0
    np.testing.assert_allclose(f.numpy(), plain(128, 1e4) / 4, rtol=1e-14)
    # the base that stretches the longest wave by the factor and leaves the shortest
    f, amp = K.kvarn_rope_frequencies(128, 1e4, S(K.KVARN_ROPE_BASE, 8.0, 0, 0, 0))
    assert f[0] == 1.0 and amp == 1.0
    np.testing.assert_allclose(f.numpy()[-1], plain(128, 1e4)[-1] / 8, rtol=1e-13)
    # bands: the two ends, and a wave between them by hand
    s = S(K.KVARN_ROPE_BANDS, 8.0, 8192.0, 1.0, 4.0)
    f, amp = K.kvarn_rope_frequencies(128, 5e5, s)
    w, f = plain(128, 5e5), f.numpy()
    turns = 8192 * w / (2 * math.pi)
    assert amp == 1.0 and (turns > 4).any() and (turns < 1).any() and ((turns > 1) & (turns < 4)).any()
    np.testing.assert_allclose(f[turns >= 4], w[turns >= 4], rtol=1e-14)
    np.testing.assert_allclose(f[turns <= 1], w[turns <= 1] / 8, rtol=1e-14)
    mid = (turns > 1) & (turns < 4)
    np.testing.assert_allclose(f[mid], w[mid] * (1 / 8 + (turns[mid] - 1) / 3 * (7 / 8)), rtol=1e-12)
    # ramp by index
    f, amp = K.kvarn_rope_frequencies(128, 1e4, S(K.KVARN_ROPE_RAMP, 16.0, 4096.0, 1.0, 32.0))
    assert amp == pytest.approx(0.1 * math.log(16) + 1, rel=1e-15)
    lo = math.floor(128 * math.log(4096 / (2 * math.pi * 32)) / (2 * math.log(1e4)))
    hi = math.ceil(128 * math.log(4096 / (2 * math.pi * 1)) / (2 * math.log(1e4)))
    w, f = plain(128, 1e4), f.numpy()
    for i in range(64):
        s = min(max(1 - (i - lo) / (hi - lo), 0.0), 1.0)
        assert f[i] == pytest.approx(w[i] * (s + (1 - s) / 16), rel=1e-12), i
    assert K.kvarn_rope_frequencies(128, 1e4, S(K.KVARN_ROPE_RAMP, 0.5, 4096.0, 1.0, 32.0))[1] == 1.0
    nan = float("nan")
    for rot, base, s in [(0, 1e4, None), (3, 1e4, None), (130, 1e4, None), (128, 1.0, None), (128, nan, None),
                         (128, float("inf"), None), (128, 1e4, S(5, 2, 1, 1, 2)), (128, 1e4, S(-1, 2, 1, 1, 2)),
                         (128, 1e4, S(1, 0, 0, 0, 0)), (128, 1e4, S(1, nan, 0, 0, 0)), (2, 1e4, S(2, 2.0, 0, 0, 0)),
                         (128, 1e4, S(3, 2, 0, 1, 4)), (128, 1e4, S(3, 2, 8192, 4, 4)), (128, 1e4, S(4, 2, 8192, 0, 4)),
                         (128, 1e4, S(4, 2, 8192, 1, nan))]:
        with pytest.raises(K.KVarNError) as e:
            K.kvarn_rope_frequencies(rot, base, s)
        assert e.value.status == -1
    with pytest.raises(K.KVarNError):
        K._check("", K.lib().kvarn_rope_frequencies(128, 1e4, None, None, None))


def test_read_refusals(K):
    keep, x = _fake()
    c = FakeCache(K)
    p = K.kvarn_params_init(2)
    ok = dict(p=p, cache=c, first=x, n_tokens=5, k_out=x, v_out=x, out_dtype=1, seq_stride=2048, head_stride=128,
              token_stride=256)
    bad = [dict(first=x + 2), dict(n_tokens=-1), dict(k_out=None, v_out=None), dict(k_out=x + 8), dict(v_out=x + 2),
           dict(out_dtype=7), dict(seq_stride=-8), dict(token_stride=129), dict(head_stride=4), dict(token_stride=64),
           dict(seq_stride=0), dict(seq_stride=1 << 60)]
    _refused(K, K.kvarn_read_tokens, ok, bad)
    K.kvarn_read_tokens(**{**ok, "n_tokens": 0}, stream=0)
    p.n_sink = 4  # the cache has no sink
    _refused(K, K.kvarn_read_tokens, ok, [{}])
    p.bits = 3
    _refused(K, K.kvarn_read_tokens, ok, [{}], -2)


def test_tree_refusals(K):
    keep, x = _fake()
    c = FakeCache(K, batch=1)
    p = K.kvarn_params_init(2)
    ok = dict(p=p, cache=c, n_q=8, n_draft=4, q=x, q_stride=1024, q_dtype=1, k_draft=x, v_draft=x, kv_stride=256, kv_dtype=1,
              mask=x, n_live=x, out=x, out_stride=1024, out_dtype=1, sm_scale=0.1, max_len_hint=600, workspace=x,
              workspace_bytes=1 << 40)
    bad = [dict(n_q=7), dict(n_q=0), dict(n_q=34), dict(n_draft=0), dict(n_draft=65), dict(q=None), dict(out=None),
           dict(k_draft=None), dict(v_draft=None), dict(q=x + 2), dict(out=x + 8), dict(k_draft=x + 4), dict(q_stride=1023),
           dict(q_stride=1020), dict(q_stride=896), dict(out_stride=-1024), dict(kv_stride=128), dict(q_dtype=3),
           dict(kv_dtype=-1), dict(out_dtype=2), dict(mask=x + 4), dict(n_live=x + 2), dict(sm_scale=float("nan")),
           dict(sm_scale=float("inf")), dict(max_len_hint=-1), dict(q_stride=1 << 60)]
    _refused(K, K.kvarn_tree_attention, ok, bad)
    need = K.kvarn_tree_workspace_bytes(p, c, 8, 4, 60000)
    if need:
        ok["max_len_hint"] = 60000
        _refused(K, K.kvarn_tree_attention, ok, [dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=x + 8)], -5)
    for args in [(7, 4, 600), (8, 0, 600), (8, 65, 600), (8, 4, -1)]:
        assert K.kvarn_tree_workspace_bytes(p, c, *args) == 0


def test_path_refusals(K):
    keep, x = _fake()
    c = FakeCache(K)
    p = K.kvarn_params_init(4)
    ok = dict(p=p, cache=c, n_draft=4, k_draft=x, v_draft=x, kv_stride=256, dtype=0, path=x, max_path=6, n_path=x)
    bad = [dict(n_draft=0), dict(n_draft=65), dict(k_draft=None), dict(v_draft=x + 8), dict(kv_stride=255), dict(kv_stride=254),
           dict(dtype=2), dict(path=x + 2), dict(max_path=0), dict(max_path=65), dict(path=None), dict(n_path=None),
           dict(n_path=x + 1)]
    _refused(K, K.kvarn_append_path, ok, bad)
