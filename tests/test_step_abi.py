"""Host-only tests of the entry points for verified drafts, block tables, token maps and positions with several axes:
refusals with status codes before the GPU is touched, and the pairs' axes."""
import ctypes

import pytest

from test_serving_abi import FakeCache, _fake, _refused


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    return kvarn


def test_verify_refusals(K):
    keep, x = _fake()
    ok = dict(batch=2, n_draft=4, vocab=100, tokens=x, parent=x, n_live=x, target=x, target_stride=100, draft=x, draft_stride=104,
              dtype=1, form=1, scale=x, uniform=x, path=x, n_path=x, next=x, workspace=x, workspace_bytes=1 << 40)
    bad = [dict(batch=-1), dict(batch=(1 << 22) + 1), dict(n_draft=0), dict(n_draft=65), dict(vocab=0),
           dict(vocab=(1 << 20) + 1), dict(tokens=None), dict(target=None), dict(target=x + 1), dict(draft=x + 1), dict(target_stride=99), dict(draft_stride=99),
           dict(draft_stride=-104), dict(target_stride=1 << 62), dict(dtype=2), dict(form=2), dict(form=-1), dict(form=0),
           dict(path=None), dict(n_path=None), dict(next=None), dict(tokens=x + 2), dict(parent=x + 1), dict(n_live=x + 2),
           dict(scale=x + 2), dict(uniform=x + 1), dict(path=x + 2), dict(n_path=x + 2), dict(next=x + 3),
           dict(dtype=0, target=x + 2)]
    _refused(K, K.kvarn_verify_drafts, ok, bad)
    K.kvarn_verify_drafts(**{**ok, "batch": 0, "target": None}, stream=0)  # nothing to do
    need = K.kvarn_verify_workspace_bytes(2, 4, 100)
    if need:
        _refused(K, K.kvarn_verify_drafts, ok, [dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=x + 8)], -5)
    for args in [(0, 4, 100), ((1 << 22) + 1, 4, 100), (2, 0, 100), (2, 65, 100), (2, 4, 0), (2, 4, (1 << 20) + 1)]:
        assert K.kvarn_verify_workspace_bytes(*args) == 0


def test_axes(K):
    def axis(*args):
        a = K.kvarn_rope_axes_init(*args)
        return a.n_axes, list(a.axis)[:args[0] // 2]

    assert axis(16, (3, 5)) == (2, [0, 0, 0, 1, 1, 1, 1, 1])
    assert axis(16, (3, 3, 2), K.KVARN_AXES_IN_TURN) == (3, [0, 1, 2, 0, 1, 2, 0, 1])
    assert axis(16, (5, 1, 2), K.KVARN_AXES_IN_TURN) == (3, [0, 1, 2, 0, 2, 0, 0, 0])
    assert axis(12, (0, 4, 0, 2)) == (4, [1, 1, 1, 1, 3, 3])
    assert axis(12, (0, 4, 0, 2), 1) == (4, [1, 3, 1, 3, 1, 1])
    assert axis(128, (64,)) == (1, [0] * 64)
    for args in [(16, (3, 4)), (16, (9,)), (16, (-1, 9)), (16, ()), (16, (2, 2, 2, 1, 1)), (0, (0,)), (7, (3,)), (130, (65,)),
                 (16, (4, 4), 2), (16, (4, 4), -1), (16, (2**31 - 1, 2**31 - 1, 10))]:
        with pytest.raises(K.KVarNError) as e:
            K.kvarn_rope_axes_init(*args)
        assert e.value.status == -1, args
    L, n = K.lib(), (ctypes.c_int32 * 1)(64)
    assert L.kvarn_rope_axes_init(None, 128, 1, n, 0) == -1
    assert L.kvarn_rope_axes_init(ctypes.byref(K.kvarn_rope_axes()), 128, 1, None, 0) == -1


def test_rotary_axes_refusals(K):
    keep, x = _fake()
    rope = lambda rot=128, layout=0, amp=1.0, freq=x: K.kvarn_rope(rot, layout, amp, freq)  # noqa: E731
    axes = K.kvarn_rope_axes_init(128, (24, 20, 20))
    bad_axis, none, five = (K.kvarn_rope_axes_init(128, (24, 20, 20)) for _ in range(3))
    bad_axis.axis[63], none.n_axes, five.n_axes = 3, 0, 5
    ok = dict(rope=rope(), axes=axes, q=x, n_q=4, q_stride=512, q_out=x, q_out_stride=512, k=x, n_kv=2, k_stride=256, k_out=x,
              k_out_stride=256, dtype=1, n_tokens=6, positions=x, pos_stride=1, axis_stride=6, seq_start=None, tokens_per_seq=3,
              inverse=0)
    bad = [dict(rope=rope(rot=r)) for r in (0, 1, 130)]
    bad += [dict(rope=rope(freq=None)), dict(axes=bad_axis), dict(axes=none), dict(axes=five), dict(positions=None),
            dict(positions=x + 2), dict(pos_stride=-1), dict(axis_stride=-6), dict(pos_stride=1 << 61), dict(axis_stride=1 << 61),
            dict(q=None), dict(k_out=None), dict(dtype=2), dict(q_stride=511), dict(q_out_stride=640), dict(n_tokens=-1),
            dict(tokens_per_seq=4), dict(inverse=2), dict(seq_start=x + 1), dict(n_q=0, n_kv=0)]
    _refused(K, K.kvarn_rotary_axes, ok, bad)
    K.kvarn_rotary_axes(**{**ok, "n_tokens": 0, "q": None, "positions": None}, stream=0)
    assert K.lib().kvarn_rotary_axes(ctypes.byref(rope()), None, x, 4, 512, x, 512, x, 2, 256, x, 256, 1, 6, x, 1, 6, None, 3, 0,
                                     0) == -1


def test_pool_refusals(K):
    keep, x = _fake()
    c = FakeCache(K)
    p = K.kvarn_params_init(2)
    pool = lambda ids=x, ring=x, n=x: K.kvarn_block_pool(ids, ring, n)  # noqa: E731
    ok = dict(p=p, cache=c, pool=pool(), lengths=x, extra=1)
    _refused(K, K.kvarn_assign_blocks, ok, [{}])  # no block table
    c.d.block_table, c.d.n_phys = x, 9
    bad = [dict(pool=pool(ids=None)), dict(pool=pool(ring=None)), dict(pool=pool(n=None)), dict(pool=pool(ids=x + 2)),
           dict(pool=pool(ring=x + 1)), dict(pool=pool(n=x + 2)), dict(lengths=x + 2), dict(extra=-1)]
    _refused(K, K.kvarn_assign_blocks, ok, bad)
    c.d.n_phys = 0
    _refused(K, K.kvarn_assign_blocks, ok, [{}])
    p.bits = 5
    _refused(K, K.kvarn_assign_blocks, ok, [{}], -2)


def test_map_refusals(K):
    keep, x = _fake()
    c = FakeCache(K)
    p = K.kvarn_params_init(2)
    ok = dict(p=p, cache=c, cu_seqlens=x, start=x, n_tokens=5, seq=x, position=x, row=x)
    bad = [dict(cu_seqlens=None), dict(cu_seqlens=x + 2), dict(start=x + 1), dict(n_tokens=-1), dict(seq=None, position=None, row=None),
           dict(seq=x + 2), dict(position=x + 1), dict(row=x + 4)]
    _refused(K, K.kvarn_token_map, ok, bad)
    K.kvarn_token_map(**{**ok, "n_tokens": 0, "cu_seqlens": None}, stream=0)
    p.n_sink = 3
    _refused(K, K.kvarn_token_map, ok, [{}])
