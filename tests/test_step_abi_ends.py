"""Host-only tests of kvarn_verify_drafts: what a greedy call does not look at, its workspace's size and refusals."""
import pytest

from test_serving_abi import _fake, _refused
from test_step_abi import K  # noqa: F401


def test_greedy_call_looks_at_neither_form_nor_scale_nor_draft(K):  # noqa: F811
    """Without random numbers they may be anything: such a call gets as far as its workspace, which is not there."""
    keep, x = _fake()
    v = 20011
    ok = dict(batch=2, n_draft=4, vocab=v, tokens=x, parent=x, n_live=x, target=x, target_stride=v, draft=None, draft_stride=0, dtype=1,
              form=1, scale=None, uniform=None, path=x, n_path=x, next=x, workspace=None, workspace_bytes=0)
    assert K.kvarn_verify_workspace_bytes(2, 4, v) > 0
    any_of_them = [dict(form=7), dict(form=-1), dict(form=0, scale=x), dict(scale=x + 2), dict(draft=x + 1, draft_stride=-3)]
    _refused(K, K.kvarn_verify_drafts, ok, [{}, *any_of_them], -5)
    _refused(K, K.kvarn_verify_drafts, {**ok, "uniform": x}, any_of_them)


@pytest.mark.parametrize("vocab", [700, 16384, 20011, 65536, 100003, 131072, 1 << 20])
def test_workspace_for_the_largest_is_enough_for_all(K, vocab):  # noqa: F811
    """Its size falls with none of the sizes, so that a buffer for the largest batch does as sequences end."""
    size = K.kvarn_verify_workspace_bytes
    batches = [*range(1, 330), *range(500, 530), *range(1010, 1040), 5000, 1 << 22]
    drafts = [1, 2, 3, 5, 8, 16, 63, 64]
    table = [[size(b, n, vocab) for b in batches] for n in drafts]
    for row in table:
        assert all(x <= y for x, y in zip(row, row[1:]))
    for below, row in zip(table, table[1:]):
        assert all(x <= y for x, y in zip(below, row))
    for n in drafts:
        for b in (1, 40, 200, 5000):
            assert size(b, n, vocab - 1) <= size(b, n, vocab)


@pytest.mark.parametrize("drawn", [True, False])
def test_workspace_refusals(K, drawn):  # noqa: F811
    """Of a call that needs one: missing, one byte short, not aligned to 16 bytes."""
    keep, x = _fake()
    v = 20011
    ok = dict(batch=2, n_draft=4, vocab=v, tokens=x, parent=x, n_live=x, target=x, target_stride=v, draft=x if drawn else None,
              draft_stride=v, dtype=1, form=1, scale=x, uniform=x if drawn else None, path=x, n_path=x, next=x, workspace=x,
              workspace_bytes=1 << 40)
    need = K.kvarn_verify_workspace_bytes(2, 4, v)
    assert need > 0
    _refused(K, K.kvarn_verify_drafts, ok, [dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace_bytes=0),
                                            dict(workspace=x + 8)], -5)
