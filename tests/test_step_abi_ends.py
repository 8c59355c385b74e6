"""Host-only tests of kvarn_verify_drafts: what a greedy call does not look at."""
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
