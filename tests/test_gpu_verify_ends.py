"""Verification of drafted tokens at the ends of its arguments' ranges, through the C ABI."""
import numpy as np
import pytest
import torch

from test_gpu_verify import K, call, check, random_case  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", ["drawn", "fixed"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,v", [(6, 3001), (6, 20011), (1, 3001), (1, 70001)])
def test_infinite_logits_without_a_temperature(K, t, v, dtype, mode):  # noqa: F811
    """An inverse temperature that is not positive leaves a row without weight wherever an infinite logit lies in it, for the walk
    alone and after the launches before it."""
    at, scales = [0, 3, 64, 2200, v - 1], [0.0, -1.0, float("nan")]
    b = len(at) * len(scales)
    case = list(random_case(121, b, t, v, dtype, True, mode, True))
    case[2] = None
    case[6] = torch.tensor(scales, device="cuda").repeat(len(at))
    for i in range(b):
        case[3][i, :, at[i // len(scales)]] = float("inf")
        if t > 1:
            case[0][i, 1:] = at[i // len(scales)]
    path, n, nxt = call(K, *case)
    assert nxt.tolist() == [-1] * b and n.tolist() == [1] * b and path.tolist() == [[0] + [-1] * (t - 1)] * b


@pytest.mark.parametrize("mode", ["drawn", "fixed"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [1000, 20011])
def test_logits_whose_difference_overflows(K, v, dtype, mode):  # noqa: F811
    """One entry at 3e38 over others at -3e38, at inverse temperatures about 10^-38: their difference is infinite in 32 bits, but
    the others hold half of the weight."""
    b, t = 64, 2
    x = torch.full((b, t, v), -3e38, device="cuda")
    x[..., 8] = 3e38
    target, draft = (x * 0.85).to(dtype), x.to(dtype)  # (the draft's token 8 is likelier than the target's)
    scale = torch.full((b,), float(np.log(v - 1) / 6e38), device="cuda")
    tokens = torch.full((b, t), 8, dtype=torch.int32, device="cuda")
    u = torch.rand((b, t), generator=torch.Generator(device="cuda").manual_seed(131), device="cuda")
    case = (tokens, None, None, target, draft if mode == "drawn" else None, True, scale, u, v)
    got = call(K, *case)
    check(got, *case)
    assert 0 < int((got[1] == 2).sum()) < 55


@pytest.mark.parametrize("t,v", [(1, 3001), (1, 70001), (4, 3001), (4, 20011)])
def test_inverse_temperatures_beyond_6e36(K, t, v):  # noqa: F811
    """They make a sequence greedy: of several largest entries the first, where one below lets them share the weight."""
    x = torch.zeros((4, t, v), device="cuda")
    x[..., [1100, 2900]] = 1.0
    scale = torch.tensor([5.9e36, 6.1e36, 6.5e36, 7e36], device="cuda")
    u = torch.full((4, t), 0.75, device="cuda")
    tokens = torch.full((4, t), 5, dtype=torch.int32, device="cuda") if t > 1 else None
    assert call(K, tokens, None, None, x, None, True, scale, u, v)[2].tolist() == [2900, 1100, 1100, 1100]


@pytest.mark.parametrize("v", [3001, 20011])
def test_greedy_without_form_and_scale(K, v):  # noqa: F811
    """Without random numbers neither form nor scale is looked at, nor a draft row."""
    case = random_case(141, 5, 6, v, torch.bfloat16, True, "greedy", True)
    want = call(K, *case)
    check(want, *case)
    need = K.kvarn_verify_workspace_bytes(5, 6, v)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    words = torch.full((6,), float("nan"), device="cuda")
    for form, scale, draft, stride in ((0, words, None, 0), (7, None, None, 0), (-1, words.data_ptr() + 2, words.data_ptr() + 1, 1)):
        got = [torch.full_like(x, 77) for x in want]
        K.kvarn_verify_drafts(5, 6, v, case[0], case[1], case[2], case[3], v, draft, stride, K.KVARN_BF16, form, scale, None, *got, ws, need)
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("mode", ["drawn", "greedy"])
@pytest.mark.parametrize("v", [20011, 70001])
def test_one_workspace_for_every_batch(K, v, mode):  # noqa: F811
    """A buffer of the size for the largest batch, as sequences end and drafts get fewer; what lies behind it stays."""
    size = K.kvarn_verify_workspace_bytes(210, 5, v)
    ws = torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda")
    for b, t in ((210, 5), (205, 5), (204, 5), (128, 5), (96, 2), (193, 1), (192, 1), (48, 1), (3, 4), (1, 1)):
        case = random_case(151, b, t, v, torch.bfloat16, True, mode, t > 1)
        want = call(K, *case)
        out = [torch.full_like(x, 77) for x in want]
        K.kvarn_verify_drafts(b, t, v, case[0], case[1], case[2], case[3], v, case[4], v, K.KVARN_BF16, K.KVARN_LOGITS, case[6], case[7], *out,
                              ws, size)
        assert all(torch.equal(x, y) for x, y in zip(out, want)), (b, t)
    assert int(ws[size:].min()) == 255
