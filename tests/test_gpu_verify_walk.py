"""Rows that a sequence's workgroup reads in several trips of its loop over ranges where the walk forms the norms itself: calls of
so many rows, or of so few ranges, that no launch goes before it.  A trip is of 16 ranges of 1024 fp32 entries or of 32 of bf16.  The
batch repeats a few sequences: those are held against the definition, the others against them."""
import numpy as np
import pytest
import torch

from test_gpu_verify import K, call, check, random_case  # noqa: F401

pytestmark = pytest.mark.gpu


def tiled(case, b):
    """The case's sequences over and over, b of them."""
    i = torch.arange(b, device="cuda") % case[3].shape[0]
    return [x[i].contiguous() if isinstance(x, torch.Tensor) else x for x in case]


def check_tiled(K, case, b):  # noqa: F811
    few = case[3].shape[0]
    got = call(K, *tiled(case, b))
    check([x[:few] for x in got], *case, few=0.2)
    for x in got:
        assert torch.equal(x, x[torch.arange(b, device="cuda") % few])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mode", ["drawn", "fixed", "greedy"])
@pytest.mark.parametrize("vocab", [17001, 33793, 50257, 65536, 70001])
def test_many_sequences(K, dtype, mode, vocab):  # noqa: F811
    """More rows than norms are formed for before the walk: 641 and more, of greedy sequences 1025."""
    case = random_case(vocab, 6, 5, vocab, dtype, True, mode, True)
    check_tiled(K, case, 129 if mode != "greedy" else 205)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("b,vocab", [(1, 32768), (3, 50257), (7, 64511), (193, 70001), (193, 131072)])
def test_next_token(K, dtype, b, vocab):  # noqa: F811
    case = random_case(b + vocab, min(b, 7), 1, vocab, dtype, True, "fixed", False)
    check_tiled(K, case, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("at", [17000, 40000, 69995])
@pytest.mark.parametrize("drawn", [True, False])
def test_decisions_close_to_their_border(K, drawn, at, dtype):  # noqa: F811
    """Random numbers 8 units of fp32 (2^-21 relative to 2^-20) from the border on either side; the few entries that hold nearly
    all of the weight lie in a later trip or in the row's last, partial range, 50 above a row's first ones."""
    few, b, t, vocab = 12, 216, 3, 70001
    rng = np.random.default_rng(at + drawn)
    x = rng.standard_normal((2, few, t, vocab)).astype(np.float32)
    x[..., at:at + 6] += 50
    x = torch.tensor(x).to(dtype)
    p, q = torch.softmax(x[:, :, 0].double(), 2).numpy()
    tokens = np.zeros((few, t), np.int32)
    u = rng.random((few, t)).astype(np.float32)
    parent = np.tile(np.array([-1, 0, 0], np.int32), (few, 1))  # two children of draft 0
    first = np.full(few, -1)
    for i in range(few):
        hit = i % 2 == 0
        if drawn:
            ratio = p[i, at:at + 6] / q[i, at:at + 6]
            tokens[i, 1], border = at + np.argmin(ratio), ratio.min()  # under 1
            tokens[i, 2], u[i, 2] = at + np.argmax(ratio), 0  # accepted if the first is not
            first[i] = 1 if hit else 2
        else:
            tokens[i, 1], u[i, 1] = at, 1 - 2.0 ** -24  # refused
            tokens[i, 2], border = at + 1, p[i, at + 1] / (1 - p[i, at])
            first[i] = 2 if hit else -1
        near = np.float32(border)
        for _ in range(8):
            near = np.nextafter(near, np.float32(0 if hit else 1))
        u[i, 1 if drawn else 2] = near
    dev = lambda y: torch.as_tensor(y, device="cuda")  # noqa: E731
    case = tiled((dev(tokens), dev(parent), None, dev(x[0]), dev(x[1]) if drawn else None, True, None, dev(u), vocab), b)
    path, n, _ = (y.cpu().numpy() for y in call(K, *case))
    first = first[np.arange(b) % few]
    assert (path[:, 1] == first).all(), np.flatnonzero(path[:, 1] != first)
    assert (n == np.where(first > 0, 2, 1)).all()
