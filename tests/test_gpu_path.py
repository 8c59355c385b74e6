"""kvarn_append_path through the C ABI: the bytes that as many kvarn_append_token calls leave."""
import numpy as np
import pytest
import torch

from serving_util import dt, make_cache

pytestmark = pytest.mark.gpu

BUFFERS = ("k_body", "v_body", "k_resid", "v_resid", "k_sink", "v_sink", "seq_len", "err_word")


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    torch.cuda.set_device(0)
    return kvarn


def _one(K, p, cache, b):
    """Sequence b of a cache as a cache of its own (views into the same buffers where they are a sequence's)."""
    c = K.Cache(p, 1, cache.n_kv, cache.max_blocks, n_phys=cache.n_phys)
    for name in ("k_resid", "v_resid", "k_sink", "v_sink", "seq_len", "block_table"):
        if getattr(cache, name) is not None:
            setattr(c, name, getattr(cache, name)[b:b + 1])
    for name in ("k_body", "v_body"):
        setattr(c, name, getattr(cache, name) if cache.n_phys else getattr(cache, name)[b:b + 1])
    c.err_word = cache.err_word
    return c


def _snapshot(cache):
    return {n: getattr(cache, n).clone() for n in BUFFERS if getattr(cache, n) is not None}


def _same(a, b):
    for n in a:
        x, y = a[n], b[n]
        if x.dtype == torch.bfloat16:
            x, y = x.view(torch.int16), y.view(torch.int16)
        assert torch.equal(x, y), n


def _both(K, p, cache, k, v, path, counts):
    """The call, and token by token on the state before it: both states."""
    start = _snapshot(cache)
    n = torch.tensor(counts, dtype=torch.int32, device="cuda")
    K.kvarn_append_path(p, cache, k.shape[1], k, v, cache.n_kv * 128, dt(K, k), path, path.shape[1] if path is not None else
                        max(1, k.shape[1]), n)
    torch.cuda.synchronize()
    got = _snapshot(cache)
    for name, x in start.items():
        getattr(cache, name).copy_(x)
    for b, count in enumerate(counts):
        one = _one(K, p, cache, b)
        for i in range(count):
            j = int(path[b, i]) if path is not None else i
            K.kvarn_append_token(p, one, k[b, j].contiguous(), v[b, j].contiguous(), dt(K, k), -1)
    torch.cuda.synchronize()
    return got, _snapshot(cache), start


@pytest.mark.parametrize("bits,aux,n_sink,rotate,iters,paged", [(2, 0, 0, 1, 8, False), (2, 1, 128, 1, 8, True), (4, 0, 40, 1, 8, True),
                                                               (4, 1, 0, 1, 2, False), (2, 0, 0, 0, 0, False)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1, 7, 64])
def test_equals_tokens_one_by_one(K, bits, aux, n_sink, rotate, iters, paged, dtype, T):
    lens = [0, 1, n_sink + 127, n_sink + 128 - T // 2, n_sink + 256, n_sink + 128 - T, max(n_sink - 3, 0), n_sink + 300]
    B = len(lens)
    p, cache, _ = make_cache(K, lens, 2, bits, aux, n_sink, rotate, paged, extra_blocks=1, seed=T)
    p.varn_iters = iters
    g = torch.Generator(device="cuda").manual_seed(T)
    k, v = (torch.randn((B, T, 2, 128), generator=g, device="cuda").to(dtype) for _ in range(2))
    path = torch.randint(0, T, (B, min(T + 3, 64)), generator=g, device="cuda", dtype=torch.int32)  # indices again and again
    counts = [T, 0, 1, T, min(T + 3, 64), T, T, T // 2]
    got, want, _ = _both(K, p, cache, k, v, path, counts)
    _same(got, want)
    assert int(got["err_word"][0]) == 0
    got, want, _ = _both(K, p, cache, k, v, None, [min(c, T) for c in counts])
    _same(got, want)


def test_a_boundary_is_not_quantized_twice(K):
    """A sequence at a group's end whose path is empty keeps its tiles: its residual's rows are old."""
    p, cache, _ = make_cache(K, [256, 384], 2, extra_blocks=1, seed=1)
    k = torch.randn((2, 4, 2, 128), device="cuda")
    got, want, start = _both(K, p, cache, k, k, None, [0, 2])
    _same(got, want)
    assert torch.equal(got["k_body"], start["k_body"]) and got["seq_len"].tolist() == [256, 386]


def test_refused_sequences(K):
    """Bad counts, bad indices and full bodies leave their sequence as it was and set their bits; the others go on."""
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn((5, 6, 2, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    for case, bit in (("count", 8), ("negative", 8), ("index", 8), ("below", 8), ("full", 1), ("length", 1)):
        p, cache, _ = make_cache(K, [100, 254, 254, 254, 10], 2, seed=3)  # one body tile each
        path = torch.arange(6, dtype=torch.int32, device="cuda").repeat(5, 1)
        counts = [6, 1, 0, 1, 6]
        touched = 3
        if case == "count":
            counts[3] = 7
        elif case == "negative":
            counts[3] = -1
        elif case == "index":
            counts[3], path[3, 0] = 1, 6
        elif case == "below":
            path[3, 0] = -1
        elif case == "full":
            counts[3] = 2
        else:
            cache.seq_len[3] = -7
        path[:, 5] = torch.tensor([5, 99, 99, 99, 0], dtype=torch.int32)  # behind the counts: not looked at
        before = _snapshot(cache)
        K.kvarn_append_path(p, cache, 6, k, v, 256, 1, path, 6, torch.tensor(counts, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        after = _snapshot(cache)
        assert int(after["err_word"][0]) == bit, case
        for n in ("k_body", "v_body", "k_resid", "v_resid"):
            x, y = before[n][touched], after[n][touched]
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), (case, n)
        want = [106, 255, 254, int(before["seq_len"][3]), 16]
        assert after["seq_len"].tolist() == want, case


def test_bad_block_id(K):
    """A group that fills without a valid block sets bit 1, like kvarn_append_token; the rest goes on."""
    p, cache, _ = make_cache(K, [250, 250], 2, paged=True, extra_blocks=1, seed=4)
    cache.block_table[0, 1] = -1
    k = torch.randn((2, 8, 2, 128), device="cuda").to(torch.bfloat16)
    got, want, _ = _both(K, p, cache, k, k, None, [8, 8])
    _same(got, want)
    assert int(got["err_word"][0]) == 2
