"""kvarn_tree_attention over caches whose tiles hold steps far apart, through the C ABI against 64 bits.

The tolerance is that of the other caches (2e-3 of a row's largest value for a bf16 out beside its rounding, 2e-5 for
an fp32 one): each product and sum is as exact relative to its own operands, whatever else a tile holds.
"""
import numpy as np
import pytest
import torch

import oracle
from gpu_util import check_output
from serving_util import SCALE, f64, tree, tree_reference
from steps_util import cache_of, check_tree, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    torch.cuda.set_device(0)
    return kvarn


# Batch, kv heads, heads of each, drafts: 16 query rows in a workgroup, and 32.
FORMS = [(2, 2, 4, 5), (64, 8, 4, 5)]


def _drafts(form, dtype, gain_v=1.0):
    B, H, g, T = form
    return (normal((B, T, H * g, 128), 1).to(dtype), normal((B, T, H, 128), 2).to(dtype), (gain_v * normal((B, T, H, 128), 3)).to(dtype))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("bits,aux", [(2, 0), (4, 0), (4, 1)])
@pytest.mark.parametrize("what", ["small", "zero", "large"])
def test_one_token_among_values(K, form, bits, aux, what):
    """A value token of 1e-5 or 1e5 times the others, or of zeros among small ones, at every place of the format."""
    B, H, _, _ = form
    for token in (20, 5, 127):
        k, v = normal((B * 300, H, 128), 4), normal((B * 300, H, 128), 5)
        gain = 1e-4 if what == "zero" else 1.0
        v *= gain
        v.view(B, 300, H, 128)[:, token] *= {"small": 1e-5, "large": 1e5, "zero": 0.0}[what]
        p, cache, hc = cache_of(K, k.bfloat16(), v.bfloat16(), [300] * B, bits, aux)
        q, dk, dv = _drafts(form, torch.bfloat16, gain)
        check_tree(K, p, cache, hc, q, dk, dv, torch.bfloat16, 300, first=2)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("bits,rotate", [(2, 1), (4, 1), (4, 0)])
@pytest.mark.parametrize("gain", [1e-3, 3e-5, 1e-6, 1e-9])
def test_zero_tokens_among_small_values(K, form, bits, rotate, gain):
    """Groups of zero range have step 1, however small the others' values are."""
    B, H, _, _ = form
    k, v = normal((B * 300, H, 128), 6), gain * normal((B * 300, H, 128), 7)
    v.view(B, 300, H, 128)[:, [3, 17, 40, 63, 64, 90, 121, 127, 128, 200]] = 0
    p, cache, hc = cache_of(K, k.bfloat16(), v.bfloat16(), [300] * B, bits, rotate=rotate)
    q, dk, dv = _drafts(form, torch.bfloat16, gain)
    check_tree(K, p, cache, hc, q, dk, dv, torch.bfloat16, 300, first=2)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("gain", [1.0, 3e-4, 1e-4, 1e-6])
def test_zero_channels_among_small_keys(K, form, bits, gain):
    """The same of keys that are not rotated: 48 channels of zeros, and one that holds a constant."""
    B, H, _, _ = form
    k, v = gain * normal((B * 300, H, 128), 8), normal((B * 300, H, 128), 9)
    k[..., 40:88] = 0
    k[..., 5] = 0.5 * gain
    p, cache, hc = cache_of(K, k.bfloat16(), v.bfloat16(), [300] * B, bits, rotate=0)
    q, dk, dv = _drafts(form, torch.bfloat16)
    check_tree(K, p, cache, hc, (q / gain).bfloat16(), (dk * gain).bfloat16(), dv, torch.bfloat16, 300, first=2)


def _logit_bound(hc, q, bits, skip=()):
    """How far `bits` bits of each rotated query value can move a logit: 2^-bits sum_c |q_c k_c| / sqrt(128) at most, over all but
    the tokens `skip`, whose weight is nothing."""
    h = np.array([[(-1.0) ** bin(i & j).count("1") for j in range(128)] for i in range(128)]) / np.sqrt(128)
    worst = 0.0
    for b in range(q.shape[0]):
        for kh in range(hc.n_kv):
            keys, g = np.abs(oracle.gather_stream(hc, b, kh)[0] @ h), q.shape[2] // hc.n_kv
            rows = np.abs(f64(q[b, :, kh * g:(kh + 1) * g]).reshape(-1, 128) @ h)
            worst = max(worst, float((rows @ np.delete(keys, skip, 0).T).max()))
    return 2.0 ** -bits * worst / np.sqrt(128)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("bits", [2, 4])
def test_a_large_token_of_no_weight(K, form, bits):
    """A value token of 10^6 whose key turns away, so that its weight is far below 10^-6: the others are as exact as without it.

    The queries' common part makes one rotated channel of about 28 that meets keys of up to 10, so that the 11 bits move a
    logit by more than elsewhere: by d, and so each probability by a factor of exp(+-2 d), and a row by 2.1 d of its
    largest value at most (values are up to about 4, rows of 300 tokens about 1: 4 times that of the row's largest)."""
    B, H, g, T = form
    k, v = normal((B * 300, H, 128), 10), normal((B * 300, H, 128), 11)
    v.view(B, 300, H, 128)[:, 33] *= 1e6
    q, dk, dv = _drafts(form, torch.bfloat16)
    q = (q * 0.5 + 2.5).bfloat16()  # logits of -30 sqrt(128) 2.5 / sqrt(128) = -75 and less for that token
    k.view(B, 300, H, 128)[:, 33] = -3.0
    p, cache, hc = cache_of(K, k.bfloat16(), v.bfloat16(), [300] * B, bits)
    d = _logit_bound(hc, q[:2], 12, 33)
    assert 4 * 2.1 * d < 0.1  # (without the token's step out of the way the rows are off by their own size)
    check_tree(K, p, cache, hc, q, dk, dv, torch.bfloat16, 300, 2e-3 + 4 * 2.1 * d, first=2)


# An fp32 out: 32 query rows go in sets of 16 here, so one form; groups of zero range from 10^-2 of the others on, where their step of 1 is felt.
FP32 = (2, 2, 4, 9)


@pytest.mark.parametrize("bits,aux,rotate", [(2, 0, 1), (4, 0, 1), (4, 0, 0), (4, 1, 1)])
@pytest.mark.parametrize("gain", [1.0, 1e-1, 1e-2, 1e-3, 3e-5, 1e-6, 1e-9])
def test_fp32_zero_tokens_among_small_values(K, bits, aux, rotate, gain):
    B, H, _, _ = FP32
    k, v = normal((B * 300, H, 128), 12), gain * normal((B * 300, H, 128), 13)
    v.view(B, 300, H, 128)[:, [3, 17, 40, 63, 64, 90, 121, 127, 128, 200]] = 0
    p, cache, hc = cache_of(K, k, v, [300] * B, bits, aux, rotate)
    q, dk, dv = _drafts(FP32, torch.float32, gain)
    check_tree(K, p, cache, hc, q, dk, dv, torch.float32, 300)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("gain", [1.0, 1e-1, 1e-2, 3e-4, 1e-4, 1e-6])
def test_fp32_zero_channels_among_small_keys(K, bits, gain):
    B, H, _, _ = FP32
    k, v = gain * normal((B * 300, H, 128), 14), normal((B * 300, H, 128), 15)
    k[..., 40:88] = 0
    k[..., 5] = 0.5 * gain
    p, cache, hc = cache_of(K, k, v, [300] * B, bits, rotate=0)
    q, dk, dv = _drafts(FP32, torch.float32)
    check_tree(K, p, cache, hc, q / gain, (dk * gain).bfloat16().float(), dv, torch.float32, 300)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("what", [1e5, 1e-5])
def test_fp32_one_token_among_values(K, bits, what):
    B, H, _, _ = FP32
    for token in (20, 5, 127):
        k, v = normal((B * 300, H, 128), 16), normal((B * 300, H, 128), 17)
        v.view(B, 300, H, 128)[:, token] *= what
        p, cache, hc = cache_of(K, k, v, [300] * B, bits)
        q, dk, dv = _drafts(FP32, torch.float32)
        check_tree(K, p, cache, hc, q, dk, dv, torch.float32, 300)


@pytest.mark.parametrize("bits,aux", [(2, 0), (4, 0), (4, 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gains", [(1.0, 1e-9), (1e-9, 1.0), (1e9, 1.0), (0.0, 1e-9), (1e-9, 0.0), (1e-20, 1e20), (1e28, 1.0)])
def test_groups_of_values_far_apart(K, bits, aux, dtype, gains):
    """A group of values far from the other's magnitude weighs by its logits alone; residual and drafts as the second one."""
    for form in (FP32,) if dtype == torch.float32 else FORMS:
        B, H, _, _ = form
        k, v = normal((B * 300, H, 128), 18), normal((B * 300, H, 128), 19)
        v.view(B, 300, H, 128)[:, :128] *= gains[0]
        v.view(B, 300, H, 128)[:, 128:] *= gains[1]
        p, cache, hc = cache_of(K, k.to(dtype), v.to(dtype), [300] * B, bits, aux)
        q, dk, dv = _drafts(form, dtype, gains[1])
        check_tree(K, p, cache, hc, q, dk, dv, dtype, 300, first=2)


@pytest.mark.parametrize("bits,rotate", [(2, 1), (4, 1), (2, 0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("far", [1e3, 1e6, 1e9, 1e20, 1e-9])
def test_queries_far_apart(K, bits, rotate, dtype, far):
    """A query row of any magnitude leaves the rows beside it as exact as they are without it; one of them is zero."""
    for form in (FP32,) if dtype == torch.float32 else FORMS:
        B, H, g, T = form
        k, v = normal((B * 300, H, 128), 20), normal((B * 300, H, 128), 21)
        p, cache, hc = cache_of(K, k.to(dtype), v.to(dtype), [300] * B, bits, rotate=rotate)
        q, dk, dv = _drafts(form, dtype)
        q[:, 3] = 0
        ref = tree_reference(hc, q[:2], dk[:2], dv[:2], None, None)
        q[:, 1, 2] *= far  # draft 1 at the third head
        out = torch.zeros(q.shape, device="cuda", dtype=dtype)
        tree(K, p, cache, q, dk, dv, None, None, out, 300)
        torch.cuda.synchronize()
        rest = np.ones((2, T, H * g), dtype=bool)
        rest[:, 1, 2] = False
        check_output(f64(out)[:2][rest], ref[rest], dtype == torch.bfloat16, 2e-3 if dtype == torch.bfloat16 else 2e-5)
        assert np.isfinite(f64(out)).all()
        if far < 1:  # nearly even weights: its logits are below 10^-8
            check_output(f64(out)[:2, 1, 2], tree_reference(hc, q[:2], dk[:2], dv[:2], None, None)[:, 1, 2], dtype == torch.bfloat16,
                         2e-3 if dtype == torch.bfloat16 else 2e-5)


@pytest.mark.parametrize("scale", [0.0, -1.0, 4.0, 40.0])
@pytest.mark.parametrize("bits", [2, 4])
def test_fp32_scales(K, bits, scale):
    """Flat, turned and peaked softmaxes of an fp32 out.  Logits d off put each probability off by a factor of exp(+-2 d), and a row by
    2.1 d of the largest value it is made of, at most 4 times its own largest (values up to about 4, peaked rows about 1); d goes
    by the 21 bits of 22 that rounding leaves and by the scale.  At 0 and -1 that stays below the bar of 2e-5 by itself."""
    B, H, _, _ = FP32
    k, v = normal((B * 900, H, 128), 22), normal((B * 900, H, 128), 23)
    p, cache, hc = cache_of(K, k, v, [900] * B, bits)
    q, dk, dv = _drafts(FP32, torch.float32)
    d = abs(scale) * _logit_bound(hc, q, 21)
    check_tree(K, p, cache, hc, q, dk, dv, torch.float32, 900, 2e-5 + (4 * 2.1 * d if scale > 1 else 0.0), scale=scale * SCALE)


# (The compact format's steps end at 448 and its offsets at 65504: keys of 10^6 are cut off at their offsets, sums of which cancel.)
@pytest.mark.parametrize("aux,gain_k,gain_v", [(0, 1e6, 1e-3), (0, 1e-6, 1e3), (0, 1e-3, 1e6), (0, 1e3, 1e-2), (1, 1e3, 1e-2)])
@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_and_small(K, bits, aux, dtype, gain_k, gain_v):
    """Keys and values far from 1, each token of its own size, queries that bring the logits back."""
    for form in (FP32,) if dtype == torch.float32 else FORMS:
        B, H, _, _ = form
        k, v = (gain * normal((B * 300, H, 128), s) * torch.exp(0.7 * normal((B * 300, 1, 1), s + 2)) for gain, s in ((gain_k, 24), (gain_v, 25)))
        p, cache, hc = cache_of(K, k.to(dtype), v.to(dtype), [300] * B, bits, aux)
        q, dk, dv = _drafts(form, dtype, gain_v)
        check_tree(K, p, cache, hc, (0.5 * q / gain_k).to(dtype), (dk * gain_k).to(dtype), dv, dtype, 300, first=2)


@pytest.mark.parametrize("bits,aux", [(2, 0), (4, 0), (4, 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("weight", [0.9, 0.99, 0.9999])
@pytest.mark.parametrize("gain", [1.0, 1e-2, 1e-3, 1e-4])
def test_a_zero_token_of_most_weight(K, bits, aux, dtype, weight, gain):
    """Rows that give most of their weight to a value token of zeros: what is left is as exact relative to itself.

    The token's key is the queries' common part, scaled so that its logit gives it about that weight of 300 others (16 kinds of
    rows lie around it).  The others' logits are off by d (the 11 or 21 bits of the queries), which moves the rest by 2.1 d, and the
    weight of the token by its own logit's part of d, which divides all of the rest alike."""
    for form in (FP32,) if dtype == torch.float32 else FORMS:
        B, H, g, T = form
        k, v = normal((B * 300, H, 128), 26), gain * normal((B * 300, H, 128), 27)
        q, dk, dv = _drafts(form, dtype, gain)
        q = (0.7 * q.float() + 0.7).to(dtype)
        x = float(np.log(weight / (1 - weight) * 300) * np.sqrt(128) / (0.7 * 128))
        k.view(B, 300, H, 128)[:, 9] = x
        v.view(B, 300, H, 128)[:, 9] = 0
        p, cache, hc = cache_of(K, k.to(dtype), v.to(dtype), [300] * B, bits, aux)
        d = _logit_bound(hc, q[:2], 12 if dtype == torch.bfloat16 else 22)
        check_tree(K, p, cache, hc, q, dk, dv, dtype, 300, (2e-3 if dtype == torch.bfloat16 else 2e-5) + 4 * 2.1 * d, first=2)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_queries_on_zero_channels(K, bits, dtype):
    """Channels of keys that hold zeros or a constant count for nothing, however large the queries there are."""
    for form in (FP32,) if dtype == torch.float32 else FORMS:
        B, H, _, _ = form
        k, v = normal((B * 300, H, 128), 28), normal((B * 300, H, 128), 29)
        k[..., 40:88] = 0
        q, dk, dv = _drafts(form, dtype)
        q[..., 40:88] *= 1000
        dk[..., 40:88] = 0
        p, cache, hc = cache_of(K, k.to(dtype), v.to(dtype), [300] * B, bits, rotate=0)
        check_tree(K, p, cache, hc, q, dk, dv, dtype, 300, first=2)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gain", [2.0 ** 60, 2.0 ** -60, 2.0 ** 104, 2.0 ** -104])
def test_keys_against_queries(K, bits, dtype, gain):
    """Keys of any magnitude with queries that bring the logits back: steps and queries outside the powers of two that the halves go by.
    (Powers of two, so that every product is what it is at 1.)"""
    for form in (FP32,) if dtype == torch.float32 else FORMS:
        B, H, _, _ = form
        k, v = normal((B * 300, H, 128), 30), normal((B * 300, H, 128), 31)
        p, cache, hc = cache_of(K, k.to(dtype), v.to(dtype), [300] * B, bits)
        for side in (cache.k_body, hc.k_body):  # the steps and offsets of the keys times the gain
            t = side.view(torch.float32) if side is cache.k_body else side.view(np.float32)
            t[..., -384:-128] *= gain
        for side, host in ((cache.k_resid, hc.k_resid),):
            side.copy_((side.float() * gain).to(torch.bfloat16))
            host[:] = side.view(torch.int16).cpu().numpy().view(np.uint16)
        q, dk, dv = _drafts(form, dtype)
        check_tree(K, p, cache, hc, (q.float() / gain).to(dtype), (dk.float() * gain).to(dtype), dv, dtype, 300, first=2)
