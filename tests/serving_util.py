"""Caches and plain 64-bit forms for the tests of rotary positions, drafted tokens and reading back."""
from __future__ import annotations

import numpy as np
import torch

import oracle
from gpu_util import host_cache

SCALE = 1.0 / np.sqrt(128.0)


def make_cache(K, lens, n_kv, bits=2, aux=0, n_sink=0, rotate=1, paged=False, extra_blocks=0, seed=0, gain=1.0):
    """A cache prefilled with random prompts of the given lengths; (params, cache, its dense host copy)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    total = max(int(sum(lens)), 1)
    k = gain * torch.randn((total, n_kv, 128), generator=g, device="cuda")
    k = (k * torch.exp(0.5 * torch.randn((1, n_kv, 128), generator=g, device="cuda"))).to(torch.bfloat16)
    v = torch.randn((total, n_kv, 128), generator=g, device="cuda").to(torch.bfloat16)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    p = K.kvarn_params_init(bits, n_sink=n_sink, aux_format=aux, rotate=rotate)
    blocks = [max(n - n_sink, 0) // 128 for n in lens]
    dense = K.Cache(p, len(lens), n_kv, max(max(blocks) + extra_blocks, 1))
    # rows that no call may use
    for x in (dense.k_resid, dense.v_resid, dense.k_sink, dense.v_sink):
        if x is not None:
            x.fill_(float("nan"))
    K.kvarn_prefill(p, dense, k, v, K.KVARN_BF16, cu, max(max(lens), 1))
    torch.cuda.synchronize()
    hc = host_cache(dense)
    if not paged:
        return p, dense, hc
    pool = sum(blocks) + extra_blocks * len(lens) + 1
    cache = K.Cache(p, len(lens), n_kv, dense.max_blocks, n_phys=pool)
    ids = torch.randperm(pool, generator=torch.Generator().manual_seed(seed)).tolist()
    for b, n in enumerate(blocks):
        for j in range(min(n + extra_blocks, dense.max_blocks)):
            i = ids.pop()
            cache.block_table[b, j] = i
            cache.k_body[i] = dense.k_body[b, :, j]
            cache.v_body[i] = dense.v_body[b, :, j]
    for name in ("k_resid", "v_resid", "k_sink", "v_sink", "seq_len"):
        if getattr(dense, name) is not None:
            getattr(cache, name).copy_(getattr(dense, name))
    return p, cache, hc


def random_masks(batch, n_draft, rng):
    """Ancestor masks of random trees, [batch, n_draft] uint64 as int64."""
    m = np.zeros((batch, n_draft), dtype=np.uint64)
    for b in range(batch):
        for i in range(n_draft):
            parent = rng.integers(-1, i) if i else -1
            m[b, i] = (m[b, parent] if parent >= 0 else np.uint64(0)) | np.uint64(1 << i)
    return torch.from_numpy(m.view(np.int64)).cuda()


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def tree_reference(hc, q, k, v, mask, live, scale=SCALE):
    """The attention of the drafts in 64 bits over the host cache: [batch, n_draft, n_q, 128], rows behind `live`
    zero.  mask: [batch, n_draft] int64 or None (a chain)."""
    B, T, n_q, _ = q.shape
    g = n_q // hc.n_kv
    qq, kk, vv = f64(q), f64(k.to(torch.bfloat16)), f64(v.to(torch.bfloat16))
    out = np.zeros(qq.shape)
    for b in range(B):
        n = T if live is None else min(max(int(live[b]), 0), T)
        for h in range(hc.n_kv):
            K0, V0 = oracle.gather_stream(hc, b, h)
            for i in range(n):
                m = (2 << i) - 1 if mask is None else int(mask[b, i]) & (2**64 - 1)
                js = [j for j in range(n) if (m >> j) & 1]
                if not js and len(K0) == 0:
                    continue
                Ka, Va = np.concatenate([K0, kk[b, js, h]]), np.concatenate([V0, vv[b, js, h]])
                z = qq[b, i, h * g:(h + 1) * g] @ Ka.T * scale
                e = np.exp(z - z.max(1, keepdims=True))
                out[b, i, h * g:(h + 1) * g] = (e / e.sum(1, keepdims=True)) @ Va
    return out


def dt(K, t):
    return K.KVARN_F32 if t.dtype == torch.float32 else K.KVARN_BF16


def tree(K, p, cache, q, k, v, mask, live, out, max_len, scale=SCALE):
    """The call on contiguous tensors, with a workspace of its own."""
    B, T, n_q, _ = q.shape
    n = K.kvarn_tree_workspace_bytes(p, cache, n_q, T, max_len)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    K.kvarn_tree_attention(p, cache, n_q, T, q, n_q * 128, dt(K, q), k, v, cache.n_kv * 128, dt(K, k), mask, live, out,
                           n_q * 128, dt(K, out), scale, max_len, ws, n)
    return ws
