"""Caches whose tiles hold steps far apart: groups without range among small ones, single large or small tokens and
channels, keys and values of any magnitude."""
from __future__ import annotations

import numpy as np
import torch

from gpu_util import check_output, host_cache
from serving_util import SCALE, f64, tree, tree_reference


def cache_of(K, k, v, lens, bits, aux=0, rotate=1):
    """A cache prefilled with the given keys and values ([tokens, n_kv, 128], the sequences one after the other);
    (params, cache, host copy)."""
    p = K.kvarn_params_init(bits, aux_format=aux, rotate=rotate)
    cache = K.Cache(p, len(lens), k.shape[1], max(max(n // 128 for n in lens), 1))
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    K.kvarn_prefill(p, cache, k.contiguous(), v.contiguous(), K.KVARN_BF16 if k.dtype == torch.bfloat16 else K.KVARN_F32, cu, max(lens))
    torch.cuda.synchronize()
    return p, cache, host_cache(cache)


def normal(shape, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def check_tree(K, p, cache, hc, q, k, v, dtype, max_len, tol=None, first=None, scale=SCALE):
    """The call in order of a chain, the first sequences against 64 bits."""
    out = torch.zeros(q.shape, device="cuda", dtype=dtype)
    tree(K, p, cache, q, k, v, None, None, out, max_len, scale)
    torch.cuda.synchronize()
    n = q.shape[0] if first is None else first
    ref = tree_reference(hc, q[:n], k[:n], v[:n], None, None, scale)
    assert np.isfinite(f64(out)).all()
    check_output(f64(out)[:n], ref, dtype == torch.bfloat16, tol or (2e-3 if dtype == torch.bfloat16 else 2e-5))
    return out
