"""Steps of a serving program with all its parts: prompts arrive in a ragged batch, the token map says where they belong, the
pool gives their sequences blocks, drafts of a tree are turned to their positions on three axes and attended, the model's rows
decide which of them are accepted, these enter the cache, and sequences that end give their blocks back.  The paged
cache is held against a dense one that takes the same calls, the decisions against the definition."""
import numpy as np
import pytest
import torch

from serving_util import SCALE
from test_gpu_pool import Model, same
from verify_util import walk

pytestmark = pytest.mark.gpu

B, H, G, T, V = 5, 2, 4, 9, 1003


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    torch.cuda.set_device(0)
    return kvarn


def _trees(rng):
    parent = np.zeros((B, T), np.int32)
    mask, depth = np.zeros((B, T), np.int64), np.zeros((B, T), np.int32)
    for b in range(B):
        for i in range(T):
            up = int(rng.integers(0, i)) if i else -1
            parent[b, i] = up
            mask[b, i] = (mask[b, up] if i else 0) | 1 << i
            depth[b, i] = depth[b, up] + 1 if i else 0
    return parent, mask, depth


@pytest.mark.parametrize("bits,aux,n_sink", [(2, 0, 0), (4, 1, 16)])
def test_steps(K, bits, aux, n_sink):
    rng = np.random.default_rng(bits)
    gen = torch.Generator(device="cuda").manual_seed(bits)
    i32 = dict(dtype=torch.int32, device="cuda")
    p = K.kvarn_params_init(bits, n_sink=n_sink, aux_format=aux)
    dense, paged = K.Cache(p, B, H, 12), K.Cache(p, B, H, 12, n_phys=26)
    pool, model = K.BlockPool(paged), Model(B, 12, 26, n_sink)
    rope = K.AxesRope(128, (24, 20, 20), K.KVARN_AXES_IN_TURN, 10000.0)
    head = torch.randn((H * G * 128, V), generator=gen, device="cuda") * 0.3
    length, drafted = np.zeros(B, np.int64), 0
    for step in range(14):
        if step % 5 == 0:  # all sequences end, others begin; one of them without a prompt
            counts = [int(rng.integers(1, 700)) if b != step % B else 0 for b in range(B)]
            total = sum(counts)
            cu = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), **i32)
            length[:] = counts
            new = torch.from_numpy(length.astype(np.int32)).cuda()
            K.kvarn_assign_blocks(p, paged, pool, new, 0)
            model.step(length)
            same(paged, pool, model)
            seq, pos, row = torch.empty(total, **i32), torch.empty(total, **i32), torch.empty(total, dtype=torch.int64, device="cuda")
            K.kvarn_token_map(p, paged, cu, None, total, seq, pos, row)
            k = torch.randn((total, H, 128), generator=gen, device="cuda").to(torch.bfloat16)
            v = torch.randn((total, H, 128), generator=gen, device="cuda").to(torch.bfloat16)
            K.kvarn_rotary_axes(rope, rope.axes, None, 0, 0, None, 0, k, H, H * 128, k, H * 128, 1, total, pos, 1, 0, None, 1)
            for c in (dense, paged):
                K.kvarn_prefill(p, c, k, v, K.KVARN_BF16, cu, max(max(counts), 1))
            # the map's rows hold these tokens: sinks and residuals as given
            plain = [x.transpose(0, 1).reshape(H, -1, 128) for x in (paged.k_sink, paged.k_resid) if x is not None]
            plain = torch.cat(plain, 1)
            held = row < plain.shape[1]
            assert int(held.sum()) == sum(min(n, n_sink) + max(n - n_sink, 0) % 128 for n in counts)
            assert torch.equal(plain[:, row[held]], k[held].transpose(0, 1))
            body = (row[~held] - plain.shape[1]).cpu().numpy()
            s, at = seq[~held].cpu().numpy(), pos[~held].cpu().numpy() - n_sink
            assert all(body[i] == model.rows[s[i]][at[i] // 128] * 128 + at[i] % 128 for i in range(len(body)))
        K.kvarn_assign_blocks(p, paged, pool, None, T)  # room for whatever is accepted
        model.step(length, T)
        same(paged, pool, model)
        parent, mask, depth = _trees(rng)
        x = torch.randn((B, T, H * (G + 2), 128), generator=gen, device="cuda").to(torch.bfloat16)
        wide = H * (G + 2) * 128
        d = torch.from_numpy(np.stack([depth, depth // 2, depth % 2])).cuda()
        K.kvarn_rotary_axes(rope, rope.axes, x, H * G, wide, x, wide, x[:, :, H * G:], H, wide, x[:, :, H * G:], wide, 1, B * T, d, 1,
                            B * T, paged.seq_len, T)
        q, kd, vd = x[:, :, :H * G], x[:, :, H * G:H * G + H], x[:, :, H * G + H:]
        outs, m = [], torch.from_numpy(mask).cuda()
        for c in (dense, paged):
            out = torch.empty((B, T, H * G, 128), dtype=torch.float32, device="cuda")
            n = K.kvarn_tree_workspace_bytes(p, c, H * G, T, 1000)
            ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
            K.kvarn_tree_attention(p, c, H * G, T, q, wide, 1, kd, vd, wide, 1, m, None, out, H * G * 128, 0, SCALE, 1000, ws, n)
            outs.append(out)
        assert torch.equal(*outs)
        target = outs[1].view(B, T, -1) @ head
        draft = target + 0.7 * torch.randn((B, T, V), generator=gen, device="cuda")
        up = torch.from_numpy(parent).cuda()
        rows = draft.gather(1, up.clamp(min=0).long().unsqueeze(2).expand(B, T, V))
        tokens = torch.multinomial(torch.softmax(rows, 2).view(B * T, V), 1, generator=gen).view(B, T).to(torch.int32)
        u = torch.rand((B, T), generator=gen, device="cuda")
        path, n_path, nxt = torch.empty((B, T), **i32), torch.empty(B, **i32), torch.empty(B, **i32)
        n = K.kvarn_verify_workspace_bytes(B, T, V)
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        K.kvarn_verify_drafts(B, T, V, tokens, up, None, target, V, draft, V, K.KVARN_F32, K.KVARN_LOGITS, None, u, path, n_path, nxt, ws, n)
        for c in (dense, paged):
            K.kvarn_append_path(p, c, T, kd, vd, wide, 1, path, T, n_path)
        torch.cuda.synchronize()
        for b in range(B):
            w = walk(tokens[b].cpu().numpy(), parent[b], T, target[b].double().cpu().numpy(), draft[b].double().cpu().numpy(), True, 1.0,
                     u[b].double().cpu().numpy())
            if w.sure > 2.0 ** -36:
                assert path[b, :int(n_path[b])].tolist() == w.path and int(nxt[b]) == w.next
        drafted += int(n_path.sum()) - B
        length += n_path.cpu().numpy()
        assert paged.seq_len.tolist() == length.tolist() == dense.seq_len.tolist()
    assert int(paged.err_word) == 0 == int(dense.err_word) and drafted > 20
    # what the two caches hold is the same
    most = int(length.max())
    rows = []
    for c in (dense, paged):
        k, v = (torch.zeros((B, most, H, 128), device="cuda") for _ in range(2))
        K.kvarn_read_tokens(p, c, None, most, k, v, K.KVARN_F32, most * H * 128, 128, H * 128)
        rows.append((k, v))
    torch.cuda.synchronize()
    assert torch.equal(rows[0][0], rows[1][0]) and torch.equal(rows[0][1], rows[1][1])
