"""Operators of a serving step around the packed cache whose time is measured: the verification of drafted
tokens, rotary positions with several axes, block tables and the map of a ragged batch's tokens.

A case is a dict of sizes and options.  Its kinds:

  verify   one ``kvarn_verify_drafts`` call: which drafts of every sequence's tree are accepted, and the
           token that follows them.  Draft 0 is certain; with one draft the call samples the next token.
  axes     one ``kvarn_rotary_axes`` call on the queries and keys of one layer's tokens.
  blocks   one ``kvarn_assign_blocks`` call: sequences grow, end and begin, and the block table follows.  The
           table and the ring of free blocks are set back first, so that every pass moves the same blocks.
  map      one ``kvarn_token_map`` call: sequence, position and cache row of every token of a ragged batch.

With ``own`` false ``run`` computes the same in plain torch operations; ``exact`` gives the results that are not
whole numbers (the rotated rows) in 64 bits from the definition.
"""
import math

import torch

own = False

D = 128  # channels of a token, tokens of a group


def listed():
    v, a, b, m = dict(kind="verify"), dict(kind="axes"), dict(kind="blocks"), dict(kind="map")
    bf, f32 = dict(dtype="bf16"), dict(dtype="fp32")
    return [
        # the smallest: the next token of one sequence from its logits
        dict(name="verify_b1_next", **v, batch=1, drafts=1, vocab=32000, tree=False, mode="drawn", logits=True, **bf),
        # chains of a serving batch, from probabilities that a sampler has filtered
        dict(name="verify_chain_b64", **v, batch=64, drafts=8, vocab=128000, tree=False, mode="drawn", logits=False, **f32),
        # the largest: a big batch's short chains straight from the logits
        dict(name="verify_chain_b256_logits", **v, batch=256, drafts=5, vocab=131072, tree=False, mode="drawn", logits=True, **bf),
        # trees with siblings drawn from the draft's distribution, an odd vocabulary, rows at odd places
        dict(name="verify_tree_b16", **v, batch=16, drafts=24, vocab=100003, tree=True, mode="drawn", logits=False, **f32),
        # wide trees of a greedy batch
        dict(name="verify_greedy_b48", **v, batch=48, drafts=64, vocab=65537, tree=True, mode="greedy", logits=True, **bf),
        # candidates without a distribution of their own, one sequence, where latency counts
        dict(name="verify_fixed_b4", **v, batch=4, drafts=13, vocab=50021, tree=True, mode="fixed", logits=True, **f32),
        # one new token of each of 64 sequences, 32 / 8 heads, three axes in turn
        dict(name="axes_decode_b64", **a, tokens=64, n_q=32, n_kv=8, rot=D, half=True, sections="24,20,20", turns=True,
             inverse=False, **bf),
        # a prompt of text and video frames
        dict(name="axes_video_16k", **a, tokens=16407, n_q=32, n_kv=8, rot=D, half=True, sections="16,24,24", turns=False,
             inverse=False, **bf),
        # image rows, height and width, half of the head, interleaved pairs, fp32, taken off again (or a gradient)
        dict(name="axes_image_fp32", **a, tokens=5003, n_q=16, n_kv=16, rot=64, half=False, sections="16,16", turns=False,
             inverse=True, **f32),
        # the streaming workload's batch, one token more each
        dict(name="blocks_decode_b64", **b, batch=64, tokens=33000, sink=0, moving=False),
        # a large batch in which prompts arrive and sequences end
        dict(name="blocks_arrive_b1024", **b, batch=1024, tokens=131000, sink=128, moving=True),
        # the tokens of a step's prompts, half a million of them
        dict(name="map_prompts", **m, batch=193, tokens=524309, sink=100, start=700, paged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["verify", "verify", "verify", "verify", "axes", "axes", "blocks", "map"])
    dtype = rng.choice(["bf16", "fp32"])
    if kind == "verify":
        drafts, vocab = rng.choice([1, _log(rng, 1, 64), _log(rng, 2, 64)]), _log(rng, 1000, 200000)
        batch = min(_log(rng, 1, 256), max(1, 160000000 // (drafts * vocab)))
        return dict(kind=kind, batch=batch, drafts=drafts, vocab=vocab, tree=rng.random() < 0.5,
                    mode=rng.choice(["drawn", "drawn", "greedy", "fixed"]), logits=rng.random() < 0.5, dtype=dtype)
    if kind == "axes":
        n_kv = rng.choice([1, 2, 4, 8, 8])
        n_q, half = n_kv * rng.choice([1, 2, 4, 4, 5, 8]), rng.random() < 0.6
        sections = rng.choice(["16,24,24", "24,20,20", "22,21,21", "32,32", "16,16", "8,12,12", "16,16,16,16", "48"])
        return dict(kind=kind, tokens=min(_log(rng, 1, 16000), 600000 // (n_q + n_kv)), n_q=n_q, n_kv=n_kv,
                    rot=2 * sum(_sections(sections)), half=half, sections=sections, turns=rng.random() < 0.5,
                    inverse=rng.random() < 0.3, dtype=dtype)
    batch, sink = _log(rng, 1, 1024), rng.choice([0, 0, 128, 100])
    if kind == "blocks":
        return dict(kind=kind, batch=batch, tokens=_log(rng, 300, 131000), sink=sink, moving=rng.random() < 0.6)
    return dict(kind=kind, batch=batch, tokens=_log(rng, 100, 500000), sink=sink, start=rng.choice([0, 700, 30000]),
                paged=rng.random() < 0.6)


# ---- sizes ----------------------------------------------------------------------------------


def _sections(text):
    return [int(x) for x in text.split(",")]


def _es(case):
    return 4 if case["dtype"] == "fp32" else 2


def _dt(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _lengths(case):
    """Tokens of each sequence before and after a step: one more each, or (moving) a quarter ends, a quarter begins and
    the others grow by up to a group."""
    n, t = case["batch"], case["tokens"]
    before = [max(1, int(t * 16.0 ** -((i * 0.6180339887498949) % 1.0))) for i in range(n)]
    if not case["moving"]:
        return before, [x + 1 for x in before]
    after = [0 if i % 4 == 1 else x + (0 if i % 4 == 2 else (i * 37) % 160) for i, x in enumerate(before)]
    return [0 if i % 4 == 2 else x for i, x in enumerate(before)], after


def _need(case, lengths):
    return [max(x - case["sink"], 0) // D for x in lengths]


def _counts(case):
    """Tokens of each sequence of a ragged batch, some of them none."""
    n, t = case["batch"], case["tokens"]
    share = [0.0 if i % 7 == 5 else 0.1 + (i * 0.6180339887498949) % 1.0 for i in range(n)]
    total = sum(share)
    count = [int(t * x / total) for x in share]
    count[0] += t - sum(count)
    return count


def work(case):
    kind = case["kind"]
    if kind == "verify":
        rows = case["batch"] * case["vocab"]
        if case["logits"] or case["mode"] == "greedy":  # the first node's row and, where there are drafts, mostly another's
            pairs = 1 if case["drafts"] == 1 else 2
        else:
            pairs = 1
        both = 2 if case["mode"] == "drawn" and case["drafts"] > 1 else 1
        return {"bytes": rows * _es(case) * pairs * both + case["batch"] * case["drafts"] * 16, "flops": rows * pairs * both * 4}
    if kind == "axes":
        rows, axes = case["tokens"] * (case["n_q"] + case["n_kv"]), len(_sections(case["sections"]))
        return {"bytes": rows * D * 2 * _es(case) + case["tokens"] * 4 * axes + case["rot"] * 4, "flops": rows * case["rot"] * 3}
    if kind == "blocks":
        before, after = [_need(case, x) for x in _lengths(case)]
        took = sum(max(y - x, 0) for x, y in zip(before, after))
        gave = sum(max(x - y, 0) for x, y in zip(before, after))
        return {"bytes": case["batch"] * 12 + took * 8 + gave * 12 + 8, "flops": case["batch"] * 4}
    blocks = sum(-(-x // D) for x in _counts(case))
    return {"bytes": case["tokens"] * 16 + case["batch"] * 8 + blocks * 4, "flops": case["tokens"] * 4}


# ---- inputs -----------------------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1009 + 31)
    return g


def _trees(case, gen):
    """The draft that each draft hangs on [batch, drafts] (-1: the first), and which child of that one it is."""
    b, t = case["batch"], case["drafts"]
    r = torch.rand((b, t), generator=gen, device="cuda").cpu()
    parent, nth = torch.full((b, t), -1, dtype=torch.int64), torch.zeros((b, t), dtype=torch.int64)
    children = torch.zeros((b, t), dtype=torch.int64)
    for i in range(1, t):
        # near the root more often than not, so that drafts have siblings
        at = (r[:, i] ** 2 * i).long() if case["tree"] else torch.full((b,), i - 1)
        parent[:, i] = at
        nth[:, i] = children.gather(1, at.view(-1, 1)).view(-1)
        children.scatter_add_(1, at.view(-1, 1), torch.ones((b, 1), dtype=torch.int64))
    return parent, nth


def _verify_state(case, seed):
    gen, b, t, v = _gen(seed), case["batch"], case["drafts"], case["vocab"]
    parent, nth = _trees(case, gen)
    # peaked logits of a model, and of a smaller one that agrees with it for the most part
    target = torch.randn((b, t, v), generator=gen, device="cuda").mul_(4.0)
    draft = torch.randn((b, t, v), generator=gen, device="cuda").mul_(0.7).add_(target)
    tokens = torch.randint(0, v, (b, t), generator=gen, device="cuda", dtype=torch.int32)
    for i in range(1, t):
        rows = draft[torch.arange(b, device="cuda"), parent[:, i].cuda()]
        if case["mode"] == "drawn":
            rows = rows - torch.log(-torch.log(torch.rand((b, v), generator=gen, device="cuda").clamp_(1e-12, 1 - 1e-7)))
            tokens[:, i] = rows.argmax(1).to(torch.int32)
        else:
            best = rows.topk(min(8, v), 1)[1]
            tokens[:, i] = best.gather(1, (nth[:, i].cuda() % best.shape[1]).view(-1, 1)).view(-1).to(torch.int32)
        del rows
    form = (lambda x: x.to(_dt(case))) if case["logits"] else (lambda x: torch.softmax(x, 2).to(_dt(case)))
    s = {"case": case, "tokens": tokens, "parent": parent.to(torch.int32).cuda() if case["tree"] else None, "target": form(target)}
    del target
    s["draft"] = form(draft) if case["mode"] == "drawn" and t > 1 else None
    del draft
    # temperatures of a batch, for logits
    s["scale"] = (0.8 + 0.6 * torch.rand((b,), generator=gen, device="cuda")) if case["logits"] and case["mode"] != "greedy" else None
    s["u"] = torch.rand((b, t), generator=gen, device="cuda") if case["mode"] != "greedy" else None
    s["live"] = torch.tensor([t - (i * 5) % max(1, t // 2) for i in range(b)], dtype=torch.int32, device="cuda") if case["tree"] else None
    i32 = dict(dtype=torch.int32, device="cuda")
    s["path"], s["n_path"], s["next"] = torch.zeros((b, t), **i32), torch.zeros(b, **i32), torch.zeros(b, **i32)
    if own:
        from paper_2606_03458_amd import kvarn as K
        n = K.kvarn_verify_workspace_bytes(b, t, v)
        s.update(K=K, ws=torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"))
    return s


def _axis_of(case):
    """The axis of each pair: the sections one after the other, or in turn as long as each has pairs left."""
    sections = _sections(case["sections"])
    if not case["turns"]:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    left, out, a = list(sections), [], 0
    while sum(left):
        if left[a]:
            out.append(a)
            left[a] -= 1
        a = (a + 1) % len(sections)
    return out


def _axes_state(case, seed):
    gen, dt, n, n_q, n_kv = _gen(seed), _dt(case), case["tokens"], case["n_q"], case["n_kv"]
    x = torch.randn((n, n_q + 2 * n_kv, D), generator=gen, device="cuda").to(dt)  # a fused projection's output
    axes = len(_sections(case["sections"]))
    # a text, then frames of a grid of patches behind it: time, height and width, each from the text's end on
    text, high, wide = torch.randint(1, 60, (3,), generator=gen, device="cuda").tolist()
    i = torch.arange(n, device="cuda")
    j = (i - text).clamp(min=0)
    grid = torch.stack([j // (high * wide), j // wide % high, j % wide, j % 5][:axes] if axes != 2 else [j // wide, j % wide])
    pos = torch.where(i < text, i, text + grid).to(torch.int32).contiguous()
    far = int(torch.randint(0, 50000, (1,), generator=gen, device="cuda"))
    freq = torch.tensor([500000.0 ** (-2.0 * k / case["rot"]) for k in range(case["rot"] // 2)], dtype=torch.float64, device="cuda")
    s = {"case": case, "x": x, "q": x[:, :n_q], "k": x[:, n_q:n_q + n_kv], "pos": pos, "freq": freq,
         "start": torch.full((1,), far, dtype=torch.int32, device="cuda"),
         "axis": torch.tensor(_axis_of(case), device="cuda")}
    s["q_out"], s["k_out"] = torch.zeros((n, n_q, D), dtype=dt, device="cuda"), torch.zeros((n, n_kv, D), dtype=dt, device="cuda")
    if own:
        from paper_2606_03458_amd import kvarn as K
        layout = K.KVARN_ROPE_HALF if case["half"] else K.KVARN_ROPE_INTERLEAVED
        order = K.KVARN_AXES_IN_TURN if case["turns"] else K.KVARN_AXES_SECTIONS
        s.update(K=K, rope=K.kvarn_rope(case["rot"], layout, 1.0, freq.data_ptr()),
                 axes=K.kvarn_rope_axes_init(case["rot"], _sections(case["sections"]), order))
    return s


def _cache_of(case, max_blocks, table, n_phys):
    """The library's parameters and a cache of which only the table and the sizes are used."""
    from paper_2606_03458_amd import kvarn as K
    p = K.kvarn_params_init(2, n_sink=case["sink"])
    cache = K.Cache(p, case["batch"], 1, 1, n_phys=1 if table is not None else 0)
    cache.max_blocks = max_blocks
    if table is not None:
        cache.block_table, cache.n_phys = table, n_phys
    return K, p, cache


def _blocks_state(case, seed):
    gen, b = _gen(seed), case["batch"]
    before, after = _lengths(case)
    have, need = _need(case, before), _need(case, after)
    wide = max(max(have), max(need), 1) + 3
    pool = sum(max(x, y) for x, y in zip(have, need)) + 5
    ids = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
    held = torch.tensor(have, device="cuda")
    # one buffer, so that one copy sets it back: the ring of free blocks, its first and count, blocks held, the table
    sizes = [pool, 4, b, b * wide]
    saved = torch.zeros(sum(sizes), dtype=torch.int32, device="cuda")
    now = torch.zeros_like(saved)

    def parts(x):
        ring, at, count, table = x.split(sizes)
        return {"ring": ring, "at": at, "count": count, "table": table.view(b, wide)}

    p = parts(saved)
    free, first = pool - sum(have), pool // 3
    p["ring"][(first + torch.arange(free, device="cuda")) % pool] = ids[:free]
    p["at"][0], p["at"][1] = first, free
    p["count"].copy_(held)
    p["table"].fill_(-1)
    mine = torch.arange(wide, device="cuda") < held.view(-1, 1)
    p["table"][mine] = ids[free:]
    s = {"case": case, "saved": saved, "now": now, **parts(now), "pool": pool, "lengths": torch.tensor(after, dtype=torch.int32, device="cuda")}
    if own:
        K, q, cache = _cache_of(case, wide, s["table"], pool)
        s.update(K=K, p=q, cache=cache, handle=K.kvarn_block_pool(s["ring"].data_ptr(), s["at"].data_ptr(), s["count"].data_ptr()))
    return s


def _map_state(case, seed):
    gen, b, n = _gen(seed), case["batch"], case["tokens"]
    count = torch.tensor(_counts(case), device="cuda")
    start = torch.randint(0, case["start"] + 1, (b,), generator=gen, device="cuda")
    ends = torch.cumsum(count, 0)
    wide = int(torch.clamp(start + count - case["sink"], min=0).max()) // D + 2
    s = {"case": case, "cu": torch.cat([ends.new_zeros(1), ends]).to(torch.int32), "start": start.to(torch.int32), "wide": wide,
         "table": torch.randint(0, b * wide, (b, wide), generator=gen, device="cuda", dtype=torch.int32) if case["paged"] else None}
    for name, dt in (("seq", torch.int32), ("pos", torch.int32), ("row", torch.int64)):
        s[name] = torch.zeros(n, dtype=dt, device="cuda")
    if own:
        s["K"], s["p"], s["cache"] = _cache_of(case, wide, s["table"], b * wide)
    return s


def prepare(case, seed):
    return {"verify": _verify_state, "axes": _axes_state, "blocks": _blocks_state, "map": _map_state}[case["kind"]](case, seed)


# ---- the calls, and their plain form -----------------------------------------------------------


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"verify": _own_verify, "axes": _own_axes, "blocks": _own_blocks, "map": _own_map}[kind](state)
    return {"verify": _plain_verify, "axes": _plain_axes, "blocks": _plain_blocks, "map": _plain_map}[kind](state)


def _own_verify(s):
    case, K = s["case"], s["K"]
    K.kvarn_verify_drafts(case["batch"], case["drafts"], case["vocab"], s["tokens"], s["parent"], s["live"], s["target"],
                          case["vocab"], s["draft"], case["vocab"] if s["draft"] is not None else 0,
                          0 if case["dtype"] == "fp32" else 1, K.KVARN_LOGITS if case["logits"] else K.KVARN_PROBABILITIES,
                          s["scale"], s["u"], s["path"], s["n_path"], s["next"], s["ws"], s["ws"].numel())
    return s["path"], s["n_path"], s["next"]


def _own_axes(s):
    case = s["case"]
    n_q, n_kv, row = case["n_q"], case["n_kv"], s["x"].shape[1] * D
    s["K"].kvarn_rotary_axes(s["rope"], s["axes"], s["q"], n_q, row, s["q_out"], n_q * D, s["k"], n_kv, row, s["k_out"], n_kv * D,
                             0 if case["dtype"] == "fp32" else 1, case["tokens"], s["pos"], 1, case["tokens"], s["start"],
                             case["tokens"], int(case["inverse"]))
    return s["q_out"], s["k_out"]


def _own_blocks(s):
    s["now"].copy_(s["saved"])
    s["K"].kvarn_assign_blocks(s["p"], s["cache"], s["handle"], s["lengths"], 0)
    return s["table"], s["count"], s["ring"], s["at"][:2]


def _own_map(s):
    s["K"].kvarn_token_map(s["p"], s["cache"], s["cu"], s["start"], s["case"]["tokens"], s["seq"], s["pos"], s["row"])
    return s["seq"], s["pos"], s["row"]


def _weights(s, rows):
    """Probabilities of rows in 64 bits: a decision may lie next to a border."""
    x = rows.double()
    if not s["case"]["logits"]:
        return x
    if s["scale"] is not None:
        x = x * s["scale"].double().view([-1] + [1] * (x.dim() - 1))
    x = torch.exp(x - x.amax(-1, keepdim=True))
    return x / x.sum(-1, keepdim=True)


def _plain_verify(s):
    case, tok = s["case"], s["tokens"].long()
    b, t, v = case["batch"], case["drafts"], case["vocab"]
    dev, every, mode = tok.device, torch.arange(b, device=tok.device), case["mode"]
    step = torch.arange(t, device=dev)
    parent = s["parent"].long() if s["parent"] is not None else (step - 1).expand(b, t)
    live = s["live"].long() if s["live"] is not None else torch.full((b,), t, device=dev)
    node, count = torch.zeros(b, dtype=torch.long, device=dev), torch.ones(b, dtype=torch.long, device=dev)
    path = torch.full((b, t), -1, dtype=torch.long, device=dev)
    path[:, 0] = 0
    if mode == "greedy":
        x = s["target"].float()
        best = torch.where(x == x.amax(2, keepdim=True), torch.arange(v, device=dev), v).amin(2)
    else:
        u = s["u"].double()
        left = torch.ones(b, dtype=torch.float64, device=dev)  # what the children refused so far leave of the node's row
        taken, p, q = torch.zeros(b, dtype=torch.float64, device=dev), None, None
        gone = torch.zeros((b, v), dtype=torch.bool, device=dev) if mode == "fixed" and t > 1 else None
        if t > 1:  # each draft's token in its parent's rows
            up = parent.clamp(min=0)
            at = _weights(s, s["target"])[every.view(-1, 1), up, tok]
            by = _weights(s, s["draft"])[every.view(-1, 1), up, tok] if mode == "drawn" else None
    for j in range(1, t):
        mine = (parent[:, j] == node) & (j < live)
        if mode == "greedy":
            ok = mine & (tok[:, j] == best[every, node])
        elif mode == "drawn":
            ok = mine & (u[:, j] * left * by[:, j] < at[:, j] - taken * by[:, j])
        else:
            fresh = ~gone[every, tok[:, j]]
            ok = mine & fresh & (u[:, j] * left < at[:, j])
        node, count = torch.where(ok, j, node), count + ok
        path.scatter_(1, torch.where(ok, count - 1, 0).view(-1, 1), torch.where(ok, j, 0).view(-1, 1))
        if mode == "greedy":
            continue
        no = mine & ~ok
        if mode == "drawn":
            taken = torch.where(ok, 0.0, torch.where(no, taken + left, taken))
            if s["parent"] is not None:  # (a chain's draft has no sibling that needs what is left)
                p, q = _weights(s, s["target"][every, node]), _weights(s, s["draft"][every, node])
                rest = (p - taken.view(-1, 1) * q).clamp(min=0).sum(1)
                left = torch.where(taken > 0, rest, 1.0)
            else:
                left = torch.ones_like(left)
        else:
            gone &= ~ok.view(-1, 1)
            left = torch.where(ok, 1.0, torch.where(no & fresh, left - at[:, j], left))
            gone[every, tok[:, j]] |= no
    if mode == "greedy":
        token = best[every, node]
    else:
        w = p = _weights(s, s["target"][every, node])
        if mode == "drawn" and t > 1:
            w = (p - taken.view(-1, 1) * _weights(s, s["draft"][every, node])).clamp(min=0)
            w = torch.where(w.sum(1, keepdim=True) > 0, w, p)
        elif t > 1:
            w = torch.where(gone, 0.0, p)
        w = torch.cumsum(w, 1)
        token = (w <= u[:, :1] * w[:, -1:]).sum(1)
    s["path"].copy_(path), s["n_path"].copy_(count), s["next"].copy_(token)
    return s["path"], s["n_path"], s["next"]


def _plain_axes(s):
    case, dt = s["case"], _dt(s["case"])
    rot, h = case["rot"], case["rot"] // 2
    pos = s["pos"].double() + s["start"].double()
    angle = (pos[s["axis"]].t() * s["freq"]).unsqueeze(1)
    cos, sin = torch.cos(angle).float(), (torch.sin(angle) * (-1.0 if case["inverse"] else 1.0)).float()
    out = []
    for name in ("q", "k"):
        x = s[name].float()
        if case["half"]:
            a, b = x[..., :h], x[..., h:rot]
            y = torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., rot:]], 2)
        else:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            y = torch.stack([a * cos - b * sin, a * sin + b * cos], 3).flatten(2)
            y = torch.cat([y, x[..., rot:]], 2)
        s[name + "_out"].copy_(y.to(dt))
        out.append(s[name + "_out"])
    return tuple(out)


def _plain_blocks(s):
    s["now"].copy_(s["saved"])
    case, pool = s["case"], s["pool"]
    have, need = s["count"].long(), torch.clamp(s["lengths"].long() - case["sink"], min=0) // D
    first, free = s["at"][0].long(), s["at"][1].long()
    more, less = torch.clamp(need - have, min=0), torch.clamp(have - need, min=0)
    took, gave = torch.cumsum(more, 0), torch.cumsum(less, 0)
    j = torch.arange(s["table"].shape[1], device=have.device)
    old, table = s["table"], s["table"]
    # what is given back goes behind the free ones, and what is taken comes off the front
    back = (j >= need.view(-1, 1)) & (j < have.view(-1, 1))
    at = free + (gave - less - need).view(-1, 1) + j
    ring = torch.cat([s["ring"], s["ring"].new_zeros(1)]).clone()
    ring[torch.where(back, (first + at) % pool, pool)] = old
    take = (j >= have.view(-1, 1)) & (j < need.view(-1, 1))
    from_ = (first + (took - more - have).view(-1, 1) + j) % pool
    new = torch.where(take, ring[torch.where(take, from_, pool)], torch.where(back, -1, table))
    # (a block that is handed on at once does not pass through the ring)
    stays = torch.where(back & (at >= took[-1]), (first + at) % pool, pool)
    kept = torch.cat([s["ring"], s["ring"].new_zeros(1)])
    kept[stays] = old
    s["ring"].copy_(kept[:pool])
    s["table"].copy_(new)
    s["count"].copy_(need)
    s["at"][0].copy_((first + took[-1]) % pool)
    s["at"][1].copy_(free + gave[-1] - took[-1])
    return s["table"], s["count"], s["ring"], s["at"][:2]


def _plain_map(s):
    case, b, n = s["case"], s["case"]["batch"], s["case"]["tokens"]
    cu, sink = s["cu"].long(), s["case"]["sink"]
    i = torch.arange(n, device=cu.device)
    seq = torch.searchsorted(cu[1:], i, right=True)
    start = s["start"].long()[seq]
    pos, length = start + i - cu[seq], start + cu[seq + 1] - cu[seq]
    full = torch.clamp(length - sink, min=0) // D
    blk = torch.clamp(pos - sink, min=0) // D
    tile = s["table"].long()[seq, blk] if case["paged"] else seq * s["wide"] + blk
    # rows are counted over the sinks, then the residuals, then the body
    row = b * (sink + D) + tile * D + (pos - sink) % D
    row = torch.where(blk >= full, b * sink + seq * D + (pos - sink) % D, row)
    row = torch.where(pos < sink, seq * sink + pos, row)
    s["seq"].copy_(seq), s["pos"].copy_(pos), s["row"].copy_(row)
    return s["seq"], s["pos"], s["row"]


# ---- the same results in 64 bits ---------------------------------------------------------------


def exact(case, seed):
    if case["kind"] != "axes":
        return None  # whole numbers
    s = _axes_state(case, seed)
    rot, h, axis = case["rot"], case["rot"] // 2, _axis_of(case)
    far = int(s["start"])
    out = []
    for name in ("q", "k"):
        x = s[name].double()
        y = x.clone()
        for i in range(h):
            angle = (s["pos"][axis[i]].double() + far) * float(s["freq"][i])
            turn = torch.polar(torch.ones_like(angle), -angle if case["inverse"] else angle).view(-1, 1)
            a, b = (i, i + h) if case["half"] else (2 * i, 2 * i + 1)
            z = torch.complex(x[..., a], x[..., b]) * turn
            y[..., a], y[..., b] = z.real, z.imag
        out.append(y)
    return tuple(out)
