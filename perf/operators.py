"""Cases and plain forms of the operators around a verification call: the attention of drafted rows over a
paged cache, the cache's writes, and the changes made to logits before a race.

`run` computes with elementary torch operations in 32 bits where `own` is false, and makes the library's
calls where it is true.  Shapes: Hq query heads share Hkv key and value heads; a cache is
[pages, page, Hkv, D], its block table [B, pages of a sequence]; `ctx` is the longest context of the batch.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

# Draft trees by name: parents of nodes 0..N, node 0 the root.
TREES = {
    "4x4": (-1, 0, 0, 0, 0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12),
    "shared": (-1, 0, 1, 2, 2, 2, 3, 4, 5),            # three sequences, the first two tokens in common
    "star8": (-1,) + (0,) * 8,
    "greedy24": (-1, 0, 1, 2, 3, 4, 3, 2, 1, 8, 9, 8, 0, 12, 13, 12, 0, 16, 17, 16, 0, 20, 0, 22, 0),
}


def listed():
    return [
        # one token of a draft model, one user: latency
        dict(name="attention one token", op="attention", dtype="bf16", B=1, R=1, Hq=32, Hkv=8, D=128, page=16, ctx=1000,
             tree="", window=0, sinks=0, ragged=False),
        # a draft tree evaluated by the target model, a serving batch
        dict(name="attention tree", op="attention", dtype="bf16", B=32, R=17, Hq=32, Hkv=8, D=128, page=64, ctx=4095,
             tree="4x4", window=0, sinks=0, ragged=False),
        # a piece of a long prompt
        dict(name="attention prompt", op="attention", dtype="bf16", B=2, R=2048, Hq=32, Hkv=8, D=128, page=64, ctx=8192,
             tree="", window=0, sinks=0, ragged=False),
        # a drafted chain over long streams: window and first tokens
        dict(name="attention window", op="attention", dtype="bf16", B=16, R=6, Hq=32, Hkv=8, D=64, page=16, ctx=20011,
             tree="", window=4096, sinks=4, ragged=True),
        # 32-bit model of a check run, a head each, odd page size and lengths
        dict(name="attention f32", op="attention", dtype="f32", B=8, R=5, Hq=16, Hkv=16, D=64, page=20, ctx=777,
             tree="", window=0, sinks=0, ragged=True),
        # one row per sequence of a serving batch: latency
        dict(name="append token", op="append", dtype="bf16", B=64, R=1, Hkv=8, D=128, page=16, ctx=300, ragged=False),
        # a piece of a prompt, every row written
        dict(name="append prompt", op="append", dtype="bf16", B=8, R=2048, Hkv=8, D=128, page=64, ctx=700, ragged=True),
        # accepted paths of a small batch, one draft model's layers
        dict(name="commit small", op="commit", dtype="bf16", B=4, layers=2, Hkv=4, D=64, page=16, ctx=200, tree="shared"),
        # accepted paths of a serving batch, all layers of the target model
        dict(name="commit layers", op="commit", dtype="bf16", B=32, layers=32, Hkv=8, D=128, page=16, ctx=90, tree="4x4"),
        # one row, a 32-bit model
        dict(name="logits one row", op="logits", dtype="f32", B=1, R=1, V=32000, history=200, tree="", penalties=True, biases=8,
             mask=False),
        # drafted chains of a serving batch, penalties and biases
        dict(name="logits chain", op="logits", dtype="bf16", B=64, R=9, V=128256, history=4096, tree="", penalties=True,
             biases=64, mask=False),
        # a draft tree under a grammar: a mask for every node
        dict(name="logits tree mask", op="logits", dtype="bf16", B=32, R=17, V=151936, history=513, tree="4x4", penalties=True,
             biases=0, mask=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention"] * 4 + ["append", "commit"] + ["logits"] * 2)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "attention":
        tree = rng.choice(["", "", ""] + sorted(TREES))
        R = len(TREES[tree]) if tree else rng.choice([1, rng.randint(2, 17), _log(rng, 18, 2048)])
        Hkv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 3, 4, 7, 8])
        D, page = rng.choice([64, 128]), rng.choice([8, 16, 20, 32, 64, 128, 256])
        ctx = _log(rng, 1, 131072) - 1
        # within the largest listed cases: products (of 32 bits far fewer), scores, cache bytes
        size = 4 if dtype == "f32" else 2
        most = min((1.2e11 if size == 2 else 3e10) / (R * Hkv * group * D), 1.2e9 / (R * Hkv * group), 2e8 / (Hkv * D * size))
        ctx = max(0, min(ctx, int(most) - R - page))
        most = min(most / (ctx + R + page), 64)
        B = _log(rng, 1, max(1, int(most)))
        window = rng.choice([0, 0, _log(rng, 1, 4096)])
        return dict(op=op, dtype=dtype, B=B, R=R, Hq=Hkv * group, Hkv=Hkv, D=D, page=page, ctx=ctx, tree=tree, window=window,
                    sinks=rng.choice([0, 4, 130]) if window else 0, ragged=rng.random() < 0.5)
    if op == "append":
        R = rng.choice([1, rng.randint(2, 24), _log(rng, 25, 2048)])
        B = _log(rng, 1, max(1, min(64, 16384 // R)))
        return dict(op=op, dtype=dtype, B=B, R=R, Hkv=rng.choice([1, 2, 8]), D=rng.choice([64, 80, 128]),
                    page=rng.choice([8, 16, 20, 64]), ctx=_log(rng, 1, 800) - 1, ragged=rng.random() < 0.5)
    if op == "commit":
        return dict(op=op, dtype=dtype, B=_log(rng, 1, 32), layers=_log(rng, 1, 16), Hkv=rng.choice([1, 4, 8]),
                    D=rng.choice([64, 80, 128]), page=rng.choice([8, 16, 20, 64]), ctx=rng.randint(0, 120),
                    tree=rng.choice(sorted(TREES)))
    tree = rng.choice(["", ""] + sorted(TREES))
    R = len(TREES[tree]) if tree else rng.randint(1, 17)
    V = rng.choice([32000, 50257, 128256, 151936, _log(rng, 1000, 160000)])
    B = _log(rng, 1, max(1, int(3.6e7 / (R * V))))
    mask = rng.random() < 0.5
    return dict(op=op, dtype=dtype, B=B, R=R, V=V, history=_log(rng, 1, 8192), tree=tree, penalties=not mask or rng.random() < 0.7,
                biases=rng.choice([0, 5, 300]), mask=mask)


# ----------------------------------------------------------------------------------------------- inputs
def _pages(case, gen):
    """Block table [B, pages of a sequence]: the pages of the pool in random order, as a server hands them out."""
    rows = case.get("R") or len(TREES[case["tree"]])
    per = -(-(case["ctx"] + rows) // case["page"])
    n = case["B"] * per
    return torch.randperm(n, generator=gen, device="cuda").view(case["B"], per).to(torch.int32), n


def _lengths(case, gen):
    """Contexts between half of the longest and the longest, which the first sequence has."""
    low = torch.rand(case["B"], generator=gen, device="cuda") * 0.5 + 0.5
    ctx = (low * case["ctx"]).to(torch.int32)
    ctx[0] = case["ctx"]
    rows = None
    if case.get("ragged"):
        rows = torch.randint(0, case["R"] + 1, (case["B"],), generator=gen, device="cuda", dtype=torch.int32)
        rows[0] = case["R"]
    return ctx, rows


def _ancestors(parent):
    """[N + 1, N + 1] truth values (node m is n or above n) and depths."""
    n = len(parent)
    anc, depth = np.eye(n, dtype=bool), np.zeros(n, dtype=np.int64)
    for i in range(1, n):
        anc[i] |= anc[parent[i]]
        depth[i] = depth[parent[i]] + 1
    return anc, depth


def _paths(case):
    """Accepted paths of a batch: each follows the tree to one of its nodes.  They are cut before a slot that one move
    fills is another move's source, so that a pass can be repeated on the cache it left."""
    parent = TREES[case["tree"]]
    depth = _ancestors(parent)[1].max()
    out = np.full((case["B"], depth + 1), -1, dtype=np.int32)
    for b in range(case["B"]):
        node, path = (7 * b + 5) % len(parent), []
        while node >= 0:
            path.append(node)
            node = parent[node]
        path = path[::-1]
        keep = len(path)
        while any(path[j] != j and path[j] < keep for j in range(keep)):
            keep -= 1
        out[b, :keep] = path[:keep]
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def randn(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dt)

    s = dict(op=case["op"])
    if case["op"] == "logits":
        B, R, V, H = case["B"], case["R"], case["V"], case["history"]
        s["parent"] = list(TREES[case["tree"]]) if case["tree"] else None
        s["logits"] = randn(B, R, V, scale=3.0)
        s["out"] = torch.empty_like(s["logits"])

        def tokens(*shape):  # few tokens are frequent, as in text
            return (torch.rand(*shape, generator=gen, device="cuda").pow(3.0) * V).to(torch.int32).clamp_(max=V - 1)

        for k in ("history", "history_lens", "prompt_lens", "draft_tokens", "repetition", "presence", "frequency",
                  "bias_tokens", "bias_values", "mask"):
            s[k] = None
        if case["penalties"]:
            s["history"] = tokens(B, H)
            s["history_lens"] = torch.randint(H // 2, H + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
            s["prompt_lens"] = s["history_lens"] // 2
            s["draft_tokens"] = tokens(B, R if case["tree"] else R - 1)
            s["repetition"] = torch.rand(B, generator=gen, device="cuda") * 0.5 + 1.0
            s["presence"] = torch.rand(B, generator=gen, device="cuda") * 2 - 0.5
            s["frequency"] = torch.rand(B, generator=gen, device="cuda") * 0.5
        if case["biases"]:
            # distinct tokens of each sequence, some of them banned
            first = torch.randint(0, V, (B, 1), generator=gen, device="cuda")
            step = torch.arange(case["biases"], device="cuda") * max(1, V // (case["biases"] + 1))
            s["bias_tokens"] = ((first + step) % V).to(torch.int32)
            s["bias_values"] = torch.randn(B, case["biases"], generator=gen, device="cuda") * 4
            s["bias_values"][:, ::4] = -math.inf
        if case["mask"]:
            # a grammar leaves some thousands of tokens in one state, a handful in another
            share = torch.rand(B, R, 1, generator=gen, device="cuda").pow(3.0)
            words = -(-V // 32)
            bits = torch.rand(B, R, words * 32, generator=gen, device="cuda") < share
            weights = (2 ** torch.arange(32, device="cuda", dtype=torch.int64))
            m = (bits.view(B, R, words, 32) * weights).sum(-1)
            s["mask"] = torch.where(m >= 2 ** 31, m - 2 ** 32, m).to(torch.int32)
        if s["parent"]:
            s["above"] = torch.from_numpy(_ancestors(s["parent"])[0]).cuda()
        else:
            s["above"] = torch.ones(R, R, dtype=torch.bool, device="cuda").tril()
        return s
    s["table"], n = _pages(case, gen)
    shape = (n, case["page"], case["Hkv"], case["D"])
    s["ctx"], s["rows"] = _lengths(case, gen)
    if case["op"] == "commit":
        s["k"], s["v"] = randn(case["layers"], *shape), randn(case["layers"], *shape)
        path = torch.from_numpy(_paths(case))[torch.randperm(case["B"], generator=gen, device="cuda").cpu()]
        s["path"] = path.cuda()
        s["accept"] = ((path >= 0).sum(1) - 1).to(torch.int32).cuda()
        s["new_ctx"] = torch.empty_like(s["ctx"])
        return s
    s["k"], s["v"] = randn(*shape), randn(*shape)
    B, R = case["B"], case["R"]
    if case["op"] == "append":
        s["k_new"], s["v_new"] = randn(B, R, case["Hkv"], case["D"]), randn(B, R, case["Hkv"], case["D"])
        return s
    s["q"] = randn(B, R, case["Hq"], case["D"], scale=2.0)
    s["out"] = torch.zeros_like(s["q"])
    s["parent"] = list(TREES[case["tree"]]) if case["tree"] else None
    s["window"], s["sinks"], s["max_context"] = case["window"], case["sinks"], case["ctx"]
    if s["parent"]:
        above, depth = _ancestors(s["parent"])
        s["above"], s["depth"] = torch.from_numpy(above).cuda(), torch.from_numpy(depth).cuda()
    else:
        s["above"] = torch.ones(R, R, dtype=torch.bool, device="cuda").tril()
        s["depth"] = torch.arange(R, device="cuda")
    return s


# ----------------------------------------------------------------------------------------------- plain forms
def _attention(s):
    q, table, ctx = s["q"].float(), s["table"].long(), s["ctx"].long()
    B, R, Hq, D = q.shape
    page, Hkv = s["k"].shape[1], s["k"].shape[2]
    L = table.shape[1] * page
    k = s["k"][table].float().view(B, L, Hkv, D)
    v = s["v"][table].float().view(B, L, Hkv, D)
    p = torch.arange(L, device=q.device)
    node = p[None, :] - ctx[:, None]                                        # [B, L], node of a slot, < 0 in the context
    own_pos = ctx[:, None] + s["depth"][None, :]                            # [B, R]
    key_pos = torch.where(node < 0, p[None, :].expand_as(node), ctx[:, None] + s["depth"][node.clamp(0, R - 1)])
    seen = (node < 0)[:, None, :] | s["above"][:, node.clamp(0, R - 1)].permute(1, 0, 2)
    seen &= (node < R)[:, None, :]
    if s["window"]:
        seen &= (key_pos[:, None, :] > own_pos[:, :, None] - s["window"]) | (key_pos < s["sinks"])[:, None, :]
    qg = q.view(B, R, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    score = torch.matmul(qg, k.permute(0, 2, 3, 1)).view(B, Hkv, Hq // Hkv, R, L) / math.sqrt(D)
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    e = torch.exp(score - score.amax(-1, keepdim=True))
    w = (e / e.sum(-1, keepdim=True)).view(B, Hkv, -1, L)
    o = torch.matmul(w, v.permute(0, 2, 1, 3)).view(B, Hkv, Hq // Hkv, R, D).permute(0, 3, 1, 2, 4).reshape(B, R, Hq, D)
    if s["rows"] is not None:
        o = torch.where((torch.arange(R, device=q.device) < s["rows"][:, None])[:, :, None, None], o, s["out"].float())
    return o.to(s["q"].dtype)


def _slots(table, pos, page):
    """Index into the cache's rows of position pos [B, n] of each sequence."""
    return torch.gather(table.long(), 1, pos // page) * page + pos % page


def _append(s):
    B, R = s["k_new"].shape[:2]
    page = s["k"].shape[1]
    pos = s["ctx"].long()[:, None] + torch.arange(R, device="cuda")
    slot = _slots(s["table"], pos, page)
    if s["rows"] is None:
        slot = slot.reshape(-1)
        pick = torch.arange(B * R, device="cuda")
    else:
        take = torch.arange(R, device="cuda") < s["rows"][:, None]
        slot, pick = slot[take], take.reshape(-1).nonzero()[:, 0]
    for cache, new in ((s["k"], s["k_new"]), (s["v"], s["v_new"])):
        cache.view(-1, *cache.shape[2:])[slot] = new.view(-1, *new.shape[2:])[pick]
    return s["k"], s["v"]


def _commit(s):
    page = s["k"].shape[2]
    path, ctx = s["path"].long(), s["ctx"].long()
    move = path >= 0
    j = torch.arange(path.shape[1], device="cuda").expand_as(path)
    src = _slots(s["table"], ctx[:, None] + path.clamp(min=0), page)[move]
    dst = _slots(s["table"], ctx[:, None] + torch.where(move, j, 0), page)[move]
    for cache in (s["k"], s["v"]):
        rows = cache.view(cache.shape[0], -1, *cache.shape[3:])
        rows[:, dst] = rows[:, src]
    s["new_ctx"].copy_(s["ctx"] + s["accept"] + 1)
    return s["k"], s["v"], s["new_ctx"]


def _logits(s):
    x = s["logits"].float()
    B, R, V = x.shape
    if s["history"] is not None:
        at = torch.arange(s["history"].shape[1], device=x.device)
        tok = s["history"].long()
        there = (at < s["history_lens"][:, None]).float()
        said = there * (at >= s["prompt_lens"][:, None]).float()
        seen = torch.zeros(B, V, device=x.device).scatter_add_(1, tok, there)
        count = torch.zeros(B, V, device=x.device).scatter_add_(1, tok, said)
        seen, count = seen[:, None].expand(B, R, V).contiguous(), count[:, None].expand(B, R, V).contiguous()
        drafted = s["draft_tokens"].long()
        if s["parent"] is not None:
            drafted = drafted[:, 1:]
        path = s["above"][:, 1:].float().expand(B, R, R - 1)
        drafted = drafted[:, None].expand(B, R, R - 1)
        seen.scatter_add_(2, drafted, path)
        count.scatter_add_(2, drafted, path)
        r = s["repetition"][:, None, None]
        x = torch.where(seen > 0, torch.where(x > 0, x / r, x * r), x)
        x = x - s["frequency"][:, None, None] * count
        x = x - s["presence"][:, None, None] * (count > 0)
    if s["bias_tokens"] is not None:
        bias = torch.zeros(B, V, device=x.device).scatter_(1, s["bias_tokens"].long(), s["bias_values"])
        x = x + bias[:, None]
    if s["mask"] is not None:
        shift = torch.arange(32, device=x.device, dtype=torch.int32)
        bits = ((s["mask"][..., None] >> shift) & 1).view(B, R, -1)[..., :V]
        x = x.masked_fill(bits == 0, -math.inf)
    return x.to(s["logits"].dtype)


def _run_own(s):
    from paper_2504_15475_b200 import binding as ersd
    op = s["op"]
    if op == "attention":
        ersd.ersd_chunk_attention(s["q"], s["k"], s["v"], s["table"], s["ctx"], s["out"], parent=s["parent"],
                                  row_counts=s["rows"], window=s["window"], sinks=s["sinks"], max_context=s["max_context"])
        return s["out"]
    if op == "append":
        ersd.ersd_cache_append(s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["ctx"], row_counts=s["rows"])
        return s["k"], s["v"]
    if op == "commit":
        ersd.ersd_cache_commit(s["k"], s["v"], s["table"], s["ctx"], s["path"], s["accept"], s["new_ctx"])
        return s["k"], s["v"], s["new_ctx"]
    ersd.ersd_process_logits(s["logits"], s["out"], history=s["history"], history_lens=s["history_lens"],
                             prompt_lens=s["prompt_lens"], draft_tokens=s["draft_tokens"], parent=s["parent"],
                             repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"],
                             bias_tokens=s["bias_tokens"], bias_values=s["bias_values"], mask=s["mask"])
    return s["out"]


def run(state):
    if own:
        return _run_own(state)
    return {"attention": _attention, "append": _append, "commit": _commit, "logits": _logits}[state["op"]](state)


# ----------------------------------------------------------------------------------------------- work
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "logits":
        B, R, V = case["B"], case["R"], case["V"]
        b = 2 * size * B * R * V + (B * R * (-(-V // 32)) * 4 if case["mask"] else 0) + 8 * B * case["biases"]
        if case["penalties"]:
            b += 4 * B * (case["history"] * 3 // 4 + R + 5)
        return dict(bytes=b, flops=2 * B * R * V)
    row = case["Hkv"] * case["D"] * size
    if case["op"] == "append":
        rows = case["B"] * case["R"] * (0.5 if case["ragged"] and case["B"] > 1 else 1.0)
        return dict(bytes=4 * rows * row + 8 * case["B"], flops=0)
    if case["op"] == "commit":
        p = _paths(case)
        moved = int(((p >= 0) & (p != np.arange(p.shape[1]))).sum())
        return dict(bytes=4 * moved * case["layers"] * row + p.size * 4 + 12 * case["B"], flops=0)
    B, R = case["B"], case["R"]
    mean_ctx = case["ctx"] if B == 1 else case["ctx"] * (0.75 + 0.25 / B)
    rows = R * (0.5 + 0.5 / B if case["ragged"] else 1.0)
    W = case["window"] or 1 << 40
    reach = min(mean_ctx, W - 1 + case["sinks"])
    if case["tree"]:
        inner = float(_ancestors(TREES[case["tree"]])[0].sum()) / R
    else:
        inner = sum(min(i + 1, W) for i in range(R)) / R
    keys = reach + rows
    return dict(bytes=2 * B * keys * row + 2 * B * rows * case["Hq"] * case["D"] * size + 4 * B * (1 + keys / case["page"]),
                flops=4 * B * rows * case["Hq"] * case["D"] * (min(mean_ctx, W) + inner))


# ----------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """From the definitions, in 64 bits, a sequence (or a row) at a time."""
    s = prepare(case, seed)
    if case["op"] in ("append", "commit"):  # copies: no arithmetic
        return None
    if case["op"] == "attention":
        return _exact_attention(s)
    return _exact_logits(s)


def _exact_attention(s):
    B, R, Hq, D = s["q"].shape
    page, Hkv = s["k"].shape[1], s["k"].shape[2]
    out = s["out"].double()
    parent = s["parent"] or list(range(-1, R - 1))
    depth, lineage = [0], [[0]]
    for n in range(1, len(parent)):
        depth.append(depth[parent[n]] + 1)
        lineage.append(lineage[parent[n]] + [n])
    for b in range(B):
        ctx = int(s["ctx"][b])
        rows = R if s["rows"] is None else int(s["rows"][b])
        if not rows:
            continue
        n = ctx + rows
        pages = s["table"][b, : -(-n // page)].long()
        k = s["k"][pages].reshape(-1, Hkv, D)[:n].double()
        v = s["v"][pages].reshape(-1, Hkv, D)[:n].double()
        pos = torch.cat([torch.arange(ctx), ctx + torch.tensor(depth[:rows], dtype=torch.int64)])
        if s["parent"] is None:
            see = torch.arange(n) <= ctx + torch.arange(rows)[:, None]
        else:
            see = torch.zeros(rows, n, dtype=torch.bool)
            see[:, :ctx] = True
            for r in range(rows):
                see[r, [ctx + m for m in lineage[r]]] = True
        if s["window"]:
            here = ctx + torch.tensor(depth[:rows])
            see &= (here[:, None] - pos < s["window"]) | (pos < s["sinks"])
        see = see.cuda()
        for h in range(Hkv):
            g = Hq // Hkv
            q = s["q"][b, :rows, h * g:(h + 1) * g].double()
            a = torch.einsum("rgd,nd->grn", q, k[:, h]) * D ** -0.5
            a = torch.softmax(torch.where(see, a, -math.inf), dim=-1)
            out[b, :rows, h * g:(h + 1) * g] = torch.einsum("grn,nd->rgd", a, v[:, h])
    return out


def _exact_logits(s):
    x = s["logits"].double()
    B, R, V = x.shape
    parent = s["parent"] or list(range(-1, R - 1))
    host = {k: s[k].cpu().numpy() for k in ("history", "history_lens", "prompt_lens", "draft_tokens", "bias_tokens") if s[k] is not None}
    for b in range(B):
        for r in range(R):
            row = x[b, r]
            if s["history"] is not None:
                n, m = int(host["history_lens"][b]), int(host["prompt_lens"][b])
                path, node = [], r
                while node > 0:
                    path.append(int(host["draft_tokens"][b, node if s["parent"] else node - 1]))
                    node = parent[node]
                said = np.concatenate([host["history"][b, m:n], np.array(path, dtype=np.int32)])
                seen = np.unique(np.concatenate([host["history"][b, :m], said]))
                tok, times = np.unique(said, return_counts=True)
                at = torch.from_numpy(seen).long().cuda()
                rep = s["repetition"][b].double()
                row[at] = torch.where(row[at] > 0, row[at] / rep, row[at] * rep)
                at = torch.from_numpy(tok).long().cuda()
                row[at] -= s["frequency"][b].double() * torch.from_numpy(times).cuda() + s["presence"][b].double()
            if s["bias_tokens"] is not None:
                row[s["bias_tokens"][b].long()] += s["bias_values"][b].double()
            if s["mask"] is not None:
                bits = np.unpackbits(s["mask"][b, r].cpu().numpy().view(np.uint8), bitorder="little")[:V]
                row[torch.from_numpy(bits == 0).cuda()] = -math.inf
    return x
