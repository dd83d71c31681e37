"""Decoding steps as a server makes them: rows of a draft tree into the cache, their attention, logits changed and
verified, the accepted path made the sequence's own -- several steps on one cache, against a cache that holds the
accepted tokens' rows from the start."""
import pytest
import torch

import operator_reference as ref
from paper_2504_15475_b200 import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ersd():
    from paper_2504_15475_b200 import binding
    binding.lib()
    return binding


class Model:
    """Keys, values, queries and logits that depend on a token and its position alone: what a row gets is known
    without any cache."""

    def __init__(self, V, Hq, H, D, dtype):
        gen = torch.Generator(device="cuda").manual_seed(3)
        r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
        self.tok = {n: r(V, h, D) for n, h in (("q", Hq), ("k", H), ("v", H))}
        self.pos = {n: r(512, h, D) for n, h in (("q", Hq), ("k", H), ("v", H))}
        self.logit, self.dtype = r(Hq * D, V), dtype

    def rows(self, name, token, position):
        return (self.tok[name][token] + self.pos[name][position]).to(self.dtype)

    def logits(self, out):
        return (out.float().flatten(-2) @ self.logit * 0.2).to(self.dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("parent", [list(wl.TREE_4x4), list(wl.TREE_SPECINFER), list(wl.chain_parent(5))])
@pytest.mark.parametrize("D,page,window", [(64, 16, 0), (128, 8, 20)])
def test_steps(ersd, dtype, parent, D, page, window):
    V, Hq, H, B, layers = 500, 4, 2, 3, 2
    m, n = Model(V, Hq, H, D, dtype), len(parent)
    depth = torch.tensor([len(x) - 1 for x in ref.lineage(parent, n)], device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(4)
    per = 20
    k, v = (torch.full((layers, B * per, page, H, D), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    table = torch.randperm(B * per, generator=gen, device="cuda").view(B, per).to(torch.int32)
    # prompts of several lengths, written in one call of ragged rows
    text = [torch.randint(0, V, (int(L),), generator=gen, device="cuda") for L in (1, 17, 40)]
    lens = torch.tensor([len(t) - 1 for t in text], dtype=torch.int32, device="cuda")   # the last token is the next root
    prompt = torch.zeros(B, 40, dtype=torch.int64, device="cuda")
    for b in range(B):
        prompt[b, : len(text[b])] = text[b]
    at = torch.arange(40, device="cuda").expand(B, 40)
    zero = torch.zeros_like(lens)
    for layer in range(layers):
        ersd.ersd_cache_append(m.rows("k", prompt, at), m.rows("v", prompt, at), k[layer], v[layer], table, zero, row_counts=lens)
    seeds = wl.make_seeds(5, 1, B).cuda()
    rep = torch.full((B,), 1.3, device="cuda")
    moved = 0
    for step in range(6):
        ctx = lens.tolist()
        drafts = torch.randint(0, V, (B, n), generator=gen, device="cuda", dtype=torch.int32)
        tokens = drafts.clone().long()
        tokens[:, 0] = torch.stack([t[-1] for t in text])
        where = lens[:, None].long() + depth
        q = m.rows("q", tokens, where)
        out = torch.empty_like(q)
        for layer in range(layers):
            ersd.ersd_cache_append(m.rows("k", tokens, where), m.rows("v", tokens, where), k[layer], v[layer], table, lens)
            ersd.ersd_chunk_attention(q, k[layer], v[layer], table, lens, out, parent=parent, window=window)
        # the same rows from every row's own text, in 64 bits
        for b in range(B):
            for r, line in enumerate(ref.lineage(parent, n)):
                words = torch.cat([text[b][:-1], tokens[b, line]])
                p = torch.arange(len(words), device="cuda")
                pages = m.rows("k", words, p)[None], m.rows("v", words, p)[None]
                want, bound = ref.attention(q[b:b + 1, r:r + 1], *pages, torch.zeros(1, 1, dtype=torch.int64, device="cuda"),
                                            torch.tensor([len(words) - 1]), window=window,
                                            weight_bits=2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
                ref.check(out[b:b + 1, r:r + 1], want, bound, "step %d, sequence %d, row %d" % (step, b, r))
        target = m.logits(out)
        changed = torch.empty_like(target)
        history = torch.zeros(B, max(len(t) for t in text), dtype=torch.int32, device="cuda")
        for b in range(B):
            history[b, : len(text[b])] = text[b]
        length = torch.tensor([len(t) for t in text], dtype=torch.int32, device="cuda")
        ersd.ersd_process_logits(target, changed, history=history, history_lens=length, draft_tokens=drafts, parent=parent, repetition=rep)
        # a draft law under which every node's children are the target's likeliest tokens: paths are accepted
        res = ersd.verify(changed, changed, seeds, parent=parent, want_rows=True,
                          pos_offsets=torch.tensor(ctx, dtype=torch.int32, device="cuda"))
        # the drafts that were accepted were drawn by the race, and stand in the cache under their nodes: write them there
        tokens[:, 1:] = res["draft_tok"][:, 1:].long()
        for layer in range(layers):
            ersd.ersd_cache_append(m.rows("k", tokens, where), m.rows("v", tokens, where), k[layer], v[layer], table, lens)
        new = torch.empty_like(lens)
        ersd.ersd_cache_commit(k, v, table, lens, res["path"], res["accept_len"], new)
        for b in range(B):
            L = int(res["accept_len"][b])
            assert int(new[b]) == ctx[b] + L + 1
            path = res["path"][b, : L + 1].tolist()
            moved += sum(j != x for j, x in enumerate(path))
            text[b] = torch.cat([text[b], res["tokens"][b, : L + 1].long()])
            p = torch.arange(int(new[b]), device="cuda")
            for layer in range(layers):
                for cache, name in ((k, "k"), (v, "v")):
                    rows = cache[layer][table[b].long()].view(-1, H, D)[: int(new[b])]
                    assert torch.equal(rows, m.rows(name, text[b][:-1], p)), (step, b, layer, name)
        lens = new
    assert moved or parent == list(wl.chain_parent(5))
