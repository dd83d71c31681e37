"""64-bit forms of the operators around a verification, a sequence and a row at a time, and the error bounds
that their 32-bit forms are held to."""
from __future__ import annotations

import numpy as np
import torch

BITS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # half a step of a rounding, relative


def lineage(parent, R):
    """Per row: the nodes it descends from and itself; None: every row follows the one before."""
    if parent is None:
        return [list(range(r + 1)) for r in range(R)]
    rows = [[0]]
    for n in range(1, R):
        rows.append(rows[parent[n]] + [n])
    return rows


def visible(ctx, R, parent, window, sinks, capacity):
    """[R, capacity] truth values: which slots each row sees."""
    rows = lineage(parent, R)
    see = np.zeros((R, capacity), dtype=bool)
    for r, nodes in enumerate(rows):
        here = ctx + len(nodes) - 1
        for p in list(range(min(ctx, capacity))):
            see[r, p] = not window or p > here - window or p < sinks
        for i, n in enumerate(nodes):
            if ctx + n < capacity:
                pos = ctx + i
                see[r, ctx + n] = not window or pos > here - window or pos < sinks
    return see


def attention(q, k_cache, v_cache, table, ctx_lens, scale=None, parent=None, row_counts=None, window=0, sinks=0,
              weight_bits=0.0):
    """(out, bound) in float64, [B, R, Hq, D]; rows that do not count are NaN in both.  weight_bits: half a step
    of what the softmax weights are rounded to (0: they are not).

    The bound: a score q.k of D products of exact bf16 or f32 values accumulated in 32 bits is off by at most
    (D + 4) steps of 2^-23 (a tensor core may cut instead of round: 2^-23, not 2^-24) of scale * sum |q k|; a
    weight then by twice that relative to the others (numerator and denominator) and by 2^-20 for the power of
    two and the rescaling, and weight_bits; n summed terms add n steps of 2^-23; the result is rounded once."""
    B, R, Hq, D = q.shape
    page, H = k_cache.shape[1], k_cache.shape[2]
    capacity = table.shape[1] * page
    scale = D ** -0.5 if scale is None else scale
    g = Hq // H
    out = torch.full((B, R, Hq, D), float("nan"), dtype=torch.float64, device=q.device)
    bound = out.clone()
    for b in range(B):
        rows = R if row_counts is None else max(0, min(R, int(row_counts[b])))
        if not rows:
            continue
        ctx = max(0, int(ctx_lens[b]))
        see = torch.from_numpy(visible(ctx, R, parent, window, sinks, capacity)[:rows]).to(q.device)
        used = see.any(0)
        n = max(1, int(used.sum()))
        slots = used.nonzero()[:, 0]
        pages = table[b].long()[slots // page]
        there = ((pages >= 0) & (pages < k_cache.shape[0]))[:, None, None]
        at = pages.clamp(0, k_cache.shape[0] - 1)
        k = torch.where(there, k_cache[at, slots % page].double(), 0.0)
        v = torch.where(there, v_cache[at, slots % page].double(), 0.0)
        m = see[:, slots]
        for h in range(H):
            x = q[b, :rows, h * g:(h + 1) * g].double()
            s = torch.einsum("rgd,nd->rgn", x, k[:, h]) * scale
            size = torch.einsum("rgd,nd->rgn", x.abs(), k[:, h].abs()) * abs(scale)
            s = torch.where(m[:, None], s, -np.inf)
            size = torch.where(m[:, None], size, 0.0)
            top = s.amax(-1, keepdim=True) if s.shape[-1] else s.new_zeros(rows, g, 1)
            e = torch.exp(s - torch.where(torch.isinf(top), 0.0, top))
            total = e.sum(-1, keepdim=True)
            w = torch.where(total > 0, e / total, 0.0)
            o = torch.einsum("rgn,nd->rgd", w, v[:, h])
            spread = torch.einsum("rgn,nd->rgd", w, v[:, h].abs())
            off = (size.amax(-1, keepdim=True) if s.shape[-1] else top) * (D + 4) * 2.0 ** -23
            out[b, :rows, h * g:(h + 1) * g] = o
            bound[b, :rows, h * g:(h + 1) * g] = (spread * (2 * off + 2.0 ** -19 + (n + 8) * 2.0 ** -23 + weight_bits)
                                                  + o.abs() * BITS[q.dtype] * 1.01 + 1e-30)
    return out, bound


def held(l, dtype=torch.float32):
    """A number beyond the largest of its type by half a step or more is an infinity there."""
    return l if abs(l) < torch.finfo(dtype).max * (1 + BITS[dtype] / 2) else float(np.copysign(np.inf, l))


def process_logits(x, history=None, history_lens=None, prompt_lens=None, draft_tokens=None, parent=None, repetition=None,
                   presence=None, frequency=None, bias_tokens=None, bias_values=None, mask=None, V=None):
    """(out, bound) in float64 of logits [B, R, ld] (host tensors).  The bound: four operations in 32 bits, each off
    by half a step of the largest value that occurs on the way, and one rounding to the logits' type."""
    B, R, ld = x.shape
    V = ld if V is None else V
    out, bound = x.double().clone(), torch.zeros(B, R, ld, dtype=torch.float64)
    rows = lineage(parent, R)
    for b in range(B):
        n = history.shape[1] if history_lens is None and history is not None else 0 if history is None else int(history_lens[b])
        n = max(0, min(n, 0 if history is None else history.shape[1]))
        m = 0 if prompt_lens is None else int(prompt_lens[b])
        tokens = [] if history is None else [int(t) for t in history[b, :n]]
        bias = {}
        if bias_tokens is not None:
            c = 0 if bias_tokens.shape[0] == 1 else b
            for t, f in zip(bias_tokens[c].tolist(), bias_values[c].tolist()):
                bias[t] = f
        for r in range(R):
            drafted = [] if draft_tokens is None else [int(draft_tokens[b, i if parent is not None else i - 1]) for i in rows[r][1:]]
            count, seen = {}, set()
            for i, t in enumerate(tokens):
                seen.add(t)
                if i >= m:
                    count[t] = count.get(t, 0) + 1
            for t in drafted:
                seen.add(t)
                count[t] = count.get(t, 0) + 1
            for t in seen | set(bias):
                if not 0 <= t < V:
                    continue
                l = float(out[b, r, t])
                big = abs(l)
                if t in seen:
                    if repetition is not None:
                        l = held(l / float(repetition[b]) if l > 0 else l * float(repetition[b]))
                        big = max(big, abs(l))
                    c = count.get(t, 0)
                    if c:
                        f = 0.0 if frequency is None else float(frequency[b]) * c
                        p = 0.0 if presence is None else float(presence[b])
                        big = max(big, abs(l), abs(f), abs(l - f))
                        l = held(l - (f + p))
                if t in bias:
                    big = max(big, abs(l), abs(bias[t]) if np.isfinite(bias[t]) else 0.0)
                    l = held(l + bias[t])
                l = held(l, x.dtype)
                out[b, r, t] = l
                if np.isfinite(l):
                    bound[b, r, t] = 5 * max(big, abs(l)) * 2.0 ** -24 + abs(l) * BITS[x.dtype] * 1.01
            if mask is not None:
                words = mask[0 if mask.shape[0] == 1 else b, 0 if mask.shape[1] == 1 else r].numpy().view(np.uint8)
                bits = np.unpackbits(words, bitorder="little")[:V]
                off = torch.from_numpy(bits == 0)
                out[b, r, :V][off] = -np.inf
                bound[b, r, :V][off] = 0.0
    return out, bound


def check(got, want, bound, what=""):
    """Every value within its bound; infinities and NaN where the 64-bit form has them."""
    got = got.double().to(want.device)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN in other places"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what + ": infinities differ"
    over = (got - want).abs()[fine] - bound[fine]
    assert not (over > 0).any(), "%s: %d values beyond their bound, the worst by %g" % (what, int((over > 0).sum()), float(over.max()))
