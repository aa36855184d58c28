"""Plain definitions of sparse attention over the pool (block summaries, selection, attention over listed blocks) and of a batch's
tables, in 64 bits and Python numbers, one block or one row at a time."""
from __future__ import annotations

import math

import torch

MOST = 127.0 * 2.0 ** 113


def exponent(top):
    """The smallest whole number from -60 on with top <= 127 * 2^e."""
    e = -60
    while top > 127.0 * 2.0 ** e:
        e += 1
    return e


def exponents(top):
    """The same for a tensor of 64-bit numbers."""
    e = torch.full(top.shape, -60.0, dtype=torch.float64, device=top.device)
    for _ in range(174):  # -60 ... 113
        e = torch.where(top > 127.0 * torch.exp2(e), e + 1, e)
    return e


def summary_ref(keys, block):
    """keys: [tokens, heads, dim] of one layer.  Codes [blocks, heads, 2, dim] and exponents [blocks, heads], whole numbers."""
    k = keys.double()
    out, exps = [], []
    for b0 in range(0, k.shape[0], block):
        rows = k[b0:b0 + block]
        nan = torch.isnan(rows)
        hi = torch.where(nan, MOST, rows).clamp(-MOST, MOST).max(0).values
        lo = torch.where(nan, -MOST, rows).clamp(-MOST, MOST).min(0).values
        e = exponents(torch.maximum(hi.abs(), lo.abs()).max(-1).values)
        unit = torch.exp2(e)[:, None]
        out.append(torch.stack((torch.ceil(hi / unit), torch.floor(lo / unit)), 1))
        exps.append(e)
    return torch.stack(out), torch.stack(exps)


def read_summary(summary, layer, table, heads, dim):
    """Codes and exponents that the records of a context's blocks hold."""
    rec = summary.view(summary.shape[0], summary.shape[1], -1)[layer, table.long().to(summary.device)].double()
    return rec[:, :heads * 2 * dim].view(-1, heads, 2, dim), rec[:, heads * 2 * dim:heads * 2 * dim + heads]


def scores_ref(codes, exps, q):
    """q: [heads of a group, dim] of one token; codes [blocks, 2, dim], exps [blocks] of its kv head: 32-bit scores as Python numbers."""
    x = torch.where(torch.isnan(q.double()), 0.0, q.double()).clamp(-MOST, MOST)
    f = exponents(x.abs().max(-1).values)
    c = torch.round(x / torch.exp2(f)[:, None])
    dot = torch.maximum(c * codes[:, None, 0], c * codes[:, None, 1]).sum(-1)  # [blocks, heads]
    return (dot * torch.exp2(exps[:, None] + f)).float().max(-1).values.tolist()


def select_ref(scores, last, keep, sink, recent):
    """Blocks [0, last] by their scores."""
    forced = [b for b in range(last + 1) if b < sink or b > last - recent]
    rest = sorted((b for b in range(last + 1) if sink <= b <= last - recent), key=lambda b: (-scores[b], b))
    return sorted(forced + rest[:keep - len(forced)])


def attend_blocks_ref(ctxs, n_q, q, blocks, block, layer=0, scale=None, softcap=0.0, window=0, slopes=None, spans=None):
    """(out, lse, slack, big) as serve_reference.attend_ref has them; blocks: [tokens, kv heads, keep]."""
    heads_q, dim = q.shape[1], q.shape[2]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    slack, big, at = torch.zeros_like(out), 0.0, 0
    within = torch.arange(block, device=q.device)
    for i, (c, nq) in enumerate(zip(ctxs, n_q)):
        k, v = c.rows[layer].double()
        t, heads = k.shape[:2]
        group, sc = heads_q // heads, dim ** -0.5 if scale is None else scale
        nblk = -(-t // block)
        for j in range(nq):
            pos, r = t - nq + j, at + j
            lo, hi = (0, pos + 1) if spans is None else (max(0, int(spans[r, 0])), min(t, int(spans[r, 1])))
            if window:
                lo = max(lo, pos + 1 - window)
            for h in range(heads):
                b = blocks[r, h].long()
                b = b[(b >= 0) & (b < nblk)]
                key = (b[:, None] * block + within).flatten()
                key = key[(key >= lo) & (key < hi)]
                if not key.numel():
                    continue
                rows = slice(h * group, (h + 1) * group)
                kh, vh, qh = k[key, h], v[key, h], q[r, rows].double()
                x = qh @ kh.T * sc
                big = max(big, float((qh.abs() @ kh.nan_to_num(0.0, 0.0, 0.0).abs().T * abs(sc)).max()))
                if softcap:
                    x = softcap * torch.tanh(x / softcap)
                if slopes is not None:
                    x = x - slopes[rows, None].double() * (pos - key).abs()
                top = x.max(-1, keepdim=True).values
                top = torch.where(torch.isinf(top) & (top < 0), 0.0, top)
                w = torch.exp(x - top)
                total = w.sum(-1, keepdim=True)
                w = w / torch.where(total == 0, 1.0, total)
                y = w @ vh
                out[r, rows] = torch.where(total == 0, 0.0, y)  # a row whose scores are all -inf
                slack[r, rows] = w @ vh.nan_to_num(0.0, 0.0, 0.0).abs()
                lse[r, rows] = torch.where(total == 0, -math.inf, top + total.log())[:, 0]
        at += nq
    return out, lse, slack, big


def batch_tables_ref(tables, lens, new, block, rows, tokens, cols):
    """Everything as Python lists."""
    n, total = len(lens), sum(new)
    t = [list(tables[i]) + [-1] * (cols - len(tables[i])) if i < n else [-1] * cols for i in range(rows)]
    got = {"tables": t, "lens": list(lens) + [0] * (rows - n), "offsets": [sum(new[:i]) for i in range(n)] + [total] * (rows + 1 - n),
           "token_row": [], "positions": [], "slots": []}
    for i in range(n):
        for p in range(lens[i] - new[i], lens[i]):
            got["token_row"].append(i)
            got["positions"].append(p)
            got["slots"].append(int(tables[i][p // block]) * block + p % block)
    for k, fill in (("token_row", -1), ("positions", 0), ("slots", -1)):
        got[k] += [fill] * (tokens - total)
    return got
