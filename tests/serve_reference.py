"""Plain definitions of the operators that compute with the pool, in 64 bits, one token and one head at a time as far
as speed allows; and the contexts the tests run them on."""
from __future__ import annotations

import math

import numpy as np
import torch

DEV = "cuda"


class Ctx:
    """What a test knows of a context: its rows, in order, for every layer: [layers, 2, tokens, kv heads, dim]."""

    def __init__(self, handle, rows):
        self.handle, self.rows = handle, rows

    def __len__(self):
        return self.rows.shape[2]


def make_pool(layers=1, heads=2, dim=64, block=16, blocks=256, max_ctx=96, max_blk=None, dtype=torch.bfloat16, seed=0, fill=math.nan):
    """A pool whose every byte is `fill` (NaN: what was never stored shows) and whose free list is permuted."""
    from paper_2607_10987_b200 import KVPool

    mem = torch.full((layers, blocks, 2, block, heads, dim), fill, dtype=dtype, device=DEV)
    order = np.random.default_rng(seed).permutation(blocks).astype(np.int32)
    pool = KVPool(layers, heads, dim, block, 2, blocks, max_ctx, max_blk or blocks, free_order=order, pool_tensor=mem)
    pool.mem, pool.dt = mem, dtype
    return pool


def rand(shape, seed, dtype=torch.bfloat16, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def add_ctx(pool, tokens, seed, rows=None):
    rows = rand((pool.L, 2, tokens, pool.H, pool.D), seed, pool.dt) if rows is None else rows
    st, h = pool.imp(rows.contiguous(), tokens)
    assert st == 0
    return Ctx(h, rows)


def attend_ref(ctxs, n_q, q, layer=0, scale=None, softcap=0.0, window=0, slopes=None, spans=None):
    """(out, lse, slack): slack is sum_t w_t |v_t|, what an error in the weights is measured by; and amax, the largest
    sum of |q_i k_i| * scale, what an error in the scores is measured by."""
    outs, lses, slacks, big, at = [], [], [], 0.0, 0
    for i, (c, nq) in enumerate(zip(ctxs, n_q)):
        rows = c.rows[layer].double()
        k, v = rows[0], rows[1]
        t, heads, dim = k.shape
        group = q.shape[1] // heads
        sc = dim ** -0.5 if scale is None else scale
        pos = torch.arange(t - nq, t, device=q.device)
        lo, hi = torch.zeros_like(pos), pos + 1
        if spans is not None:
            lo, hi = spans[at:at + nq, 0].long().clamp(0, t), spans[at:at + nq, 1].long().clamp(0, t)
        if window:
            lo = torch.maximum(lo, pos + 1 - window)
        key = torch.arange(t, device=q.device)
        see = (key >= lo[:, None]) & (key < hi[:, None])
        out = torch.zeros(nq, q.shape[1], dim, dtype=torch.float64, device=q.device)
        lse = torch.zeros(nq, q.shape[1], dtype=torch.float64, device=q.device)
        slack = torch.zeros_like(out)
        for h in range(q.shape[1]):
            kh, vh = k[:, h // group], v[:, h // group]
            qh = q[at:at + nq, h].double()
            x = qh @ kh.nan_to_num(0.0, 0.0, 0.0).T * sc if not torch.isfinite(kh).all() else qh @ kh.T * sc
            big = max(big, float((qh.abs() @ kh.nan_to_num(0.0, 0.0, 0.0).abs().T * abs(sc)).max()))
            if softcap:
                x = softcap * torch.tanh(x / softcap)
            if slopes is not None:
                x = x - slopes[h].double() * (pos[:, None] - key).abs()
            x = x.masked_fill(~see, -math.inf)
            top = x.max(-1, keepdim=True).values.nan_to_num(neginf=0.0)
            w = torch.exp(x - top)
            total = w.sum(-1, keepdim=True)
            w = w / total.clamp_min(1e-300)
            # a row is the sum over the keys it sees only: what the others hold does not enter
            vz = vh.clone()
            bad = ~torch.isfinite(vz)
            fine = torch.where(bad, 0.0, vz)
            y = w @ fine
            if bad.any():
                for r in range(nq):
                    for j in (bad.any(-1) & see[r]).nonzero().flatten().tolist():
                        y[r] += torch.where(bad[j], w[r, j] * vz[j], 0.0)
            out[:, h] = y
            slack[:, h] = w @ fine.abs()
            lse[:, h] = (top + total.log())[:, 0]
        outs.append(out)
        lses.append(lse)
        slacks.append(slack)
        at += nq
    return torch.cat(outs), torch.cat(lses), torch.cat(slacks), big


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def check_attend(got, ref, dtype, dim, p_rounded):
    """Tolerance.  out = sum w v / sum w, rounded once: half a step of the value.  Scores: dim products added in 32 bits,
    each addition off by at most 2^-23 (the tensor cores may truncate) of the partial sums, which sum |q k| bounds, and a
    few roundings of the score itself and of the exponential (8 * 2^-24 of it): a weight's relative error is at most
    `ds`, numerator and denominator move by ds each.  p_rounded: weights rounded to 16 bits before the product with v,
    half a step each; otherwise two 16-bit parts, half a step squared."""
    out, lse = got
    ref_out, ref_lse, slack, big = ref
    h = half_step(dtype)
    ds = dim * 2.0 ** -23 * big + 8 * 2.0 ** -24 * (big + 8)
    fine = torch.isfinite(ref_out)
    o = out.double()
    assert torch.equal(torch.isnan(o), torch.isnan(ref_out))
    assert torch.equal(o[torch.isinf(ref_out)], ref_out[torch.isinf(ref_out)])
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps  # values below the type's range
    tol = h * ref_out.abs() + (2 * ds + (h if p_rounded else h * h) + 2.0 ** -20) * slack * (1 + h) + tiny
    err = (o - ref_out).abs()
    worst = float((err / tol.clamp_min(1e-300))[fine].max()) if fine.any() else 0.0
    assert worst <= 1.0, f"out: {worst:.2f} of the tolerance"
    if lse is not None:
        inf = torch.isinf(ref_lse)
        assert torch.equal(lse.double()[inf], ref_lse[inf])
        e = (lse.double() - ref_lse).abs()[~inf]
        lim = ds + 2.0 ** -22 + 4 * 2.0 ** -24 * ref_lse.abs()[~inf]
        assert (e <= lim).all(), f"lse: {float((e / lim).max()):.2f} of the tolerance"


def rotate_ref(x, pos, inv_freq, rot, interleaved, mscale):
    y = x.double().clone()
    half = rot // 2
    w = pos.double()[:, None] * inv_freq
    c, s = (w.cos() * mscale)[:, None], (w.sin() * mscale)[:, None]
    a, b = (y[..., 0:rot:2].clone(), y[..., 1:rot:2].clone()) if interleaved else (y[..., :half].clone(), y[..., half:rot].clone())
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * s, a * s + b * c
    else:
        y[..., :half], y[..., half:rot] = a * c - b * s, a * s + b * c
    return y


def mass_ref(ctxs, n_q, q, lse, prev=None, layer=0, scale=None, softcap=0.0, window=0, slopes=None, spans=None):
    out, at = [], 0
    for i, (c, nq) in enumerate(zip(ctxs, n_q)):
        k = c.rows[layer, 0].double()
        t, heads, dim = k.shape
        group = q.shape[1] // heads
        pos = torch.arange(t - nq, t, device=q.device)
        lo, hi = torch.zeros_like(pos), pos + 1
        if spans is not None:
            lo, hi = spans[at:at + nq, 0].long(), spans[at:at + nq, 1].long()
        if window:
            lo = torch.maximum(lo, pos + 1 - window)
        key = torch.arange(t, device=q.device)
        see = (key >= lo[:, None]) & (key < hi[:, None])
        m = torch.zeros(t, dtype=torch.float64, device=q.device)
        for h in range(q.shape[1]):
            x = q[at:at + nq, h].double() @ k[:, h // group].T * (dim ** -0.5 if scale is None else scale)
            if softcap:
                x = softcap * torch.tanh(x / softcap)
            if slopes is not None:
                x = x - slopes[h].double() * (pos[:, None] - key).abs()
            z = lse[at:at + nq, h].double()[:, None]
            m += torch.where(see & torch.isfinite(z), torch.exp(x - z), 0.0).sum(0)
        out.append(m + (prev[i, :t].double() if prev is not None else 0.0))
        at += nq
    return out


def prune_ref(scores, budget, sink, recent):
    t = len(scores)
    s = [(-math.inf, 1) if math.isnan(x) else (x, 0) for x in scores]  # a NaN ranks below -inf
    mid = sorted(range(sink, t - recent), key=lambda i: (-s[i][0], s[i][1], i))[:budget - sink - recent]
    return list(range(sink)) + sorted(mid) + list(range(t - recent, t))
