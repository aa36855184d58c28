"""Cases of the operators that compute with the paged KV pool's bytes, with their plain forms.

  store    rotary positions on new queries and keys, keys and values written into their cache slots
  attend   attention of a context's last tokens over its paged keys and values: one new token per
           sequence (the cache's length split and joined) or many (score cap, distance bias, document,
           prefix and window masks)
  mass     attention weight that every cached token received, added to a running sum
  prune    token eviction: a new context of the first, the latest and the heaviest tokens of another

A pool is [layers][blocks][K, V][block_size][kv heads][head_dim]; a context is a list of block numbers
and a token count.  Each case's inputs are made by ``prepare`` from a seed; ``run`` is one call of the
operator, in elementary torch operations or, where ``own`` is set, through the library.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ------------------------------------------------------------------------------------------ the cases
def _case(kind, **kw):
    c = {"kind": kind, "pick": 1, "n": 1, "heads": 32, "kv_heads": 8, "dim": 128, "block": 16, "dtype": "bf16", "layers": 1,
         "prefix": 0, "len_lo": 1, "len_hi": 1, "new_lo": 1, "new_hi": 1, "mask": "causal", "window": 0, "docs": 1,
         "softcap": 0.0, "slopes": False, "rot": 0, "pairs": "half", "base": 10000.0, "factor": 1.0, "mscale": 1.0,
         "pos0": 0, "budget": 0, "sink": 0, "recent": 0}
    c.update(kw)
    return c


def listed():
    return [
        # one decoding step of 16 agents: a token each, rotated and written behind its 8.7 K-token context
        _case("store", name="store_decode_16_agents", n=16, len_lo=8699, len_hi=8699, rot=128, base=500000.0),
        # prefill of an 8187-token context whose positions start far out: interleaved pairs, half of the head
        # rotated, frequencies stretched for a long context
        _case("store", name="store_prefill_far", len_lo=8187, len_hi=8187, new_lo=8187, new_hi=8187, rot=64,
              pairs="interleaved", factor=8.0, mscale=1.2, pos0=1000003),
        # the shortest decoding step: the tiny pool's one agent, where latency counts
        _case("attend", name="decode_tiny", heads=4, kv_heads=2, dim=64, len_lo=508, len_hi=508),
        # 16 agents forked from one 8187-token context, 512 tokens of their own each: one token per agent
        _case("attend", name="decode_16_forked_agents", n=16, prefix=8187, len_lo=512, len_hi=512),
        # one long context of the 70B shape (64 query heads), alone on the GPU: the cache's length is split
        _case("attend", name="decode_one_long", heads=64, dtype="f16", len_lo=33787, len_hi=33787),
        # 64 agents of a churning pool, ragged lengths around 2 K, blocks of 64, capped scores
        _case("attend", name="decode_64_ragged", n=64, block=64, len_lo=509, len_hi=8100, softcap=30.0, pick=5),
        # the agents' continuations: 512 new tokens each on a private 8187-token context, causal
        _case("attend", name="extend_16_agents", n=16, len_lo=8699, len_hi=8699, new_lo=512, new_hi=512),
        # a composed context of four documents, all of it computed anew under the document mask, capped scores
        _case("attend", name="extend_documents", len_lo=10007, len_hi=10007, new_lo=10007, new_hi=10007, mask="docs",
              docs=4, softcap=50.0),
        # the decoding step's weights per cached token, for eviction: 16 agents with ragged private contexts
        _case("mass", name="mass_decode_16_agents", n=16, len_lo=2048, len_hi=8699, pick=7),
        # an observation window of 32 queries at the end of a long prompt
        _case("mass", name="mass_window_long", len_lo=32763, len_hi=32763, new_lo=32, new_hi=32),
        # the tiny pool's context down to a quarter
        _case("prune", name="prune_tiny", heads=4, kv_heads=2, dim=64, layers=2, len_lo=507, len_hi=507, budget=125,
              sink=4, recent=32),
        # an 8B-shaped context of 8187 tokens down to 2048, all layers
        _case("prune", name="prune_8b", layers=32, len_lo=8187, len_hi=8187, budget=2048, sink=4, recent=512),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["store", "attend", "attend", "extend", "mass", "prune"])
    kv = rng.choice([1, 2, 4, 8])
    c = dict(pick=rng.randrange(1 << 20), kv_heads=kv, heads=kv * rng.choice([1, 2, 3, 4, 5, 8]), dim=rng.choice([64, 64, 96, 128, 128, 128]),
             block=rng.choice([8, 16, 16, 32, 64]), dtype=rng.choice(["bf16", "bf16", "f16"]))
    if kind == "store":
        n = _log(rng, 1, 64)
        c.update(n=n, rot=rng.choice([c["dim"], c["dim"] // 2, c["dim"] // 4]), pairs=rng.choice(["half", "interleaved"]),
                 base=rng.choice([10000.0, 500000.0]), factor=rng.choice([1.0, 4.0, 8.0]), mscale=rng.choice([1.0, 1.2]),
                 pos0=rng.choice([0, 0, rng.randrange(1 << 20)]))
        c["new_lo"] = _log(rng, 1, max(1, 2000 // n))
        c["new_hi"] = c["new_lo"] + rng.randrange(1 + c["new_lo"])
        c["len_lo"] = c["new_hi"] + _log(rng, 1, 2000) - 1
        c["len_hi"] = c["len_lo"] + rng.randrange(500)
        return _case("store", **c)
    mask = dict(softcap=rng.choice([0.0, 0.0, 30.0, 50.0]), slopes=rng.random() < 0.3)
    if kind == "attend":
        n = _log(rng, 1, 64)
        c.update(mask, n=n, prefix=rng.choice([0, 0, _log(rng, 16, 4000)]), len_lo=_log(rng, 1, 1000))
        c["len_hi"] = _log(rng, c["len_lo"], max(c["len_lo"], 60000 // n))
        c["new_lo"] = c["new_hi"] = min(c["len_lo"], rng.choice([1, 1, 1, 2, 4]))
        if rng.random() < 0.25:
            c.update(mask="window", window=_log(rng, 16, 4000))
        return _case("attend", **c)
    if kind == "extend":
        n = _log(rng, 1, 8)
        c.update(mask, n=n, new_lo=_log(rng, 5, max(16, 2500 // n)))
        c["new_hi"] = c["new_lo"] + rng.randrange(1 + c["new_lo"] // 2)
        c["len_lo"] = c["new_hi"] + _log(rng, 1, 4000) - 1
        c["len_hi"] = c["len_lo"] + rng.randrange(1000)
        c["mask"] = rng.choice(["causal", "docs", "prefix", "window"])
        c["docs"] = rng.choice([2, 3, 7])
        c["window"] = _log(rng, 16, 4000) if c["mask"] == "window" else 0
        return _case("attend", **c)
    if kind == "mass":
        n = _log(rng, 1, 16)
        c.update(mask, n=n, len_lo=_log(rng, 64, 2000))
        c["len_hi"] = _log(rng, c["len_lo"], max(c["len_lo"], 40000 // n))
        c["new_lo"] = c["new_hi"] = rng.choice([1, 1, 8, 32])
        return _case("mass", **c)
    length = _log(rng, 20, 30000)
    c.update(layers=_log(rng, 1, 16), len_lo=length, len_hi=length, budget=max(1, int(length * rng.uniform(0.05, 0.9))))
    c["sink"] = min(rng.choice([0, 4]), c["budget"] // 2)
    c["recent"] = rng.randrange(1 + (c["budget"] - c["sink"]) // 2)
    return _case("prune", **c)


# ------------------------------------------------------------------------------------------ the inputs
def _lengths(case):
    """Tokens of every sequence (a shared prefix apart), and how many of them are new."""
    r = random.Random(case["pick"])
    lens = [_log(r, case["len_lo"], case["len_hi"]) for _ in range(case["n"])]
    new = [min(ln, r.randint(case["new_lo"], case["new_hi"])) for ln in lens]
    return lens, new


def _nblk(case, tokens):
    return -(-tokens // case["block"])


def _spans(case, total, new):
    """The keys [lo, hi) that each new token sees, where that is not [0, its position]: an int32 pair a row."""
    r = random.Random(case["pick"] + 1)
    out = []
    for t, q in zip(total, new):
        starts = [0] + sorted(r.randrange(t) for _ in range(case["docs"] - 1))
        prefix = r.randrange(t + 1)
        for p in range(t - q, t):
            if case["mask"] == "docs":
                out.append((max(s for s in starts if s <= p), p + 1))
            else:
                out.append((0, max(p + 1, prefix)))
    return out


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    bs, hkv, d, heads = case["block"], case["kv_heads"], case["dim"], case["heads"]
    lens, new = _lengths(case)
    total = [case["prefix"] + ln for ln in lens]
    s = {"case": case, "total": total, "new": new, "scale": 1.0 / math.sqrt(d)}

    # block numbers: a context takes the next ones of a permuted free list
    shared = case["prefix"] // bs
    need = [_nblk(case, t) - shared for t in total]
    root = _nblk(case, case["prefix"])
    extra = _nblk(case, case["budget"])
    nb = root + sum(need) + extra
    order = random.Random(seed).sample(range(nb), nb)
    tables, at = [], root
    for k in need:
        tables.append(order[:shared] + order[at:at + k])
        at += k
    wide = max(len(t) for t in tables)
    s["tables"] = torch.tensor([t + [0] * (wide - len(t)) for t in tables], device=dev)
    s["len"] = torch.tensor(total, device=dev)
    s["nq"] = torch.tensor(new, device=dev)

    pool = torch.empty(case["layers"], nb, 2, bs, hkv, d, dtype=dt, device=dev)
    if own:  # the pool's handle and contexts, as a serving program holds them
        from paper_2607_10987_b200 import KVPool

        kv = KVPool(case["layers"], hkv, d, bs, 2, nb, len(total) + 2, max(wide, root, extra), free_order=order, pool_tensor=pool)
        s["kv"] = kv
        junk = torch.empty(kv.bpt * max([case["prefix"]] + lens), dtype=torch.uint8, device=dev)
        if case["prefix"]:
            first = _done(kv.imp(junk, case["prefix"]))
            s["ctxs"] = _done(kv.fork(first, len(total)))
            _done(kv.append(s["ctxs"], lens, [junk] * len(total)))
        else:
            s["ctxs"] = [_done(kv.imp(junk, t)) for t in total]
        torch.cuda.synchronize()
    torch.randn(pool.shape, generator=g, device=dev, dtype=dt, out=pool)
    s["pool"] = pool

    rows = sum(new)
    if case["kind"] != "prune":
        s["q"] = torch.randn(rows, heads, d, generator=g, device=dev, dtype=dt)
    if case["kind"] == "store":
        s["k"] = torch.randn(rows, hkv, d, generator=g, device=dev, dtype=dt)
        s["v"] = torch.randn(rows, hkv, d, generator=g, device=dev, dtype=dt)
        half = case["rot"] // 2
        s["inv_freq"] = case["base"] ** (-torch.arange(half, device=dev, dtype=torch.float64) / half) / case["factor"]
        s["pos"] = torch.tensor([case["pos0"] + p for t, q in zip(total, new) for p in range(t - q, t)], device=dev)
        s["q_out"] = torch.empty_like(s["q"])
        if own:
            from paper_2607_10987_b200.binding import Rope

            s["rope"] = Rope(case["rot"], s["inv_freq"], interleaved=case["pairs"] == "interleaved", mscale=case["mscale"])
    if case["kind"] in ("attend", "mass"):
        s["q"] *= 2.0  # scores with a spread of two: some keys stand out
        s["spans"] = None
        if case["mask"] in ("docs", "prefix"):
            s["spans"] = torch.tensor(_spans(case, total, new), dtype=torch.int32, device=dev)
        s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, heads + 1, device=dev) / heads) if case["slopes"] else None
    if case["kind"] == "mass":
        s["lse"] = _attend_plain(s)["lse"]
        s["prev"] = torch.rand(len(total), max(total), generator=g, device=dev)
        s["out"] = torch.zeros_like(s["prev"])
    if case["kind"] == "prune":
        t = total[0]
        s["scores"] = torch.rand(t, generator=g, device=dev) ** 4
        s["scores"][torch.randint(0, t, (t // 4,), generator=g, device=dev)] = 0.0  # tokens nobody looked at: ties
        s["new_table"] = torch.tensor(order[at:at + extra], device=dev)
        s["kept"] = torch.empty(case["budget"], dtype=torch.int32, device=dev)
        s["kept_scores"] = torch.empty(case["budget"], device=dev)
    torch.cuda.synchronize()
    return s


def _done(answer):
    status, value = answer
    if status != 0:
        raise RuntimeError(f"status {status}")
    return value


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"store": _store_own, "attend": _attend_own, "mass": _mass_own, "prune": _prune_own}[kind](s)
    return {"store": _store_plain, "attend": _attend_plain, "mass": _mass_plain, "prune": _prune_plain}[kind](s)


def _store_own(s):
    _done(s["kv"].store(0, s["ctxs"], s["new"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], rope=s["rope"],
                        pos=s["pos"] if s["case"]["pos0"] else None))
    return {"q": s["q_out"], "pool": s["pool"]}


def _attend_own(s):
    c = s["case"]
    out, lse = _done(s["kv"].attend(0, s["ctxs"], s["new"], s["q"], scale=s["scale"], softcap=c["softcap"],
                                    window=c["window"], slopes=s["slopes"], spans=s["spans"]))
    return {"out": out, "lse": lse}


def _mass_own(s):
    c = s["case"]
    _done(s["kv"].attn_mass(0, s["ctxs"], s["new"], s["q"], s["lse"], s["out"], prev=s["prev"], scale=s["scale"],
                            softcap=c["softcap"], window=c["window"], slopes=s["slopes"], spans=s["spans"]))
    return {"mass": s["out"]}


def _prune_own(s):
    c = s["case"]
    ctx = _done(s["kv"].prune(s["ctxs"][0], s["scores"], c["budget"], sink=c["sink"], recent=c["recent"], kept=s["kept"],
                              kept_scores=s["kept_scores"]))
    _done(s["kv"].evict([ctx]))  # the next pass finds the same blocks free
    return {"kept": s["kept"], "kept_scores": s["kept_scores"], "pool": s["pool"]}


# ------------------------------------------------------------------------------------------ plain forms
def _rows(s):
    """Of every packed query row: its sequence, its place among that sequence's new tokens, its position."""
    seq = torch.repeat_interleave(torch.arange(len(s["new"]), device=s["nq"].device), s["nq"], output_size=sum(s["new"]))
    j = torch.arange(seq.numel(), device=seq.device) - (torch.cumsum(s["nq"], 0) - s["nq"])[seq]
    return seq, j, (s["len"] - s["nq"])[seq] + j


def _rotate_plain(x, pos, s):
    c = s["case"]
    rot, half = c["rot"], c["rot"] // 2
    angle = pos.double()[:, None, None] * s["inv_freq"]
    cos, sin = (angle.cos() * c["mscale"]).float(), (angle.sin() * c["mscale"]).float()
    y = x.float()
    head = y[..., :rot]
    a, b = (head[..., 0::2], head[..., 1::2]) if c["pairs"] == "interleaved" else (head[..., :half], head[..., half:])
    a, b = a * cos - b * sin, a * sin + b * cos
    head = torch.stack((a, b), -1).flatten(-2) if c["pairs"] == "interleaved" else torch.cat((a, b), -1)
    return torch.cat((head, y[..., rot:]), -1).to(x.dtype)


def _store_plain(s):
    bs = s["case"]["block"]
    seq, _, slot = _rows(s)
    block = s["tables"][seq, slot // bs]
    s["q_out"].copy_(_rotate_plain(s["q"], s["pos"], s))
    s["pool"][0, block, 0, slot % bs] = _rotate_plain(s["k"], s["pos"], s)
    s["pool"][0, block, 1, slot % bs] = s["v"]
    return {"q": s["q_out"], "pool": s["pool"]}


def _scores_plain(s):
    """Masked scores [sequence, kv head, head of its group, new token, key], values, and where the packed rows are."""
    c = s["case"]
    seq, j, pos = _rows(s)
    n, widest = len(s["new"]), max(s["new"])
    hkv, group = c["kv_heads"], c["heads"] // c["kv_heads"]
    k = s["pool"][0, :, 0][s["tables"]].flatten(1, 2).float()
    v = s["pool"][0, :, 1][s["tables"]].flatten(1, 2).float()
    q = torch.zeros(n, widest, hkv, group, c["dim"], device=k.device)
    q[seq, j] = s["q"].float().view(-1, hkv, group, c["dim"])
    x = torch.einsum("nqhgd,nthd->nhgqt", q, k) * s["scale"]
    if c["softcap"]:
        x = c["softcap"] * torch.tanh(x / c["softcap"])
    t = torch.arange(k.shape[1], device=k.device)
    if s["slopes"] is not None:
        at = torch.zeros(n, widest, device=k.device, dtype=pos.dtype)
        at[seq, j] = pos
        x = x - s["slopes"].view(hkv, group, 1, 1) * (at[..., None] - t).abs()[:, None, None]
    lo, hi = torch.zeros_like(pos), pos + 1
    if s["spans"] is not None:
        lo, hi = s["spans"][:, 0].long(), s["spans"][:, 1].long()
    if c["window"]:
        lo = torch.maximum(lo, pos + 1 - c["window"])
    see = torch.zeros(n, widest, t.numel(), dtype=torch.bool, device=k.device)
    see[seq, j] = (t >= lo[:, None]) & (t < hi[:, None])
    return torch.where(see[:, None, None], x, -math.inf), v, seq, j


def _attend_plain(s):
    x, v, seq, j = _scores_plain(s)
    top = x.amax(-1, keepdim=True).nan_to_num(neginf=0.0)
    p = torch.exp(x - top)
    norm = p.sum(-1, keepdim=True)
    y = torch.einsum("nhgqt,nthd->nqhgd", p / norm.clamp_min(1e-37), v)
    lse = (top + norm.log())[..., 0].permute(0, 3, 1, 2)
    return {"out": y[seq, j].flatten(1, 2).to(s["q"].dtype), "lse": lse[seq, j].flatten(1, 2)}


def _mass_plain(s):
    c = s["case"]
    x, _, seq, j = _scores_plain(s)
    lse = torch.zeros(len(s["new"]), max(s["new"]), c["heads"], device=x.device)
    lse[seq, j] = s["lse"]
    lse = lse.view(*lse.shape[:2], c["kv_heads"], -1).permute(0, 2, 3, 1)[..., None]
    mass = torch.exp(x - lse).sum((1, 2, 3))
    here = torch.arange(s["out"].shape[1], device=x.device) < s["len"][:, None]
    s["out"].copy_(torch.where(here, s["prev"] + mass[:, :s["out"].shape[1]], s["out"]))
    return {"mass": s["out"]}


def _prune_plain(s):
    c, bs = s["case"], s["case"]["block"]
    t = s["total"][0]
    end = t - c["recent"]
    middle = torch.sort(s["scores"][c["sink"]:end], descending=True, stable=True).indices[:c["budget"] - c["sink"] - c["recent"]]
    at = torch.arange(t, device=middle.device)
    kept = torch.cat((at[:c["sink"]], torch.sort(middle + c["sink"]).values, at[end:]))
    i = torch.arange(c["budget"], device=middle.device)
    rows = s["pool"][:, s["tables"][0][kept // bs], :, kept % bs]
    s["pool"][:, s["new_table"][i // bs], :, i % bs] = rows
    s["kept"].copy_(kept)
    s["kept_scores"].copy_(s["scores"][kept])
    return {"kept": s["kept"], "kept_scores": s["kept_scores"], "pool": s["pool"]}


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def _visible(case):
    """Pairs (new token, key) that the mask leaves, and the distinct cached tokens that a pass reads."""
    lens, new = _lengths(case)
    total = [case["prefix"] + ln for ln in lens]
    if case["mask"] in ("docs", "prefix"):
        spans = _spans(case, total, new)
    else:
        w = case["window"] or 1 << 40
        spans = [(max(0, p + 1 - w), p + 1) for t, q in zip(total, new) for p in range(t - q, t)]
    pairs, tokens, at, shared = 0, 0, 0, None
    for q in new:
        mine = spans[at:at + q]
        at += q
        pairs += sum(max(0, b - a) for a, b in mine)
        seen = [(a, b) for a, b in mine if b > a]
        if not seen:
            continue
        a, b = min(x for x, _ in seen), max(y for _, y in seen)
        tokens += b - max(a, min(b, case["prefix"]))
        if a < case["prefix"]:
            shared = a if shared is None else min(a, shared)
    return pairs, tokens + (case["prefix"] - shared if shared is not None else 0)


def work(case):
    lens, new = _lengths(case)
    rows, row = sum(new), case["kv_heads"] * case["dim"] * 2
    q = rows * case["heads"] * case["dim"] * 2
    if case["kind"] == "store":
        turned = rows * (case["heads"] + case["kv_heads"]) * case["rot"] // 2
        return {"bytes": 2 * q + 4 * rows * row + (8 * rows if case["pos0"] else 0), "flops": 6 * turned}
    if case["kind"] == "prune":
        return {"bytes": 4 * case["budget"] * case["layers"] * row + 4 * lens[0] + 8 * case["budget"], "flops": 0}
    pairs, tokens = _visible(case)
    flops = 2 * pairs * case["heads"] * case["dim"]
    if case["kind"] == "mass":
        return {"bytes": q + tokens * row + 4 * rows * case["heads"] + 8 * sum(lens), "flops": flops}
    return {"bytes": 2 * q + 2 * tokens * row + 4 * rows * case["heads"], "flops": 2 * flops}


# ------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = _inputs_only(case, seed)
    return {"store": _store_exact, "attend": _attend_exact, "mass": _mass_exact, "prune": _prune_exact}[case["kind"]](s)


def _inputs_only(case, seed):
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def _cached(s, i, which, layer=0):
    """Keys (0) or values (1) of sequence i, token by token: [tokens, kv heads, dim] in 64 bits."""
    bs = s["case"]["block"]
    t = s["total"][i]
    blocks = s["tables"][i, :-(-t // bs)]
    return s["pool"][layer, blocks, which].reshape(-1, s["case"]["kv_heads"], s["case"]["dim"])[:t].double()


def _turned_exact(x, pos, s):
    """Every pair of a head is a complex number, turned by exp(i * position * frequency)."""
    c = s["case"]
    x = x.double().clone()
    r = c["rot"]
    if r:
        inter = c["pairs"] == "interleaved"
        pair = x[..., :r].reshape(*x.shape[:-1], r // 2, 2) if inter else x[..., :r].reshape(*x.shape[:-1], 2, r // 2).transpose(-1, -2)
        z = torch.view_as_complex(pair.contiguous())
        z = z * torch.polar(torch.full_like(s["inv_freq"], c["mscale"]), torch.zeros_like(s["inv_freq"])) \
            * torch.exp(1j * (pos.double()[:, None] * s["inv_freq"]))[:, None]
        pair = torch.view_as_real(z)
        x[..., :r] = pair.flatten(-2) if inter else pair.transpose(-1, -2).flatten(-2)
    return x


def _store_exact(s):
    bs = s["case"]["block"]
    pool = s["pool"].double()
    k = _turned_exact(s["k"], s["pos"], s)
    at = 0
    for i, (t, q) in enumerate(zip(s["total"], s["new"])):
        slot = torch.arange(t - q, t, device=pool.device)
        block = s["tables"][i][slot // bs]
        pool[0, block, 0, slot % bs] = k[at:at + q]
        pool[0, block, 1, slot % bs] = s["v"][at:at + q].double()
        at += q
    return {"q": _turned_exact(s["q"], s["pos"], s), "pool": pool}


def _weights_exact(s):
    """For each sequence and kv head: its rows (packed), log weights [group, new token, key] with -inf where masked."""
    c = s["case"]
    group, at = c["heads"] // c["kv_heads"], 0
    for i, (t, q) in enumerate(zip(s["total"], s["new"])):
        k = _cached(s, i, 0)
        p = torch.arange(t - q, t, device=k.device)
        lo, hi = torch.zeros_like(p), p + 1
        if s["spans"] is not None:
            lo, hi = s["spans"][at:at + q].long().unbind(1)
        if c["window"]:
            lo = torch.maximum(lo, p - c["window"] + 1)
        key = torch.arange(t, device=k.device)
        hide = (key < lo[:, None]) | (key >= hi[:, None])
        for h in range(c["kv_heads"]):
            x = s["q"][at:at + q, h * group:(h + 1) * group].double().transpose(0, 1) @ k[:, h].T * s["scale"]
            if c["softcap"]:
                x = torch.tanh(x / c["softcap"]) * c["softcap"]
            if s["slopes"] is not None:
                x -= s["slopes"][h * group:(h + 1) * group, None, None].double() * (p[:, None] - key).abs()
            yield i, h, slice(at, at + q), x.masked_fill_(hide, -math.inf)
        at += q


def _attend_exact(s):
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=s["q"].device)
    for i, h, rows, x in _weights_exact(s):
        z = torch.logsumexp(x, -1)
        y = torch.exp(x - z.clamp_min(-1e300)[..., None]) @ _cached(s, i, 1)[:, h]
        out[rows, h * group:(h + 1) * group] = y.transpose(0, 1)
        lse[rows, h * group:(h + 1) * group] = z.T
    return {"out": out, "lse": lse}


def _mass_exact(s):
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    out = s["out"].double()
    for i, t in enumerate(s["total"]):
        out[i, :t] = s["prev"][i, :t].double()
    for i, h, rows, x in _weights_exact(s):
        lse = s["lse"][rows, h * group:(h + 1) * group].double().T[..., None]
        out[i, :s["total"][i]] += torch.exp(x - lse).sum((0, 1))
    return {"mass": out}


def _prune_exact(s):
    c, bs, t = s["case"], s["case"]["block"], s["total"][0]
    score = s["scores"].tolist()
    middle = sorted(range(c["sink"], t - c["recent"]), key=lambda i: (-score[i], i))[:c["budget"] - c["sink"] - c["recent"]]
    kept = list(range(c["sink"])) + sorted(middle) + list(range(t - c["recent"], t))
    table, new_table = s["tables"][0].tolist(), s["new_table"].tolist()
    pool = s["pool"]
    old = torch.tensor([table[i // bs] * bs + i % bs for i in kept], device=pool.device)
    new = torch.tensor([new_table[i // bs] * bs + i % bs for i in range(len(kept))], device=pool.device)
    for layer in range(c["layers"]):
        for which in range(2):
            flat = pool[layer, :, which].reshape(-1, c["kv_heads"], c["dim"])
            flat[new] = flat[old]
            pool[layer, :, which] = flat.view(pool[layer, :, which].shape)
    return {"kept": torch.tensor(kept, dtype=torch.int32), "kept_scores": torch.tensor([score[i] for i in kept], dtype=torch.float64),
            "pool": pool}
