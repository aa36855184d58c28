"""Cases of sparse attention over the paged KV pool and of the batch's tables, with their plain forms.

  summarize  of every block and kv head, bounds of its keys per channel, in 8 bits with a power of two for scale
  select     for every query token and kv head, the blocks with the largest bound on a score
  attend     attention over the listed blocks alone
  tables     block tables, lengths, positions and cache slots of a batch, padded to a fixed shape

A pool is [layers][blocks][K, V][block_size][kv heads][head_dim]; a context is a list of block numbers and a token
count.  A block's summary is a record of [kv heads][2][head_dim] codes (upper, lower), then one exponent a head, filled
up to 16 bytes.  Each case's inputs are made by ``prepare`` from a seed; ``run`` is one call of the operator, in
elementary torch operations or, where ``own`` is set, through the library.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
MOST = 127.0 * 2.0 ** 113  # values beyond count as this
LEAST_EXP = -60


# ------------------------------------------------------------------------------------------ the cases
def _case(kind, **kw):
    c = {"kind": kind, "pick": 1, "n": 1, "heads": 32, "kv_heads": 8, "dim": 128, "block": 16, "dtype": "bf16", "layers": 1,
         "len_lo": 1, "len_hi": 1, "new_lo": 1, "new_hi": 1, "keep": 64, "sink": 1, "recent": 4, "softcap": 0.0, "slopes": False,
         "window": 0, "pad_rows": 0, "pad_tokens": 0}
    c.update(kw)
    return c


def listed():
    return [
        # one decoding step of 16 agents: the block of each agent's new token is summed up anew, in one layer
        _case("summarize", name="summarize_decode_16_agents", n=16, len_lo=8699, len_hi=8699),
        # a context that has just been imported: every block of all 32 layers
        _case("summarize", name="summarize_import_8b", layers=32, len_lo=8187, len_hi=8187, new_lo=8187, new_hi=8187),
        # the same step's choice: 64 of each agent's 544 blocks, for every kv head
        _case("select", name="select_decode_16_agents", n=16, len_lo=8699, len_hi=8699),
        # 32 agents with long ragged contexts, f16
        _case("select", name="select_decode_long_ragged", n=32, len_lo=8187, len_hi=65531, keep=128, dtype="f16", pick=3),
        # a prompt's last 128 tokens behind a long context: a choice for each of them
        _case("select", name="select_extend_long", len_lo=65531, len_hi=65531, new_lo=128, new_hi=128, keep=128),
        # the shortest decoding step: the tiny pool's one agent, a quarter of its blocks, where latency counts
        _case("attend", name="attend_tiny", heads=4, kv_heads=2, dim=64, len_lo=508, len_hi=508, keep=8, recent=2),
        # the 16 agents' decoding step over their 64 blocks
        _case("attend", name="attend_decode_16_agents", n=16, len_lo=8699, len_hi=8699),
        # 64 agents of a churning pool, ragged lengths, capped scores, up to 256 blocks each: the largest decoding step
        _case("attend", name="attend_decode_64_ragged", n=64, len_lo=2043, len_hi=32763, keep=256, softcap=30.0, pick=5),
        # the prompt's last 128 tokens over their 128 blocks each, f16
        _case("attend", name="attend_extend_long", len_lo=65531, len_hi=65531, new_lo=128, new_hi=128, keep=128, dtype="f16"),
        # tables and slots of the 16 agents' decoding step
        _case("tables", name="tables_decode_16_agents", n=16, len_lo=8699, len_hi=8699),
        # a mixed batch of 256 ragged contexts with up to 512 new tokens each, padded to a fixed shape
        _case("tables", name="tables_prefill_ragged", n=256, len_lo=509, len_hi=16381, new_lo=1, new_hi=512, pad_rows=32, pad_tokens=1000, pick=7),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["summarize", "select", "select", "attend", "attend", "tables"])
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 2, 3, 4, 5, 8, 16])
    c = dict(pick=rng.randrange(1 << 20), kv_heads=kv, heads=heads, dim=rng.choice([64, 96, 128, 128, 128]),
             block=rng.choice([8, 16, 16, 32, 64]), dtype=rng.choice(["bf16", "bf16", "f16"]))
    if kind == "tables":
        n = _log(rng, 1, 256)
        c.update(n=n, len_lo=_log(rng, 1, 2000), pad_rows=rng.choice([0, rng.randrange(32)]), pad_tokens=rng.choice([0, rng.randrange(500)]))
        c["len_hi"] = _log(rng, c["len_lo"], max(c["len_lo"], min(60000, 1000000 // n)))
        c["new_hi"] = _log(rng, 1, min(c["len_hi"], 512))
        return _case("tables", **c)
    if kind == "summarize":
        n = _log(rng, 1, 64)
        c.update(n=n, layers=_log(rng, 1, 16))
        most = 200000 // n // c["layers"]
        c["len_lo"] = _log(rng, 1, min(1000, most))
        c["len_hi"] = _log(rng, c["len_lo"], most)
        c["new_lo"], c["new_hi"] = rng.choice([(1, 1), (1, c["len_hi"]), (c["len_hi"], c["len_hi"])])
        return _case("summarize", **c)
    if rng.random() < 0.6:  # a token or a few each
        n = _log(rng, 1, 64)
        c.update(n=n, len_lo=_log(rng, 4, 4000))
        c["len_hi"] = _log(rng, c["len_lo"], max(c["len_lo"], 300000 // n))
        c["new_lo"] = c["new_hi"] = rng.choice([1, 1, 1, 2, 4]) if n < 16 else 1
    else:
        n = _log(rng, 1, 4)
        c.update(n=n, new_lo=_log(rng, 8, max(8, 96 * 32 // max(heads, 32) // n)))
        c["new_hi"] = c["new_lo"] + rng.randrange(1 + c["new_lo"] // 4)
        c["len_lo"] = c["new_hi"] + _log(rng, 1, 4000)
        c["len_hi"] = _log(rng, c["len_lo"], 4000 * min(c["block"], 15))
    c["keep"] = _log(rng, 4, 256)
    if kind == "attend":  # no more keys listed than in the largest listed case
        c["keep"] = max(4, min(c["keep"], 64 * 8 * 256 * 16 // (n * c["new_hi"] * kv * c["block"])))
        c.update(softcap=rng.choice([0.0, 0.0, 30.0, 50.0]), slopes=rng.random() < 0.3, window=rng.choice([0, 0, 0, _log(rng, 16, 4000)]))
    c["sink"] = rng.choice([0, 1, 1, 2])
    c["recent"] = rng.randint(1, 1 + (c["keep"] - c["sink"]) // 2)
    return _case(kind, **c)


# ------------------------------------------------------------------------------------------ the inputs
def _lengths(case):
    """Tokens of every sequence, and how many of them are new."""
    r = random.Random(case["pick"])
    lens = [_log(r, case["len_lo"], case["len_hi"]) for _ in range(case["n"])]
    return lens, [min(ln, r.randint(case["new_lo"], case["new_hi"])) for ln in lens]


def _record(case):
    """Bytes of a block's summary: codes, exponents, filling."""
    return case["kv_heads"] * 2 * case["dim"] + -(-case["kv_heads"] // 16) * 16


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    bs, hkv, d, heads, kind = case["block"], case["kv_heads"], case["dim"], case["heads"], case["kind"]
    dt = DTYPES[case["dtype"]]
    lens, new = _lengths(case)
    s = {"case": case, "total": lens, "new": new, "scale": 1.0 / math.sqrt(d)}

    # block numbers: a context takes the next ones of a permuted free list
    need = [-(-t // bs) for t in lens]
    nb, wide = sum(need) + 64, max(need)  # some blocks stay free
    order = random.Random(seed).sample(range(nb), nb)
    tables, at = [], 0
    for k in need:
        tables.append(order[at:at + k] + [0] * (wide - k))
        at += k
    s["tables"] = torch.tensor(tables, device=dev)
    s["len"] = torch.tensor(lens, device=dev)
    s["nq"] = torch.tensor(new, device=dev)
    s["need"] = torch.tensor(need, device=dev)

    row = 8 if kind == "tables" else hkv * d  # tables do not look at what the blocks hold
    pool = torch.empty(case["layers"], nb, 2, bs, row, dtype=dt, device=dev).view(case["layers"], nb, 2, bs, -1, 8 if kind == "tables" else d)
    if own:  # the pool's handle, sized for this batch, and its contexts: a token each, the others' slots reserved, no payload copied
        import numpy
        from paper_2607_10987_b200 import KVPool

        table = s["tables"].cpu().numpy()
        later = numpy.arange(1, wide) < numpy.array(need)[:, None]
        free = numpy.concatenate((table[:, 0], table[:, 1:][later], order[at:]))
        kv = KVPool(case["layers"], pool.shape[4], pool.shape[5], bs, 2, nb, len(lens) + 1, max(wide, at // 2), free_order=free, max_batch=len(lens),
                    pool_tensor=pool)
        one = torch.empty(kv.bpt, dtype=torch.uint8, device=dev)
        s["kv"], s["ctxs"] = kv, _done(kv.import_batch([one] * len(lens), [1] * len(lens)))
        longer = [(c, t - 1) for c, t in zip(s["ctxs"], lens) if t > 1]
        if longer:
            _done(kv.reserve(*zip(*longer)))
    torch.randn(pool.shape, generator=g, device=dev, dtype=dt, out=pool)
    s["pool"] = pool

    rows = sum(new)
    if kind in ("summarize", "select"):
        # keys of one context lean one way, as they do in a model; some channels are larger than others
        lean = torch.randn(len(lens), 1, 1, hkv, d, generator=g, device=dev)
        lean *= torch.rand(d, generator=g, device=dev) ** 2
        blocks = torch.tensor(order[:at], device=dev)
        owner = torch.repeat_interleave(torch.arange(len(lens), device=dev), s["need"])
        pool[:, blocks, 0] += lean[owner, 0].to(dt)
        s["summary"] = torch.randint(-128, 128, (case["layers"], nb, _record(case)), generator=g, device=dev, dtype=torch.int8)
    if kind in ("select", "attend"):
        s["q"] = torch.randn(rows, heads, d, generator=g, device=dev, dtype=dt) * 2.0
    if kind == "select":
        everything = dict(s, nq=s["len"], case=dict(case, layers=1))
        _summarize_plain(everything)
        s["blocks"] = torch.empty(rows, hkv, case["keep"], dtype=torch.int32, device=dev)
        s["scores"] = torch.empty(rows, hkv, case["keep"], device=dev)
    if kind == "attend":
        chance = torch.rand(rows, hkv, wide, generator=g, device=dev)
        s["blocks"] = _take(s, chance).to(torch.int32)
        s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, heads + 1, device=dev) / heads) if case["slopes"] else None
    if kind == "tables":
        r, t = len(lens) + case["pad_rows"], rows + case["pad_tokens"]
        s["shape"] = {"rows": r, "tokens": t, "cols": wide + 3}
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
        return {"summarize": _summarize_own, "select": _select_own, "attend": _attend_own, "tables": _tables_own}[kind](s)
    return {"summarize": _summarize_plain, "select": _select_plain, "attend": _attend_plain, "tables": _tables_plain}[kind](s)


def _summarize_own(s):
    _done(s["kv"].summarize(0 if s["case"]["layers"] == 1 else None, s["ctxs"], s["new"], s["summary"], s["pool"].dtype))
    return {"summary": s["summary"]}


def _select_own(s):
    c = s["case"]
    _done(s["kv"].select(0, s["ctxs"], s["new"], s["q"], s["summary"], c["keep"], sink=c["sink"], recent=c["recent"], blocks=s["blocks"],
                         scores=s["scores"]))
    return {"blocks": s["blocks"], "scores": s["scores"]}


def _attend_own(s):
    c = s["case"]
    out, lse = _done(s["kv"].attend_blocks(0, s["ctxs"], s["new"], s["q"], s["blocks"], scale=s["scale"], softcap=c["softcap"],
                                           window=c["window"], slopes=s["slopes"]))
    return {"out": out, "lse": lse}


def _tables_own(s):
    return _done(s["kv"].batch_tables(s["ctxs"], s["new"], **s["shape"]))


# ------------------------------------------------------------------------------------------ plain forms
def _rows(s):
    """Of every packed query row: its sequence, and its position."""
    seq = torch.repeat_interleave(torch.arange(len(s["new"]), device=s["nq"].device), s["nq"], output_size=sum(s["new"]))
    j = torch.arange(seq.numel(), device=seq.device) - (torch.cumsum(s["nq"], 0) - s["nq"])[seq]
    return seq, (s["len"] - s["nq"])[seq] + j


def _exponent(top):
    """The smallest whole number from LEAST_EXP with top <= 127 * 2^e."""
    m, e = torch.frexp(top)
    return torch.where(top == 0, LEAST_EXP, (e - 7 + (m > 127 / 128)).clamp_min(LEAST_EXP))


def _summarize_plain(s):
    c, bs, hkv, d = s["case"], s["case"]["block"], s["case"]["kv_heads"], s["case"]["dim"]
    column = torch.arange(s["tables"].shape[1], device=s["pool"].device)
    touched = (column < s["need"][:, None]) & ((column + 1) * bs > (s["len"] - s["nq"])[:, None])
    seq, column = touched.nonzero(as_tuple=True)
    block = s["tables"][seq, column]
    here = torch.arange(bs, device=block.device) < (s["len"][seq] - column * bs)[:, None]
    k = s["pool"][:c["layers"], block, 0].float()
    hi = torch.where(here[:, :, None, None], k.nan_to_num(MOST, MOST, -MOST).clamp(-MOST, MOST), -math.inf).amax(2)
    lo = torch.where(here[:, :, None, None], k.nan_to_num(-MOST, MOST, -MOST).clamp(-MOST, MOST), math.inf).amin(2)
    e = _exponent(torch.maximum(hi.abs(), lo.abs()).amax(-1))
    unit = torch.ldexp(torch.ones_like(hi[..., :1]), e[..., None])
    codes = torch.stack(((hi / unit).ceil(), (lo / unit).floor()), -2).to(torch.int8)
    s["summary"][:c["layers"], block, :hkv * 2 * d] = codes.flatten(2)
    s["summary"][:c["layers"], block, hkv * 2 * d:hkv * (2 * d + 1)] = e.to(torch.int8)
    return {"summary": s["summary"]}


def _take(s, score):
    """Lists of table columns from a score of every column ([row, kv head, column]): the first `sink`, the last `recent`, the
    best others, in ascending order, -1 behind the last."""
    c = s["case"]
    _, pos = _rows(s)
    last = (pos // c["block"])[:, None, None]
    column = torch.arange(score.shape[2], device=pos.device)
    bits = score.float().view(torch.int32)
    rank = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
    rank = torch.where((column < c["sink"]) | (column > last - c["recent"]), 1 << 40, rank)
    rank = torch.where(column <= last, rank, -1 << 40)
    rank = torch.nn.functional.pad(rank, (0, max(0, c["keep"] - rank.shape[2])), value=-1 << 40)
    rank, column = torch.sort(rank, dim=-1, descending=True, stable=True)
    column = torch.where(rank > -1 << 40, column, 1 << 40)[..., :c["keep"]].sort(-1).values
    return torch.where(column < 1 << 40, column, -1)


def _select_plain(s):
    c, hkv, d = s["case"], s["case"]["kv_heads"], s["case"]["dim"]
    group = c["heads"] // hkv
    seq, _ = _rows(s)
    q = s["q"].float().view(-1, hkv, group, d).nan_to_num(0.0, MOST, -MOST).clamp(-MOST, MOST)
    f = _exponent(q.abs().amax(-1))
    q = (q / torch.ldexp(torch.ones_like(q[..., :1]), f[..., None])).round()
    n, widest = len(s["new"]), max(s["new"])
    j = torch.arange(seq.numel(), device=seq.device) - (torch.cumsum(s["nq"], 0) - s["nq"])[seq]
    packed = torch.zeros(n, widest, hkv, group, 2 * d, device=q.device)
    packed[seq, j] = torch.cat((q.clamp_min(0), q.clamp_max(0)), -1)
    record = s["summary"][0][s["tables"]]
    codes = record[..., :hkv * 2 * d].unflatten(-1, (hkv, 2 * d)).float()
    e = record[..., hkv * 2 * d:hkv * (2 * d + 1)].to(torch.int32)
    dot = torch.einsum("nqhgd,nthd->nqhgt", packed, codes)[seq, j]  # whole numbers below 2^24: exact in any order
    power = (e.transpose(1, 2)[seq][:, :, None] + f[..., None]).double()
    score = (dot.double() * torch.exp2(power)).float().amax(2)
    column = _take(s, score)
    s["blocks"].copy_(column)
    s["scores"].copy_(torch.where(column >= 0, torch.gather(score, 2, column.clamp_min(0)), -math.inf))
    return {"blocks": s["blocks"], "scores": s["scores"]}


def _attend_plain(s):
    c, bs, hkv, d = s["case"], s["case"]["block"], s["case"]["kv_heads"], s["case"]["dim"]
    group = c["heads"] // hkv
    seq, pos = _rows(s)
    column = s["blocks"].long()
    t = (column[..., None] * bs + torch.arange(bs, device=column.device)).flatten(2)
    see = (column >= 0).repeat_interleave(bs, -1) & (t <= pos[:, None, None])
    if c["window"]:
        see &= t > pos[:, None, None] - c["window"]
    slot = torch.where(see, t, 0)
    block = s["tables"][seq[:, None, None], slot // bs]
    head = torch.arange(hkv, device=seq.device)[:, None]
    k, v = s["pool"][0, block, 0, slot % bs, head].float(), s["pool"][0, block, 1, slot % bs, head].float()
    q = s["q"].float().view(-1, hkv, group, d)
    x = torch.einsum("rhgd,rhtd->rhgt", q, k) * s["scale"]
    if c["softcap"]:
        x = c["softcap"] * torch.tanh(x / c["softcap"])
    if s["slopes"] is not None:
        x = x - s["slopes"].view(hkv, group, 1) * (pos[:, None, None] - t).abs()[:, :, None]
    x = torch.where(see[:, :, None], x, -math.inf)
    top = x.amax(-1, keepdim=True).nan_to_num(neginf=0.0)
    p = torch.exp(x - top)
    norm = p.sum(-1, keepdim=True)
    y = torch.einsum("rhgt,rhtd->rhgd", p / norm.clamp_min(1e-37), v)
    return {"out": y.flatten(1, 2).to(s["q"].dtype), "lse": (top + norm.log())[..., 0].flatten(1, 2)}


def _tables_plain(s):
    n, bs, shape, dev = len(s["new"]), s["case"]["block"], s["shape"], s["nq"].device
    seq, pos = _rows(s)
    tables = torch.full((shape["rows"], shape["cols"]), -1, dtype=torch.int32, device=dev)
    here = torch.arange(s["tables"].shape[1], device=dev) < s["need"][:, None]
    tables[:n, :s["tables"].shape[1]] = torch.where(here, s["tables"], -1)
    lens = torch.zeros(shape["rows"], dtype=torch.int32, device=dev)
    lens[:n] = s["len"]
    offsets = torch.full((shape["rows"] + 1,), seq.numel(), dtype=torch.int32, device=dev)
    offsets[:n] = torch.cumsum(s["nq"], 0) - s["nq"]
    token_row = torch.full((shape["tokens"],), -1, dtype=torch.int32, device=dev)
    token_row[:seq.numel()] = seq
    positions = torch.zeros(shape["tokens"], dtype=torch.int64, device=dev)
    positions[:seq.numel()] = pos
    slots = torch.full((shape["tokens"],), -1, dtype=torch.int64, device=dev)
    slots[:seq.numel()] = s["tables"][seq, pos // bs] * bs + pos % bs
    return {"tables": tables, "lens": lens, "offsets": offsets, "token_row": token_row, "positions": positions, "slots": slots}


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    lens, new = _lengths(case)
    bs, hkv, d, heads = case["block"], case["kv_heads"], case["dim"], case["heads"]
    seen = hkv * (2 * d + 1)  # what counts of a block's summary
    q = sum(new) * heads * d * 2
    if case["kind"] == "summarize":
        first = [(t - k) // bs for t, k in zip(lens, new)]
        blocks = sum(-(-t // bs) - f for t, f in zip(lens, first))
        keys = sum(t - f * bs for t, f in zip(lens, first)) * hkv * d * case["layers"]
        return {"bytes": 2 * keys + blocks * seen * case["layers"], "flops": 2 * keys}
    if case["kind"] == "tables":
        entries = sum(-(-t // bs) for t in lens)
        rows, tokens = case["n"] + case["pad_rows"], sum(new) + case["pad_tokens"]
        cols = max(-(-t // bs) for t in lens) + 3
        return {"bytes": 4 * entries + 4 * rows * cols + 4 * rows + 4 * (rows + 1) + 20 * tokens, "flops": 0}
    last = [[p // bs for p in range(t - k, t)] for t, k in zip(lens, new)]
    if case["kind"] == "select":
        pairs = sum(sum(b) + len(b) for b in last)
        return {"bytes": q + 8 * sum(new) * hkv * case["keep"] + sum(b[-1] + 1 for b in last) * seen, "flops": 2 * pairs * heads * d}
    # the listed keys that a token sees, as many as it may list; distinct ones by how likely a block is on no list
    keys = listed_keys = 0.0
    for t, b in zip(lens, last):
        missed = 1.0
        for i, at in enumerate(b):
            share = min(1.0, case["keep"] / (at + 1))
            p = t - len(b) + i
            see = min(p + 1, case["window"] or p + 1) * share
            keys += see
            missed *= 1.0 - share
        listed_keys += min(t, (case["window"] or t) + len(b)) * (1.0 - missed)
    return {"bytes": int(2 * q + 4 * sum(new) * heads + 4 * sum(new) * hkv * case["keep"] + 4 * listed_keys * hkv * d),
            "flops": int(4 * keys * heads * d)}


# ------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = _inputs_only(case, seed)
    return {"summarize": _summarize_exact, "select": _select_exact, "attend": _attend_exact, "tables": lambda s: None}[case["kind"]](s)


def _inputs_only(case, seed):
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def _scale_exact(top):
    e = torch.ceil(torch.log2(top.clamp_min(1e-300) / 127)).clamp_min(LEAST_EXP)
    e = torch.where(top <= 127 * torch.exp2(e - 1), e - 1, e)
    return torch.where(top > 127 * torch.exp2(e), e + 1, e).clamp_min(LEAST_EXP)


def _summarize_exact(s):
    """Block by block of a context, in 64 bits: the largest and smallest key of every channel in steps of a power of two."""
    c, bs, hkv, d = s["case"], s["case"]["block"], s["case"]["kv_heads"], s["case"]["dim"]
    out = s["summary"]
    for i, (t, q) in enumerate(zip(s["total"], s["new"])):
        for layer in range(c["layers"]):
            for full in (True, False):  # the whole blocks at once, then the last one's tokens
                first, end = ((t - q) // bs, t // bs) if full else (max((t - q) // bs, t // bs), -(-t // bs))
                if end <= first:
                    continue
                blocks = s["tables"][i, first:end]
                k = s["pool"][layer, blocks, 0][:, :bs if full else t - first * bs].double().clamp(-MOST, MOST)
                hi, lo = k.max(1).values, k.min(1).values
                e = _scale_exact(torch.stack((hi, -lo)).abs().amax((0, -1)))
                codes = torch.stack((torch.ceil(hi * torch.exp2(-e)[..., None]), torch.floor(lo * torch.exp2(-e)[..., None])), 2)
                out[layer, blocks, :hkv * 2 * d] = codes.reshape(len(blocks), -1).to(torch.int8)
                out[layer, blocks, hkv * 2 * d:hkv * (2 * d + 1)] = e.to(torch.int8)
    return {"summary": out}


def _select_exact(s):
    """Token by token: every channel's larger product, summed up in 64 bits; ranks by score, then by place."""
    c, bs, hkv, d = s["case"], s["case"]["block"], s["case"]["kv_heads"], s["case"]["dim"]
    group, at = c["heads"] // hkv, 0
    out = torch.full(s["blocks"].shape, -1, dtype=torch.int32)
    scores = torch.full(s["blocks"].shape, -math.inf, dtype=torch.float64)
    for i, (t, q) in enumerate(zip(s["total"], s["new"])):
        record = s["summary"][0, s["tables"][i]].double()
        for j in range(q):
            last = (t - q + j) // bs
            x = s["q"][at + j].double().clamp(-MOST, MOST).view(hkv, group, d)
            f = _scale_exact(x.abs().amax(-1))
            x = torch.round(x * torch.exp2(-f)[..., None])
            for h in range(hkv):
                code = record[:last + 1, h * 2 * d:(h + 1) * 2 * d].view(-1, 1, 2, d)
                e = record[:last + 1, hkv * 2 * d + h]
                dot = torch.maximum(code[:, :, 0] * x[h], code[:, :, 1] * x[h]).sum(-1)
                score = (dot * torch.exp2(e[:, None] + f[h])).amax(1).tolist()
                forced = [b for b in range(last + 1) if b < c["sink"] or b > last - c["recent"]]
                rest = sorted((b for b in range(c["sink"], last + 1 - c["recent"])), key=lambda b: (-score[b], b))
                kept = sorted(forced + rest[:c["keep"] - len(forced)])[:c["keep"]]
                out[at + j, h, :len(kept)] = torch.tensor(kept, dtype=torch.int32)
                scores[at + j, h, :len(kept)] = torch.tensor([score[b] for b in kept], dtype=torch.float64)
        at += q
    return {"blocks": out, "scores": scores}


def _attend_exact(s):
    """Token by token and head by head, in 64 bits, over the tokens that its list and its mask leave."""
    c, bs, hkv, d = s["case"], s["case"]["block"], s["case"]["kv_heads"], s["case"]["dim"]
    group, at = c["heads"] // hkv, 0
    dev = s["pool"].device
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=dev)
    within = torch.arange(bs, device=dev)
    for i, (t, q) in enumerate(zip(s["total"], s["new"])):
        flat = s["tables"][i]
        for j in range(q):
            p = t - q + j
            for h in range(hkv):
                column = s["blocks"][at + j, h].long()
                column = column[column >= 0]
                key = (column[:, None] * bs + within).flatten()
                key = key[(key <= p) & (key > p - (c["window"] or p + 1))]
                if not key.numel():
                    continue
                k, v = s["pool"][0, flat[key // bs], :, key % bs, h].double().unbind(1)
                x = s["q"][at + j, h * group:(h + 1) * group].double() @ k.T * s["scale"]
                if c["softcap"]:
                    x = torch.tanh(x / c["softcap"]) * c["softcap"]
                if s["slopes"] is not None:
                    x -= s["slopes"][h * group:(h + 1) * group, None].double() * (p - key)
                z = torch.logsumexp(x, -1)
                out[at + j, h * group:(h + 1) * group] = torch.exp(x - z[:, None]) @ v
                lse[at + j, h * group:(h + 1) * group] = z
        at += q
    return {"out": out, "lse": lse}
