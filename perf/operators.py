"""The operators around a key/value cache held in 4 bits, as timed cases.

  append   queries and keys of a chunk normed per head, rotated by their position, keys and values written to the cache in 4
           bits (Kv4Cache.append); the new slots are read back as the numbers they stand for (Kv4Cache.read)
  attend   causal attention of a chunk's queries over the cache, with the attention weight of every slot added to the ledger
           where the case asks for it (Kv4Cache.attend)
  evict    the slots with the least accumulated weight given up, the recent ones kept, what stays moved to the front
           (Kv4Cache.evict); the slots that stay are read back

Head layouts are those of the framework's model shapes (12/2, 28/4, 40/8 heads of 128 channels, 4/2 of 64).  Lengths: single
tokens, catch-ups of 10 to 125 tokens, chunks of up to 4096, contexts of some hundred to some thousand slots.

`own` false: the plain form, elementary torch operations in 32 bits.  `own` true: the framework's calls.
"""
import math
import random

import torch

own = False

EPS, THETA = 1e-6, 1e6
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
SHAPES = {"tiny": (4, 2, 64), "1.5b": (12, 2, 128), "7b": (28, 4, 128), "32b": (40, 8, 128)}


# ---- cases ----

def _heads(shape):
    nq, nkv, d = SHAPES[shape]
    return dict(nq=nq, nkv=nkv, d=d)


def _chunk(op, shape, n, ctx, rows, **more):
    return dict(op=op, **_heads(shape), n=n, ctx_lo=ctx[0], ctx_hi=ctx[1], rows_lo=rows[0], rows_hi=rows[1], **more)


def listed():
    return [
        # one token of the speculative model: the call of every decode step and layer, all latency
        dict(name="append_1p5b_1", **_chunk("append", "1.5b", 1, (1300, 1300), (1, 1), norm=False, weights=False, mix=1)),
        # one token each of sixteen problems, heads with norms, a ledger for a later eviction
        dict(name="append_32b_16x1", **_chunk("append", "32b", 16, (128, 6000), (1, 1), norm=True, weights=True, mix=2)),
        # ragged catch-ups of a dozen problems
        dict(name="append_7b_ragged", **_chunk("append", "7b", 12, (128, 1500), (10, 60), norm=True, weights=True, mix=3)),
        # the target reading a whole chunk
        dict(name="append_32b_4096", **_chunk("append", "32b", 1, (4096, 4096), (4096, 4096), norm=True, weights=False, mix=4)),
        # one token of the speculative model on a finished trace
        dict(name="attend_1p5b_1", **_chunk("attend", "1.5b", 1, (4607, 4607), (1, 1), weights=False, mix=5)),
        # one token each of sixteen problems, weights kept for a later eviction
        dict(name="attend_32b_16x1", **_chunk("attend", "32b", 16, (500, 6000), (1, 1), weights=True, mix=6)),
        # the target catching up on what the speculative model wrote since the last hand-over
        dict(name="attend_32b_86", **_chunk("attend", "32b", 1, (4096, 4096), (86, 86), weights=False, mix=7)),
        # ragged catch-ups of a dozen problems, weights kept
        dict(name="attend_7b_ragged", **_chunk("attend", "7b", 12, (128, 1500), (10, 60), weights=True, mix=8)),
        # one full chunk on as many cached slots: the largest
        dict(name="attend_32b_4096", **_chunk("attend", "32b", 1, (4096, 4096), (4096, 4096), weights=False, mix=9)),
        # a speculative model's context brought back to its budget after some steps, all layers at once
        dict(name="evict_1p5b_28", op="evict", **_heads("1.5b"), layers=28, n=1, ctx_lo=577, ctx_hi=577, keep=512, recent=128, mix=10),
        # sixteen problems of the target, one layer, some below the budget
        dict(name="evict_32b_16", op="evict", **_heads("32b"), layers=1, n=16, ctx_lo=500, ctx_hi=6000, keep=1024, recent=256, mix=11),
        # a long prompt cut to a quarter, once, in two layers
        dict(name="evict_32b_16k", op="evict", **_heads("32b"), layers=2, n=1, ctx_lo=16385, ctx_hi=16385, keep=4096, recent=1000, mix=12),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "evict"))
    shape = rng.choice(("tiny", "1.5b", "7b", "32b", "32b"))
    n = _between(rng, 1, 16)
    mix = rng.randrange(1 << 30)
    if op == "evict":
        keep = _between(rng, 16, 4096)
        hi = _between(rng, keep + 1, max(keep + 2, 16384 // n))
        return dict(op=op, **_heads(shape), layers=1 if n > 4 else _between(rng, 1, 4), n=n, ctx_lo=max(1, min(hi, keep // 2)) if n > 1 else hi, ctx_hi=hi,
                    keep=keep, recent=rng.randrange(0, keep // 2), mix=mix)
    rows = _between(rng, 1, 4096 // n)
    ctx = _between(rng, 1, max(8, 4096 // n)) if rows > 64 else _between(rng, 1, 16384 if n == 1 else 6000)
    ctx_lo, rows_lo = rng.randrange(0, ctx + 1), max(1, rows // rng.choice((1, 2, 4)))
    if op == "append":
        return dict(**_chunk(op, shape, n, (ctx_lo, ctx), (rows_lo, rows), norm=rng.random() < 0.7, weights=rng.random() < 0.5, mix=mix))
    return dict(**_chunk(op, shape, n, (ctx_lo, ctx), (rows_lo, rows), weights=rng.random() < 0.5, mix=mix))


def _spans(case):
    """(sequence, cached slots, position of the first new row, new rows) of each sequence of a call."""
    r = random.Random(case["mix"])
    got = []
    for j in range(case["n"]):
        ctx = r.randint(case["ctx_lo"], case["ctx_hi"])
        if case["op"] == "evict":
            if j == 0:
                ctx = case["ctx_hi"]
            got.append((1 + j, ctx, ctx + 11 * j, 0))
        else:  # a sequence that has been thinned out is at a later position than it has slots
            got.append((1 + j, ctx, ctx + r.choice((0, 0, 37)), r.randint(case["rows_lo"], case["rows_hi"])))
    return got


def work(case):
    nq, nkv, d, spans = case["nq"], case["nkv"], case["d"], _spans(case)
    rows, slot = sum(s[3] for s in spans), 2 * nkv * (d // 2 + d // 32)
    if case["op"] == "append":
        return {"bytes": rows * (2 * (nq + 2 * nkv) * d + 2 * nq * d + 2 * slot + 4 * nkv * d + (8 * nkv if case["weights"] else 0)), "flops": rows * (nq + nkv) * d * 8}
    if case["op"] == "attend":
        seen = sum(rows * ctx + rows * (rows + 1) // 2 for _, ctx, _, rows in spans)
        held = sum(ctx + rows for _, ctx, _, rows in spans)
        return {"bytes": held * (slot + (8 * nkv if case["weights"] else 0)) + 4 * rows * nq * d, "flops": 4 * nq * d * seen}
    moved = stay = 0.0
    for _, ctx, _, _ in spans:
        k = min(ctx, case["keep"])
        stay += k
        if ctx > k:
            late, fixed = ctx - k, min(case["recent"], ctx - k)
            moved += fixed + (late - fixed) * (k - case["recent"]) / (ctx - case["recent"])
    held = sum(s[1] for s in spans)
    return {"bytes": case["layers"] * (8 * nkv * (held + stay) + 2 * slot * moved + stay * (slot + 4 * nkv * d)), "flops": case["layers"] * nkv * held}


# ---- inputs ----

def _quantise(x):
    """Groups of 32 channels of fp32 `x` -> (codes, two to a byte, scale bytes)."""
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = g.abs().amax(-1)
    fine = torch.isfinite(top)
    m, e = torch.frexp(torch.where(fine, top, 0.0))      # top = m 2^e, m in [0.5, 1)
    s = torch.clamp(torch.where(m > 0.875, e - 2, e - 3), -100, 125)
    s = torch.where(top > 0, s, -100)
    y = torch.where(fine[..., None], g, 0.0) * _power(-s)[..., None]
    a = y.abs()
    code = ((a > 0.25).to(torch.int32) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
            + 8 * torch.signbit(y)).reshape(x.shape)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), torch.where(fine, s + 127, 255).to(torch.uint8)


def _power(s):
    """2^s in fp32, s in [-126, 127]."""
    return ((s.to(torch.int32) + 127) << 23).view(torch.float32)


def _values(codes, scales):
    """What codes and scale bytes stand for, in fp32."""
    table = torch.tensor([*LEVELS, *(-v for v in LEVELS)], device=codes.device)
    v = table[torch.stack((codes & 15, codes >> 4), -1).to(torch.int64)]
    s = scales.to(torch.int32)
    unit = torch.where(s == 255, math.nan, _power(s - 127))
    return (v.reshape(*codes.shape[:-1], scales.shape[-1], 32) * unit[..., None]).reshape(*codes.shape[:-1], -1)


def _planes(case, cache, n_seq, max_seq):
    """The cache's four planes, [layer][sequence][kv head][slot][bytes], as the framework lays them out in one buffer."""
    d, at, got = case["d"], 0, []
    for per_slot in (d // 2, d // 2, d // 32, d // 32):
        shape = (case["layers"], n_seq, case["nkv"], max_seq, per_slot)
        got.append(cache[at:at + math.prod(shape)].view(shape))
        at += -(-math.prod(shape) // 256) * 256
    return got


def prepare(case, seed):
    case = dict(case, layers=case.get("layers", 2))       # append and attend: the second of two layers
    nq, nkv, d, spans, dev = case["nq"], case["nkv"], case["d"], _spans(case), "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    normal = lambda *shape: torch.randn(shape, generator=g, device=dev)  # noqa: E731
    rows, n_seq = sum(s[3] for s in spans), case["n"] + 2
    max_seq = max(ctx + r for _, ctx, _, r in spans) + 5
    max_pos = max(pos + r for _, _, pos, r in spans) + 1
    cfg = dict(n_layers=case["layers"], n_seq=n_seq, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, max_seq=max_seq, max_rows=max(rows, 1),
               max_pos=max_pos, rms_eps=EPS)
    size = sum(-(-case["layers"] * n_seq * nkv * max_seq * b // 256) * 256 for b in (d // 2, d // 2, d // 32, d // 32))
    cache = torch.zeros(size, dtype=torch.uint8, device=dev)
    planes = _planes(case, cache, n_seq, max_seq)
    gain = 1 + 2.5 * (torch.rand(nkv, 1, d, generator=g, device=dev) < 0.04)          # some channels of the keys are larger
    for layer in range(case["layers"]) if case["op"] == "evict" else (1,):
        for seq, ctx, _, r in spans:
            for p, x in ((0, normal(nkv, ctx + r, d) * gain), (1, normal(nkv, ctx + r, d))):
                planes[p][layer, seq, :, :ctx + r], planes[2 + p][layer, seq, :, :ctx + r] = _quantise(x)
    angle = torch.arange(max_pos, device=dev, dtype=torch.float64)[:, None] * THETA ** (-torch.arange(d // 2, device=dev, dtype=torch.float64) * 2 / d)
    s = dict(case=case, spans=spans, cfg=cfg, cache=cache, planes=planes, rope=torch.stack((angle.cos(), angle.sin()), -1).float().contiguous())
    at = torch.tensor([(seq, ctx, pos, r) for seq, ctx, pos, r in spans], device=dev)
    if case["op"] == "append":
        s["qkv"] = (normal(rows, (nq + 2 * nkv) * d) * 2).bfloat16()
        s["q_norm"], s["k_norm"] = ((1 + 0.2 * normal(2, d)).bfloat16() if case["norm"] else (None, None))
    if case["op"] == "attend":
        s["q"] = (normal(rows, nq, d) * 1.5).bfloat16()
    if case["op"] == "evict" or case.get("weights"):
        w = torch.exp(2.5 * normal(case["layers"], n_seq, nkv, max_seq) - (3 if case["op"] == "evict" else 10))   # few slots have most of the weight
        w = torch.where(torch.rand(w.shape, generator=g, device=dev) < 0.1, 0.0, w)       # some none, so that there are ties
        slots = torch.arange(max_seq, device=dev)
        held = torch.zeros(n_seq, dtype=torch.int64, device=dev).index_copy_(0, at[:, 0], at[:, 1])
        s["weights"] = torch.where(slots < held[:, None, None], w, 0.0).contiguous()
        # a context that was thinned out before: its slots are in no order
        order = torch.rand(w.shape, generator=g, device=dev).masked_fill_(slots >= held[:, None, None], 2.0).argsort(-1)
        first = torch.zeros(n_seq, dtype=torch.int64, device=dev).index_copy_(0, at[:, 0], at[:, 2] - at[:, 1])
        s["positions"] = (order + first[:, None, None]).to(torch.int32)
        s["weights_to"], s["positions_to"] = torch.zeros_like(s["weights"]), torch.zeros_like(s["positions"])
    # which row of a padded [sequence][row] grid each row is, and the reverse
    s["owner"] = torch.repeat_interleave(torch.arange(case["n"], device=dev), at[:, 3])
    s["inside"] = torch.arange(rows, device=dev) - (torch.cumsum(at[:, 3], 0) - at[:, 3])[s["owner"]]
    s["at"] = at
    if own:
        from paper_2504_12329_amd import binding as B
        s["kv"] = B.Kv4Cache(cfg, rope=s["rope"], cache=cache)
        s["plan"] = B.Kv4Spans(spans)
        s["stay"] = B.Kv4Spans([(seq, 0, 0, min(ctx, case.get("keep", 0))) for seq, ctx, _, _ in spans])
        if "weights" in s:
            s["ledger"], s["ledger_to"] = B.Kv4Ledger(s["weights"], s["positions"]), B.Kv4Ledger(s["weights_to"], s["positions_to"])
    return s


# ---- the operators ----

def run(s):
    return globals()["_%s_%s" % (s["case"]["op"], "own" if own else "plain")](s)


def _with_ledger(s, got):
    return dict(got, weights=s["weights"][1, 1:-1], positions=s["positions"][1, 1:-1]) if "weights" in s else got


def _append_own(s):
    q = s["kv"].append(1, s["plan"], s["qkv"], s["q_norm"], s["k_norm"], s.get("ledger"))
    k, v = s["kv"].read(1, 2, s["plan"])
    return _with_ledger(s, {"q": q, "k": k[0], "v": v[0]})


def _attend_own(s):
    out = s["kv"].attend(1, s["plan"], s["q"], s.get("ledger"))
    return {"out": out, "weights": s["weights"][1, 1:-1]} if "weights" in s else {"out": out}


def _evict_own(s):
    c = s["case"]
    s["kv"].evict(0, c["layers"], s["plan"], c["keep"], c["recent"], s["ledger"], s["ledger_to"])
    k, v = s["kv"].read(0, c["layers"], s["stay"])
    return {"weights": s["weights_to"][:, 1:-1, :, :c["keep"]], "positions": s["positions_to"][:, 1:-1, :, :c["keep"]], "k": k, "v": v}


def _pairwise(x):
    """Sum over the last axis, neighbours first: a fixed order."""
    while x.shape[-1] > 1:
        x = x[..., 0::2] + x[..., 1::2]
    return x


def _append_plain(s):
    c = s["case"]
    nq, nkv, d = c["nq"], c["nkv"], c["d"]
    x = s["qkv"].float().view(-1, nq + 2 * nkv, d)
    q, k, v = x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:]
    if c["norm"]:
        q, k = ((y * (1.0 / torch.sqrt(_pairwise(y * y) / d + EPS))) * w.float() for y, w in ((q, s["q_norm"]), (k, s["k_norm"])))
    at = s["rope"][s["at"][s["owner"], 2] + s["inside"]][:, None]
    cos, sin = at[..., 0], at[..., 1]
    turn = lambda y: torch.cat((y[..., :d // 2] * cos - y[..., d // 2:] * sin, y[..., d // 2:] * cos + y[..., :d // 2] * sin), -1)  # noqa: E731
    q, k = turn(q).bfloat16(), _quantise(turn(k))
    v = _quantise(v)
    seq, slot = s["at"][s["owner"], 0], s["at"][s["owner"], 1] + s["inside"]
    for plane, x in zip(s["planes"], (k[0], v[0], k[1], v[1])):
        plane[1, seq, :, slot] = x
    if "weights" in s:
        s["weights"][1, seq, :, slot] = 0.0
        s["positions"][1, seq, :, slot] = (s["at"][s["owner"], 2] + s["inside"]).to(torch.int32)[:, None]
    return _with_ledger(s, {"q": q, "k": _values(*k).bfloat16(), "v": _values(*v).bfloat16()})


def _attend_plain(s):
    c = s["case"]
    n, nq, nkv, d, g = c["n"], c["nq"], c["nkv"], c["d"], c["nq"] // c["nkv"]
    held = max(ctx + r for _, ctx, _, r in s["spans"])
    most = max(r for _, _, _, r in s["spans"])
    k, v = (_values(s["planes"][p][1, 1:1 + n, :, :held], s["planes"][2 + p][1, 1:1 + n, :, :held]).view(n * nkv, held, d) for p in (0, 1))
    q = torch.zeros(n, most, nq, d, device=k.device)
    q[s["owner"], s["inside"]] = s["q"].float()
    q = q.view(n, most, nkv, g, d).transpose(1, 2).reshape(n * nkv, most * g, d)
    ctx, rows = s["at"][:, 1], s["at"][:, 3]
    i, slot = torch.arange(most, device=k.device), torch.arange(held, device=k.device)
    sees = (slot <= (ctx[:, None] + i)[..., None]) & (i < rows[:, None])[..., None]         # [sequence][row][slot]
    x = torch.bmm(q, k.transpose(1, 2).contiguous()).view(n, nkv, most, g, held) * d ** -0.5
    x = torch.where(sees[:, None, :, None], x, -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    x = x / x.sum(-1, keepdim=True)
    x = torch.where(sees[:, None, :, None], x, 0.0)
    out = torch.bmm(x.view(n * nkv, most * g, held), v).view(n, nkv, most, g, d).transpose(1, 2)[s["owner"], s["inside"]].reshape(-1, nq, d).bfloat16()
    if not c["weights"]:
        return {"out": out}
    s["weights"][1, 1:1 + n, :, :held] += x.sum((2, 3))
    return {"out": out, "weights": s["weights"][1, 1:-1]}


def _evict_plain(s):
    c = s["case"]
    n, keep, nkv, d = c["n"], c["keep"], c["nkv"], c["d"]
    ctx, pos = s["at"][:, 1], s["at"][:, 2]
    w, p = s["weights"][:, 1:-1], s["positions"][:, 1:-1]
    slot = torch.arange(w.shape[-1], device=w.device)
    held = (slot < ctx[:, None])[:, None]                                                   # [sequence][1][slot]
    key = torch.where(p >= (pos - c["recent"])[:, None, None], math.inf, w)
    key = torch.where(held, key, -1.0)
    order = torch.where(held, p, 2 ** 31 - 1).argsort(dim=-1, stable=True)                      # by position, then by weight
    order = order.gather(-1, torch.sort(key.gather(-1, order), dim=-1, descending=True, stable=True).indices)
    stays = torch.zeros_like(key, dtype=torch.bool).scatter_(-1, order[..., :keep], True) & held
    # freed slots in front take the kept ones behind, in order
    freed, late = ~stays & held & (slot < keep), stays & (slot >= keep)
    behind = torch.where(late, slot, 2 ** 31 - 1).sort(-1).values[..., :keep]
    behind = torch.nn.functional.pad(behind, (0, keep - behind.shape[-1]))
    source = torch.where(freed[..., :keep], behind.gather(-1, (freed[..., :keep].cumsum(-1) - 1).clamp_(min=0)), slot[:keep].expand(behind.shape))
    there = (slot[:keep] < ctx[:, None])[:, None]
    s["weights_to"][:, 1:-1, :, :keep] = torch.where(there, w.gather(-1, source), s["weights_to"][:, 1:-1, :, :keep])
    s["positions_to"][:, 1:-1, :, :keep] = torch.where(there, p.gather(-1, source), s["positions_to"][:, 1:-1, :, :keep])
    at = source[..., None]
    for plane in s["planes"]:
        plane[:, 1:-1, :, :keep] = plane[:, 1:-1].gather(-2, at.expand(*at.shape[:-1], plane.shape[-1]))
    stay = torch.clamp(ctx, max=keep)
    owner = torch.repeat_interleave(torch.arange(n, device=w.device), stay, output_size=sum(min(a[1], keep) for a in s["spans"]))
    inside = torch.arange(owner.numel(), device=w.device) - (torch.cumsum(stay, 0) - stay)[owner]
    k, v = (_values(s["planes"][i][:, 1 + owner, :, inside], s["planes"][2 + i][:, 1 + owner, :, inside]).bfloat16().transpose(0, 1).contiguous()
            for i in (0, 1))
    return {"weights": s["weights_to"][:, 1:-1, :, :keep], "positions": s["positions_to"][:, 1:-1, :, :keep], "k": k, "v": v}


# ---- the definitions in 64 bits, apart from the plain forms ----

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"append": _append_exact, "attend": _attend_exact, "evict": _evict_exact}[case["op"]](s)


def _nearest64(x):
    """fp64 values as their 4-bit groups hold them, by the distance to every level."""
    out = torch.empty_like(x)
    for a in range(0, x.shape[-1], 32):
        g = x[..., a:a + 32]
        top = g.abs().amax(-1, keepdim=True)
        unit = 2.0 ** torch.ceil(torch.log2(top.clamp(min=1e-30) / 7))
        levels = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
        best = torch.zeros_like(g)
        for code in range(1, 8):
            high, middle = levels[code], (levels[code - 1] + levels[code]) / 2
            best = torch.where((g.abs() / unit > middle) | ((g.abs() / unit == middle) & (code % 2 == 0)), high, best)   # ties to the even code
        out[..., a:a + 32] = torch.sign(g) * best * unit
    return out


def _append_exact(s):
    c = s["case"]
    nq, nkv, d = c["nq"], c["nkv"], c["d"]
    x = s["qkv"].double().view(-1, nq + 2 * nkv, d)
    got = {"q": x[:, :nq], "k": x[:, nq:nq + nkv]}
    for name, w in (("q", s["q_norm"]), ("k", s["k_norm"])):
        y = got[name]
        if w is not None:
            y = y / ((y ** 2).mean(-1, keepdim=True) + EPS).sqrt() * w.double()
        z = torch.complex(y[..., :d // 2].contiguous(), y[..., d // 2:].contiguous())
        parts = []
        at = 0
        for _, _, pos, rows in s["spans"]:
            angle = torch.arange(pos, pos + rows, device=x.device, dtype=torch.float64)[:, None] / THETA ** (torch.arange(0, d, 2, device=x.device, dtype=torch.float64) / d)
            parts.append(z[at:at + rows] * torch.polar(torch.ones_like(angle), angle)[:, None])
            at += rows
        z = torch.cat(parts)
        got[name] = torch.cat((z.real, z.imag), -1)
    got.update(k=_nearest64(got["k"]), v=_nearest64(x[:, nq + nkv:].clone()))
    if "weights" in s:
        weights = s["weights"].double()[1, 1:-1]
        for j, (_, ctx, _, rows) in enumerate(s["spans"]):
            weights[j, :, ctx:ctx + rows] = 0.0
        got["weights"], got["positions"] = weights, None
    return got


def _held64(s, plane, layer, seq, n):
    """[kv head][slot][channel] of a sequence, from the bytes."""
    codes, scales = s["planes"][plane][layer, seq, :, :n], s["planes"][2 + plane][layer, seq, :, :n]
    size = torch.tensor(LEVELS, dtype=torch.float64, device=codes.device)
    out = torch.empty(*codes.shape[:-1], codes.shape[-1] * 2, dtype=torch.float64, device=codes.device)
    for half in (0, 1):
        nibble = (codes.to(torch.int64) >> (4 * half)) & 15
        out[..., half::2] = size[nibble & 7] * (1 - 2 * (nibble >> 3))
    return out * (2.0 ** (scales.to(torch.float64) - 127)).repeat_interleave(32, -1)


def _attend_exact(s):
    c = s["case"]
    nq, nkv, d = c["nq"], c["nkv"], c["d"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    weights = s["weights"].double()[1, 1:-1] if c["weights"] else None
    at = 0
    for j, (seq, ctx, _, rows) in enumerate(s["spans"]):
        n = ctx + rows
        k, v = _held64(s, 0, 1, seq, n), _held64(s, 1, 1, seq, n)
        hidden = torch.ones(rows, n, dtype=torch.bool, device="cuda").triu(ctx + 1)
        for h in range(nq):
            kv = h * nkv // nq
            x = (s["q"][at:at + rows, h].double() @ k[kv].t().contiguous()) / math.sqrt(d)
            p = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
            out[at:at + rows, h] = p @ v[kv]
            if weights is not None:
                weights[j, kv, :n] += p.sum(0)
        at += rows
    return {"out": out, "weights": weights} if weights is not None else {"out": out}


def _evict_exact(s):
    c, keep = s["case"], s["case"]["keep"]
    nkv = c["nkv"]
    weights = torch.zeros(c["layers"], c["n"], nkv, keep, dtype=torch.float64)
    layers_k, layers_v = [], []
    w_all, p_all = s["weights"].cpu(), s["positions"].cpu()
    for layer in range(c["layers"]):
        ks, vs = [], []
        for j, (seq, ctx, pos, _) in enumerate(s["spans"]):
            k, v = _held64(s, 0, layer, seq, ctx), _held64(s, 1, layer, seq, ctx)
            for_k, for_v = [], []
            for h in range(nkv):
                w, p = w_all[layer, seq, h, :ctx].tolist(), p_all[layer, seq, h, :ctx].tolist()
                ranked = sorted(range(ctx), key=lambda i: (p[i] < pos - c["recent"], -w[i] if p[i] < pos - c["recent"] else 0.0, p[i]))
                kept = set(ranked[:keep])
                late = iter(sorted(i for i in kept if i >= keep))
                source = [i if i in kept else next(late) for i in range(min(ctx, keep))]
                weights[layer, j, h, :len(source)] = torch.tensor([w[i] for i in source], dtype=torch.float64)
                index = torch.tensor(source, device=k.device)
                for_k.append(k[h, index])
                for_v.append(v[h, index])
            ks.append(torch.stack(for_k, 1))
            vs.append(torch.stack(for_v, 1))
        layers_k.append(torch.cat(ks))
        layers_v.append(torch.cat(vs))
    return {"weights": weights, "positions": None, "k": torch.stack(layers_k), "v": torch.stack(layers_v)}
