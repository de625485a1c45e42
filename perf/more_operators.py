"""Drafted tokens and the target that verifies them over a key/value cache in pages, as timed cases.

  append   queries and keys of new rows normed per head, rotated by their position, keys and values written to the pages of their
           sequences (PagedCache.append)
  attend   attention of the new rows over the pages: causal, or each drafted row over the context and its own branch (PagedCache.attend)
  verify   the target's logits after every drafted row against given random numbers: which rows stay, and the token that follows them
           (DraftVerifier.verify)
  keep     keys and values of the branch that stays moved to consecutive slots, all layers at once (PagedCache.keep)

Head layouts and vocabularies are those of the framework's model shapes.  The rows of a span are the last decided token and the drafts after
it: chains and trees of 5 to 64 rows, single tokens where nothing is drafted, chunks of up to 4096 where a model catches up.

`own` false: the plain form, elementary torch operations in 32 bits (in 64 where a decision hangs on them).  `own` true: the framework's calls.
"""
import math
import random

import torch

own = False

EPS, THETA = 1e-6, 1e6
SHAPES = {"tiny": (4, 2, 64, 1024), "1.5b": (12, 2, 128, 151936), "7b": (28, 4, 128, 152064), "32b": (40, 8, 128, 152064)}
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---- cases ----

def _heads(shape):
    nq, nkv, d, _ = SHAPES[shape]
    return dict(nq=nq, nkv=nkv, d=d)


def _chunk(op, shape, n, ctx, rows, page, width=0, dtype="bf16", **more):
    """width: most drafts after one row; 0: each row follows the one before."""
    return dict(op=op, **_heads(shape), n=n, ctx_lo=ctx[0], ctx_hi=ctx[1], rows_lo=rows[0], rows_hi=rows[1], page=page, width=width, dtype=dtype, **more)


def _verify(vocab, n, rows, width, draft, heat, dtype, mix):
    """heat: 0 all sequences greedy, 1 none, 2 some."""
    return dict(op="verify", vocab=vocab, n=n, ctx_lo=0, ctx_hi=0, rows_lo=rows[0], rows_hi=rows[1], width=width, draft=draft, heat=heat, dtype=dtype, mix=mix)


def listed():
    return [
        # one token of the speculative model: the call of every drafting step and layer, all latency
        dict(name="append_1p5b_1", **_chunk("append", "1.5b", 1, (1300, 1300), (1, 1), 16, norm=False, rot=128, pairs="halves", mix=1)),
        # the target reading a whole chunk
        dict(name="append_32b_4096", **_chunk("append", "32b", 1, (4096, 4096), (4096, 4096), 64, norm=True, rot=128, pairs="halves", mix=2)),
        # one token of the speculative model on a finished trace
        dict(name="attend_1p5b_1", **_chunk("attend", "1.5b", 1, (4607, 4607), (1, 1), 16, mix=3)),
        # sixteen problems of very unequal length, a tree of 21 rows each
        dict(name="attend_32b_16x21", **_chunk("attend", "32b", 16, (500, 6000), (21, 21), 64, width=3, mix=4)),
        # one wide tree late in a long trace
        dict(name="attend_32b_64", **_chunk("attend", "32b", 1, (16000, 16000), (64, 64), 32, width=4, mix=5)),
        # ragged catch-ups of a dozen problems
        dict(name="attend_7b_ragged", **_chunk("attend", "7b", 12, (128, 1500), (10, 60), 16, dtype="fp16", mix=6)),
        # a chunk on as many cached slots
        dict(name="attend_32b_2048", **_chunk("attend", "32b", 1, (2048, 2048), (2048, 2048), 128, mix=7)),
        # the speculative model's own tree, brought together in 28 layers
        dict(name="keep_1p5b_1", **_chunk("keep", "1.5b", 1, (1300, 1300), (16, 16), 16, width=2, layers=28, mix=8)),
        # eight problems of the target, 64 layers
        dict(name="keep_32b_8", **_chunk("keep", "32b", 8, (20, 150), (21, 40), 16, width=3, layers=64, mix=9)),
        # one short chain of drafts
        dict(name="verify_1p5b_5", **_verify(151936, 1, (5, 5), 1, True, 1, "fp32", 10)),
        # sixteen problems, twenty drafts each, with the distributions that they were drawn from: the largest
        dict(name="verify_32b_16x21", **_verify(152064, 16, (21, 21), 1, True, 2, "fp32", 11)),
        # trees of 64 rows whose drafts were drawn independently after each row
        dict(name="verify_7b_4x64", **_verify(152064, 4, (64, 64), 4, True, 1, "bf16", 12)),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "verify", "verify", "keep"))
    shape = rng.choice(("tiny", "1.5b", "7b", "32b", "32b"))
    n, mix = _between(rng, 1, 16), rng.randrange(1 << 30)
    if op == "verify":
        vocab = rng.choice((SHAPES[shape][3], _between(rng, 17, 151936)))
        rows = _between(rng, 1, max(1, min(64, 320 // n)))
        draft = rng.random() < 0.7
        width = rng.choice((1, 1, 2, 3, 4))
        if draft and width > 1:           # every draft after the first of a row is one more look at the distributions
            rows = max(1, min(rows, 200 // n))
        return _verify(vocab, n, (max(1, rows // rng.choice((1, 2))), rows), width, draft, rng.choice((0, 1, 1, 2)), rng.choice(("fp32", "fp32", "bf16", "fp16")), mix)
    page, dtype = rng.choice((16, 16, 32, 64, 128, 256)), rng.choice(("bf16", "bf16", "fp16"))
    if op == "keep":
        rows = _between(rng, 2, 64)
        ctx = _between(rng, 1, 200)
        return _chunk(op, shape, min(n, 8), (rng.randrange(0, ctx + 1), ctx), (max(2, rows // 2), rows), min(page, 64), width=rng.choice((2, 3, 4)), dtype=dtype,
                      layers=_between(rng, 1, 32), mix=mix)
    tree = rng.random() < 0.5
    rows = _between(rng, 1, 64 if tree else 4096 // n if op == "append" else 2048 // n)
    ctx = _between(rng, 1, max(8, 2048 // n)) if rows > 64 else _between(rng, 1, 16384 if n == 1 else 6000)
    ctx, rows = (rng.randrange(0, ctx + 1), ctx), (max(1, rows // rng.choice((1, 2, 4))), rows)
    width = rng.choice((1, 2, 3, 4)) if tree else 0
    if op == "append":
        d = SHAPES[shape][2]
        return _chunk(op, shape, n, ctx, rows, page, width=width, dtype=dtype, norm=rng.random() < 0.6, rot=rng.choice((d, d, d // 2, d // 4)),
                      pairs=rng.choice(("halves", "halves", "neighbours")), mix=mix)
    return _chunk(op, shape, n, ctx, rows, page, width=width, dtype=dtype, mix=mix)


def _spans(case):
    """(sequence, cached slots, position of the first new row, new rows) of each sequence of a call, and the row that each row follows."""
    r = random.Random(case["mix"])
    spans, parents = [], []
    for j in range(case["n"]):
        ctx, rows = r.randint(case["ctx_lo"], case["ctx_hi"]), r.randint(case["rows_lo"], case["rows_hi"])
        spans.append((1 + j, ctx, ctx + r.choice((0, 0, 37)), rows))
        p, free = [-1], [case["width"]]
        for i in range(1, rows):
            at = i - 1 if case["width"] <= 1 else r.choice([k for k in range(max(0, i - 12), i) if free[k] > 0])
            free[at] -= 1
            free.append(case["width"])
            p.append(at)
        parents.append(p)
    return spans, parents


def _branches(parents):
    """For each row the rows from the first one to it."""
    got = []
    for i, p in enumerate(parents):
        got.append((got[p] if p >= 0 else []) + [i])
    return got


def _kept(case):
    """The branch of every sequence that stays, its first row left out: one of the longer ones, as where drafts are good."""
    r = random.Random(case["mix"] + 1)
    return [sorted((b[1:] for b in _branches(p)), key=len)[r.randrange(len(p) // 2, len(p))] for p in _spans(case)[1]]


def work(case):
    spans, parents = _spans(case)
    rows = sum(s[3] for s in spans)
    if case["op"] == "verify":
        size = {"fp32": 4, "bf16": 2, "fp16": 2}[case["dtype"]]
        inner = sum(len(set(p)) - 1 for p in parents) if case["draft"] else 0       # rows that drafts follow
        return {"bytes": (rows + inner) * case["vocab"] * size + 24 * rows, "flops": 4 * (rows + inner) * case["vocab"]}
    nq, nkv, d = case["nq"], case["nkv"], case["d"]
    if case["op"] == "append":
        return {"bytes": rows * (2 * (nq + 2 * nkv) * d * 2 + 4 * case["rot"]), "flops": rows * (nq + nkv) * d * 8}
    if case["op"] == "keep":
        moved = sum(sum(1 for i, x in enumerate(b) if x != i + 1) for b in _kept(case))
        return {"bytes": case["layers"] * moved * 2 * 2 * nkv * d * 2, "flops": 0}
    tree = case["width"] > 0
    seen = sum(s[3] * s[1] + (sum(map(len, _branches(p))) if tree else s[3] * (s[3] + 1) // 2) for s, p in zip(spans, parents))
    held = sum(s[1] + s[3] for s in spans)
    return {"bytes": held * 2 * nkv * d * 2 + 4 * rows * nq * d, "flops": 4 * nq * d * seen}


# ---- inputs ----

def _structure(s, spans, parents, dev):
    """What the plain forms need of the rows: owner, place, depth, branch, children."""
    n, most = len(spans), max(sp[3] for sp in spans)
    depth = [[len(b) - 1 for b in _branches(p)] for p in parents]
    sees = torch.zeros(n, most, most, dtype=torch.bool)
    for j, p in enumerate(parents):
        for i, b in enumerate(_branches(p)):
            sees[j, i, b] = True
    s["sees"] = sees.to(dev)
    s["at"] = torch.tensor(spans, device=dev)
    s["owner"] = torch.repeat_interleave(torch.arange(n, device=dev), s["at"][:, 3])
    s["inside"] = torch.cat([torch.arange(sp[3]) for sp in spans]).to(dev)
    s["depth"] = torch.tensor([x for d in depth for x in d], device=dev)
    s["deepest"] = max(max(d) for d in depth)
    s["most"] = most


def prepare(case, seed):
    spans, parents = _spans(case)
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    s = dict(case=case, spans=spans, parents=parents)
    _structure(s, spans, parents, dev)
    (_prepare_verify if case["op"] == "verify" else _prepare_cache)(s, g, dev)
    if own:
        from paper_2504_12329_amd import binding as B
        tree = case["op"] in ("verify", "keep") or case["width"] > 0
        s["plan"] = B.DraftSpans(spans, parents, device=dev) if tree else B.Kv4Spans(spans)
        if case["op"] == "verify":
            s["verifier"] = B.DraftVerifier(case["vocab"], len(s["owner"]), max_width=max(1, case["width"]), dtype=TYPES[case["dtype"]], device=dev)
        else:
            s["kv"] = B.PagedCache(s["cfg"], rope=s["rope"], table=s["table"], cache=s["cache"])
    return s


def _prepare_cache(s, g, dev):
    case, spans = s["case"], s["spans"]
    nq, nkv, d, page, t, layers = case["nq"], case["nkv"], case["d"], case["page"], TYPES[case["dtype"]], case.get("layers", 1)
    normal = lambda *shape: torch.randn(shape, generator=g, device=dev)  # noqa: E731
    rows = sum(sp[3] for sp in spans)
    need = [-(-(ctx + r) // page) for _, ctx, _, r in spans]
    n_seq, n_pages, max_pages = case["n"] + 2, sum(need) + 3, max(need) + 2
    max_pos, rot = max(pos + r for _, _, pos, r in spans) + 1, case.get("rot", d)
    s["cfg"] = dict(n_layers=layers, n_seq=n_seq, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, n_pages=n_pages, page_size=page, max_pages=max_pages,
                    max_rows=rows, max_pos=max_pos, dtype=t, rot_dim=rot, rot_pairs=case.get("pairs", "halves"), rms_eps=EPS)
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)                 # pages come in no order
    table = torch.full((n_seq, max_pages), -1, dtype=torch.int32, device=dev)
    for (seq, _, _, _), m, at in zip(spans, need, [sum(need[:j]) for j in range(len(need))]):
        table[seq, :m] = order[at:at + m]
    s["table"] = table
    s["cache"] = cache = torch.empty(2, layers, n_pages, nkv, page, d, dtype=t, device=dev)
    gain = 1 + 2.5 * (torch.rand(nkv, 1, d, generator=g, device=dev) < 0.04)                 # some channels of the keys are larger
    for layer in range(layers):
        cache[0, layer], cache[1, layer] = normal(n_pages, nkv, page, d) * gain, normal(n_pages, nkv, page, d)
    angle = torch.arange(max_pos, device=dev, dtype=torch.float64)[:, None] * THETA ** (-torch.arange(rot // 2, device=dev, dtype=torch.float64) * 2 / rot)
    s["rope"] = torch.stack((angle.cos(), angle.sin()), -1).float().contiguous()
    if case["op"] == "append":
        s["qkv"] = (normal(rows, (nq + 2 * nkv) * d) * 2).to(t)
        s["q_norm"], s["k_norm"] = ((1 + 0.2 * normal(2, d)).to(t) if case["norm"] else (None, None))
    if case["op"] == "attend":
        s["q"] = (normal(rows, nq, d) * 1.5).to(t)
    if case["op"] == "keep":
        kept = _kept(case)
        s["path"] = torch.full((case["n"], s["most"]), -1, dtype=torch.int32)
        for j, b in enumerate(kept):
            s["path"][j, :len(b)] = torch.tensor(b, dtype=torch.int32)
        s["path"] = s["path"].to(dev)
        s["accepted"] = torch.tensor([len(b) for b in kept], dtype=torch.int32, device=dev)


def _prepare_verify(s, g, dev):
    case, spans, parents = s["case"], s["spans"], s["parents"]
    vocab, t, width = case["vocab"], TYPES[case["dtype"]], max(1, case["width"])
    rows = sum(sp[3] for sp in spans)
    heat = [0.0 if case["heat"] == 0 or (case["heat"] == 2 and j % 4 == 3) else (1.0, 0.6, 0.8)[j % 3] for j in range(case["n"])]
    s["heat"] = heat
    s["target"], s["draft"] = (torch.empty(rows, vocab, dtype=t, device=dev) for _ in range(2))
    first = [sum(sp[3] for sp in spans[:j]) for j in range(len(spans))]
    parent = [-1 if p < 0 else first[j] + p for j, ps in enumerate(parents) for p in ps]
    nth = []                                                                                  # which of its parent's drafts a row is
    for i, p in enumerate(parent):
        nth.append(sum(1 for x in parent[:i] if x == p and p >= 0))
    tokens = torch.zeros(rows, dtype=torch.int32, device=dev)
    for i in range(rows):
        base = 4 * torch.randn(vocab, generator=g, device=dev)                                # the two models agree on most
        s["target"][i], s["draft"][i] = base, base + 0.9 * torch.randn(vocab, generator=g, device=dev)
        after = [c for c in range(rows) if parent[c] == i]
        T = heat[max(j for j in range(len(first)) if first[j] <= i)]
        for c in after:
            if case["draft"] and T > 0:                                                       # drawn from the draft's distribution
                noise = -torch.log(-torch.log(torch.rand(vocab, generator=g, device=dev).clamp_(1e-20, 1 - 1e-7)))
                tokens[c] = torch.argmax(s["draft"][i].float() / T + noise)
            else:                                                                             # its best ones
                tokens[c] = torch.topk(s["draft"][i].float(), nth[c] + 1).indices[nth[c]]
    s["tokens"] = tokens
    s["accept"] = torch.rand(rows, generator=g, device=dev, dtype=torch.float64)
    s["sample"] = torch.rand(case["n"], generator=g, device=dev, dtype=torch.float64)
    child = torch.full((rows, width), -1, dtype=torch.int64)
    for i, p in enumerate(parent):
        if p >= 0:
            child[p, nth[i]] = i
    s["child"], s["first"], s["width"] = child.to(dev), torch.tensor(first, device=dev), width
    s["heat_at"] = torch.tensor(heat, dtype=torch.float64, device=dev)


# ---- the operators ----

def run(s):
    return globals()["_%s_%s" % (s["case"]["op"], "own" if own else "plain")](s)


def _append_own(s):
    return {"q": s["kv"].append(0, s["plan"], s["qkv"], s["q_norm"], s["k_norm"]), "cache": s["cache"]}


def _attend_own(s):
    return {"out": s["kv"].attend(0, s["plan"], s["q"])}


def _keep_own(s):
    s["kv"].keep(0, s["case"]["layers"], s["plan"], s["path"], s["accepted"])
    return {"cache": s["cache"]}


def _verify_own(s):
    path, accepted, after = s["verifier"].verify(s["plan"], s["tokens"], s["target"], s["heat"], s["accept"], s["sample"], draft=s["draft"] if s["case"]["draft"] else None)
    return {"path": path, "accepted": accepted, "next": after}


def _places(s, slot):
    """(page, slot in it) of slots of the rows' sequences."""
    page = s["case"]["page"]
    return s["table"][s["at"][s["owner"], 0], slot // page].long(), slot % page


def _append_plain(s):
    c = s["case"]
    nq, nkv, d, rot, t = c["nq"], c["nkv"], c["d"], c["rot"], TYPES[c["dtype"]]
    x = s["qkv"].float().view(-1, nq + 2 * nkv, d)
    q, k, v = x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:]
    if c["norm"]:
        q, k = (y * (1.0 / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS)) * w.float() for y, w in ((q, s["q_norm"]), (k, s["k_norm"])))
    at = s["rope"][s["at"][s["owner"], 2] + (s["depth"] if c["width"] else s["inside"])][:, None]
    cos, sin = at[..., 0], at[..., 1]

    def turn(y):
        if c["pairs"] == "halves":
            a, b = y[..., :rot // 2], y[..., rot // 2:rot]
            turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        else:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        return torch.cat((turned, y[..., rot:]), -1)

    page, slot = _places(s, s["at"][s["owner"], 1] + s["inside"])
    s["cache"][0, 0, page, :, slot], s["cache"][1, 0, page, :, slot] = turn(k).to(t), v.to(t)
    return {"q": turn(q).to(t), "cache": s["cache"]}


def _attend_plain(s):
    c = s["case"]
    n, nq, nkv, d, g = c["n"], c["nq"], c["nkv"], c["d"], c["nq"] // c["nkv"]
    most, held = s["most"], max(ctx + r for _, ctx, _, r in s["spans"])
    pages = s["table"][s["at"][:, 0], :-(-held // c["page"])].clamp(min=0).long()
    k, v = (s["cache"][p, 0][pages].transpose(1, 2).reshape(n * nkv, -1, d)[:, :held].float().contiguous() for p in (0, 1))
    q = torch.zeros(n, most, nq, d, device=k.device)
    q[s["owner"], s["inside"]] = s["q"].float()
    q = q.view(n, most, nkv, g, d).transpose(1, 2).reshape(n * nkv, most * g, d)
    slot, ctx, rows = torch.arange(held, device=k.device), s["at"][:, 1], s["at"][:, 3]
    i = torch.arange(most, device=k.device)
    j = slot - ctx[:, None]                                                                       # row in a slot, negative for the context
    if c["width"]:
        new = s["sees"].gather(2, j.clamp(0, most - 1)[:, None].expand(n, most, held))
        sees = (j < 0)[:, None] | (new & (j < rows[:, None])[:, None])
    else:
        sees = j[:, None] <= i[:, None]
    sees = sees & (i < rows[:, None])[..., None]
    x = torch.bmm(q, k.transpose(1, 2).contiguous()).view(n, nkv, most, g, held) * d ** -0.5
    x = torch.where(sees[:, None, :, None], x, -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    x = x / x.sum(-1, keepdim=True)
    x = torch.where(sees[:, None, :, None], x, 0.0)
    out = torch.bmm(x.view(n * nkv, most * g, held), v).view(n, nkv, most, g, d).transpose(1, 2)[s["owner"], s["inside"]].reshape(-1, nq, d)
    return {"out": out.to(TYPES[c["dtype"]])}


def _keep_plain(s):
    seq, ctx = s["at"][:, 0], s["at"][:, 1]
    i = torch.arange(s["most"], device=seq.device)
    stays = i < s["accepted"][:, None]
    page = s["case"]["page"]
    source = torch.where(stays, ctx[:, None] + s["path"], ctx[:, None])                           # (what does not stay: the first row onto itself)
    into = torch.where(stays, ctx[:, None] + 1 + i, ctx[:, None])
    place = [(s["table"][seq[:, None], x // page].long(), x % page) for x in (source, into)]
    (p0, s0), (p1, s1) = place
    s["cache"][:, :, p1, :, s1] = s["cache"][:, :, p0, :, s0]
    return {"cache": s["cache"]}


def _distribution(x, heat):
    """Rows of logits over their sequences' temperatures, in 64 bits; greedy rows: all on the largest."""
    x = x.double()
    best = torch.zeros_like(x).scatter_(1, x.argmax(1, keepdim=True), 1.0)
    e = torch.exp((x - x.amax(1, keepdim=True)) / torch.where(heat > 0, heat, 1.0)[:, None])
    return torch.where((heat > 0)[:, None], e / e.sum(1, keepdim=True), best)


def _verify_plain(s):
    c, width, child = s["case"], s["width"], s["child"]
    heat = s["heat_at"][s["owner"]]
    rows = len(heat)
    p = _distribution(s["target"], heat)
    outcome = torch.full((rows,), -1, dtype=torch.int64, device=p.device)                         # the draft after each row that is accepted
    if c["draft"]:
        q = torch.where((heat > 0)[:, None], _distribution(s["draft"], heat), 0.0)
    a = torch.zeros(rows, dtype=torch.float64, device=p.device)
    b = torch.ones_like(a)
    left = p.clone()
    for k in range(width):
        at = child[:, k]
        there = (at >= 0) & (outcome < 0)
        t = s["tokens"][at.clamp(min=0)].long()
        if c["draft"]:
            pt, qt = p.gather(1, t[:, None])[:, 0], q.gather(1, t[:, None])[:, 0]
            good = torch.where(heat > 0, s["accept"][at.clamp(min=0)] * qt * b < (pt - a * qt).clamp(min=0.0), pt > 0)
        else:
            good = torch.where(heat > 0, s["accept"][at.clamp(min=0)] * b < left.gather(1, t[:, None])[:, 0], left.gather(1, t[:, None])[:, 0] > 0)
        outcome = torch.where(there & good, at, outcome)
        fails = there & ~good
        if c["draft"]:
            a = torch.where(fails, a + b, a)
            if k + 1 < width:
                b = torch.where(fails, (p - a[:, None] * q).clamp_(min=0.0).sum(1), b)
        else:
            left = left.scatter(1, t[:, None], torch.where(fails & (heat > 0), 0.0, left.gather(1, t[:, None])[:, 0])[:, None])
            b = left.sum(1)
    now, steps = s["first"], []
    for _ in range(s["most"]):
        ahead = outcome[now]
        steps.append(torch.where(ahead >= 0, ahead - s["first"], -1))
        now = torch.where(ahead >= 0, ahead, now)
    path = torch.stack(steps, 1)
    w = (p[now] - a[now, None] * q[now]).clamp_(min=0.0) if c["draft"] else left[now]
    w = torch.where((w.sum(1) > 0)[:, None], w, p[now])
    total = w.cumsum(1)
    chosen = (total <= s["sample"][:, None] * total[:, -1:]).sum(1)
    chosen = torch.where(s["heat_at"] > 0, chosen, p[now].argmax(1))
    return {"path": path.to(torch.int32), "accepted": (path >= 0).sum(1).to(torch.int32), "next": chosen.to(torch.int32)}


# ---- the definitions in 64 bits, apart from the plain forms ----

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"append": _append_exact, "attend": _attend_exact, "keep": _keep_exact, "verify": _verify_exact}[case["op"]](s)


def _append_exact(s):
    c = s["case"]
    nq, nkv, d, rot = c["nq"], c["nkv"], c["d"], c["rot"]
    x = s["qkv"].double().view(-1, nq + 2 * nkv, d)
    got = []
    for y, w in ((x[:, :nq], s["q_norm"]), (x[:, nq:nq + nkv], s["k_norm"])):
        if w is not None:
            y = y / ((y ** 2).mean(-1, keepdim=True) + EPS).sqrt() * w.double()
        z = y.clone()
        one, two = (slice(0, rot // 2), slice(rot // 2, rot)) if c["pairs"] == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
        at = 0
        for (_, _, pos, rows), p in zip(s["spans"], s["parents"]):
            where = [len(b) - 1 for b in _branches(p)] if c["width"] else list(range(rows))
            turn = (pos + torch.tensor(where, dtype=torch.float64, device=x.device))[:, None, None] / THETA ** (torch.arange(0, rot, 2, dtype=torch.float64, device=x.device) / rot)
            n = y[at:at + rows]
            z[at:at + rows, :, one] = n[..., one] * turn.cos() - n[..., two] * turn.sin()
            z[at:at + rows, :, two] = n[..., one] * turn.sin() + n[..., two] * turn.cos()
            at += rows
        got.append(z)
    cache, at = s["cache"].double(), 0
    table = s["table"].tolist()
    for seq, ctx, _, rows in s["spans"]:
        done = 0
        while done < rows:                                                                        # a page, or the part of it that is new
            page, first = table[seq][(ctx + done) // c["page"]], (ctx + done) % c["page"]
            m = min(rows - done, c["page"] - first)
            cache[0, 0, page, :, first:first + m] = got[1][at + done:at + done + m].transpose(0, 1)
            cache[1, 0, page, :, first:first + m] = x[at + done:at + done + m, nq + nkv:].transpose(0, 1)
            done += m
        at += rows
    return {"q": got[0], "cache": cache}


def _attend_exact(s):
    c = s["case"]
    nq, nkv, d = c["nq"], c["nkv"], c["d"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    table, at = s["table"].tolist(), 0
    for (seq, ctx, _, rows), p in zip(s["spans"], s["parents"]):
        held = ctx + rows
        pages = table[seq][:-(-held // c["page"])]
        k, v = (torch.cat([s["cache"][i, 0, x] for x in pages], 1)[:, :held].double() for i in (0, 1))
        hidden = torch.ones(rows, held, dtype=torch.bool)
        hidden[:, :ctx] = False
        for i, b in enumerate(_branches(p) if c["width"] else [list(range(i + 1)) for i in range(rows)] if rows <= 128 else []):
            hidden[i, [ctx + x for x in b]] = False
        if rows > 128:
            hidden = torch.ones(rows, held, dtype=torch.bool).triu(ctx + 1)
        hidden = hidden.cuda()
        for h in range(nq):
            kv = h * nkv // nq
            x = (s["q"][at:at + rows, h].double() @ k[kv].t().contiguous()) / math.sqrt(d)
            out[at:at + rows, h] = torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ v[kv]
        at += rows
    return {"out": out}


def _keep_exact(s):
    c, table = s["case"], s["table"].tolist()
    cache = s["cache"].double()
    for (seq, ctx, _, _), b in zip(s["spans"], _kept(c)):
        place = lambda x: (table[seq][x // c["page"]], x % c["page"])  # noqa: E731
        rows = [cache[:, :, place(ctx + r)[0], :, place(ctx + r)[1]].clone() for r in b]
        for i, x in enumerate(rows):
            page, slot = place(ctx + 1 + i)
            cache[:, :, page, :, slot] = x
    return {"cache": cache}


def _verify_exact(s):
    c, at = s["case"], 0
    path = torch.full((c["n"], s["most"]), -1, dtype=torch.int32)
    accepted, after = [], []
    tokens, accept, sample = s["tokens"].tolist(), s["accept"].tolist(), s["sample"].tolist()
    for j, p in enumerate(s["parents"]):
        T, node, n = s["heat"][j], 0, 0
        while True:
            x = s["target"][at + node].double()
            now = torch.softmax(x / T, 0) if T > 0 else torch.nn.functional.one_hot(x.argmax(), len(x)).double()
            q = torch.softmax(s["draft"][at + node].double() / T, 0) if c["draft"] and T > 0 else None
            onto = None
            for child in [i for i in range(len(p)) if p[i] == node]:
                t = tokens[at + child]
                chance = now[t] if q is None else now[t] / q[t]
                if accept[at + child] < float(chance) if T > 0 else now[t] > 0:
                    onto = child
                    break
                if T > 0:                                     # what is left once this draft has failed
                    now = now.clone()
                    if q is None:
                        now[t] = 0.0
                    else:
                        now = (now - q).clamp_(min=0.0)
                    now = now / now.sum()
            if onto is None:
                break
            path[j, n] = node = onto
            n += 1
        if T > 0:
            sums = now.cumsum(0)
            after.append(int((sums > sample[j] * sums[-1]).to(torch.int8).argmax()))
        else:
            after.append(int(now.argmax()))
        accepted.append(n)
        at += len(p)
    return {"path": path.cuda(), "accepted": torch.tensor(accepted, dtype=torch.int32).cuda(), "next": torch.tensor(after, dtype=torch.int32).cuda()}
