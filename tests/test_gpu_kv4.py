"""The 4-bit key/value cache on the GPU against its definition in 64 bits (kv4_ref).

Tolerances.  bf16 has eight bits: rounding to it is off by up to 2^-8 of a number.  attend: every weight is rounded to bf16 and so is the output, which
makes 2^-8 sum p |v| + 2^-8 |out|; fp32 arithmetic adds what the scores are off, their 128 products summed in fp32 and scaled, at most
about 2^-17 of a weight for scores up to 40; bound 2^-15 sum p |v|.  weights: the same 2^-17 and the sum's roundings; bound 2^-15 of the value.  append: exact
where nothing is rounded before the codes; with norms and rotation (a dozen fp32 roundings) a query lies between the bf16 numbers
nearest to the 64-bit value -+ 2^-19 of its head's largest, and a code may only differ where the 64-bit value is within that of a boundary."""
import math

import numpy as np
import pytest
import torch

from paper_2504_12329_amd import binding as B

from . import kv4_ref as R

pytestmark = pytest.mark.gpu
WEIGHT_TOL = 2.0 ** -15


def out_tol(want, size):
    return (2.0 ** -8 + 2.0 ** -15) * size + 2.0 ** -8 * np.abs(want)


def make(nq, nkv, d, n_seq=3, max_seq=64, max_rows=256, max_pos=8192, n_layers=1, fill=None, stream=None, eps=1e-6):
    cfg = dict(n_layers=n_layers, n_seq=n_seq, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, max_seq=max_seq, max_rows=max_rows,
               max_pos=max_pos, rms_eps=eps)
    kv = B.Kv4Cache(cfg, B.rope_table(max_pos, d, 1e6), stream=stream)
    if fill is not None:
        kv.cache.fill_(fill)
        kv._ws.fill_(fill)
    return kv


def planes(kv):
    """K codes, V codes, K scales, V scales as views of the cache."""
    c, at, got = kv.cfg, 0, []
    for per in (c["head_dim"] // 2, c["head_dim"] // 2, c["head_dim"] // 32, c["head_dim"] // 32):
        shape = (c["n_layers"], c["n_seq"], c["n_kv_heads"], c["max_seq"], per)
        got.append(kv.cache[at:at + math.prod(shape)].view(shape))
        at += -(-math.prod(shape) // 256) * 256
    return got


def put(kv, layer, seq, n, rng, gain=1.0):
    """Random codes in slots [0, n) of a sequence; returns (k, v) float64 [nkv][n][d]."""
    c, pl, got = kv.cfg, planes(kv), []
    for p in (0, 1):
        codes = rng.integers(0, 16, (c["n_kv_heads"], n, c["head_dim"])).astype(np.uint8)
        scales = (126 + rng.integers(-2, 1, (c["n_kv_heads"], n, c["head_dim"] // 32)) + int(math.log2(gain))).astype(np.uint8)
        pl[p][layer, seq, :, :n] = torch.from_numpy(R.pack(codes)).cuda()
        pl[2 + p][layer, seq, :, :n] = torch.from_numpy(scales).cuda()
        got.append(R.values(codes, scales))
    return got


def bf16(x):
    return torch.from_numpy(np.asarray(x)).to(torch.bfloat16).cuda()


def f64(t):
    return t.to(torch.float64).cpu().numpy()


def ledger_for(kv, rng):
    c = kv.cfg
    shape = (c["n_layers"], c["n_seq"], c["n_kv_heads"], c["max_seq"])
    return B.Kv4Ledger(torch.from_numpy(rng.random(shape).astype(np.float32)).cuda(), torch.zeros(shape, dtype=torch.int32, device="cuda"))


def check_attend(kv, layer, spans, rng, with_ledger=True, scale=0.3, q_pad=0):
    c = kv.cfg
    nq, d, rows = c["n_q_heads"], c["head_dim"], sum(s[3] for s in spans)
    kvs = [put(kv, layer, seq, n + r, rng) for seq, n, _, r in spans]
    wide = bf16(rng.standard_normal((rows, nq * d + q_pad)) * scale)
    q = wide[:, :nq * d]
    led = ledger_for(kv, rng) if with_ledger else None
    before = f64(led.weights) if led else None
    out = torch.full((rows, nq * d + 8 * bool(q_pad)), 7.0, dtype=torch.bfloat16, device="cuda")
    view = out[:, :nq * d]
    kv.attend(layer, B.Kv4Spans(spans), q, led, out=view)
    assert (out[:, nq * d:] == 7).all()
    got, at = f64(view).reshape(rows, nq, d), 0
    want_w = None if before is None else before.copy()
    for (seq, n, _, r), (k, v) in zip(spans, kvs):
        if r == 0:
            continue
        want, size, w = R.attention(f64(q[at:at + r]).reshape(r, nq, d), k, v, n)
        err = np.abs(got[at:at + r] - want) / out_tol(want, size).clip(1e-30)
        assert err.max() <= 1, (spans, seq, err.max(), np.unravel_index(err.argmax(), err.shape))
        if want_w is not None:
            want_w[layer, seq, :, :n + r] += w
        at += r
    if want_w is not None:
        err = np.abs(f64(led.weights) - want_w) / want_w.clip(1e-30)
        assert err.max() <= WEIGHT_TOL, (spans, err.max())


# ---- append and read ----

@pytest.mark.parametrize("d", [64, 128])
def test_values_of_every_bf16_number(d):
    """All finite bf16 numbers as values (nothing is computed before the codes): groups in which each is the largest, and mixed ones."""
    print("append: every bf16 number, head_dim", d, flush=True)
    every = np.arange(65536, dtype=np.uint32)
    every = every[(every & 0x7f80) != 0x7f80]
    x = (every << 16).astype(np.uint32).view(np.float32).astype(np.float64)
    rng = np.random.default_rng(1)
    # smaller companions of the same group spread below its size
    alone = x[:, None] * np.concatenate([[1.0], rng.choice([0, -1, 0.5, 1 / 7, 2.5 / 7, 5 / 7, 3.5 / 6, 1 / 24, 1e-3], 31)])
    mixed = rng.permutation(np.concatenate([x, x[:-len(x) % 32]])).reshape(-1, 32)
    groups = torch.from_numpy(np.concatenate([alone, mixed])).to(torch.float32).to(torch.bfloat16)
    groups = torch.where(groups.isinf(), torch.zeros_like(groups), groups)
    groups = torch.cat([groups, torch.zeros(-len(groups) % (2 * d // 32), 32, dtype=torch.bfloat16)])
    v = groups.reshape(-1, 2, d)
    rows = v.shape[0]
    kv = make(2, 2, d, n_seq=1, max_seq=rows, max_rows=rows, max_pos=rows)
    qkv = torch.zeros(rows, 6, d, dtype=torch.bfloat16)
    qkv[:, 4:] = v
    kv.append(0, B.Kv4Spans([(0, 0, 0, rows)]), qkv.view(rows, 6 * d).cuda())
    _, got = kv.read(0, 1, B.Kv4Spans([(0, 0, 0, rows)]))
    # the reference, vectorised over groups
    g = f64(v).reshape(-1, 32)
    top = np.abs(g).max(1)
    m, e = np.frexp(top)
    s = np.where(top > 0, np.clip(np.where(m > 0.875, e - 2, e - 3), -100, 125), -100)
    a = np.abs(g) / 2.0 ** s[:, None]
    code = np.zeros(g.shape, dtype=np.int64)
    for c in range(1, 8):
        middle = (R.LEVELS[c - 1] + R.LEVELS[c]) / 2
        code[(a > middle) | ((a == middle) & (c % 2 == 0))] = c
    want = np.sign(g) * R.LEVELS[code] * 2.0 ** s[:, None]
    got = f64(got[0]).reshape(-1, 32)
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]
    some = rng.integers(0, len(g), 50)
    for i in some:                                        # the vectorised reference is the plain one
        c, b = R.quantise_group(g[i])
        assert b == s[i] + 127 and np.array_equal(c & 7, code[i])


def test_groups_that_hold_no_numbers():
    print("append: inf and NaN", flush=True)
    kv = make(2, 2, 128, max_seq=8, fill=0x5a)
    qkv = torch.ones(3, 6, 128, dtype=torch.bfloat16)
    qkv[0, 2, 5], qkv[1, 5, 40], qkv[1, 4, 127], qkv[2, 4, 64] = math.nan, math.inf, -math.inf, math.nan
    kv.append(0, B.Kv4Spans([(1, 2, 0, 3)]), qkv.view(3, -1).cuda())
    k, v = kv.read(0, 1, B.Kv4Spans([(1, 2, 0, 3)]))
    nan_k, nan_v = k[0].isnan().cpu(), v[0].isnan().cpu()
    want_k, want_v = torch.zeros(3, 2, 128, dtype=torch.bool), torch.zeros(3, 2, 128, dtype=torch.bool)
    want_k[0, 0, :32] = want_k[0, 0, 64:96] = True       # the rotation pairs channel 5 with channel 69
    want_v[1, 1, 32:64] = want_v[1, 0, 96:] = want_v[2, 0, 64:96] = True
    assert torch.equal(nan_k, want_k) and torch.equal(nan_v, want_v)
    assert (v[0].cpu()[~want_v] == 1).all()


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (12, 2, 128), (5, 5, 128), (40, 8, 128), (16, 1, 64)])
@pytest.mark.parametrize("norm", [False, True])
def test_append(nq, nkv, d, norm):
    print("append", nq, nkv, d, norm, flush=True)
    rng = np.random.default_rng(nq * 10 + nkv + norm)
    spans = [(2, 5, 4000, 3), (0, 0, 0, 0), (1, 0, 7, 1), (3, 13, 8191 - 5, 5)]
    rows = 9
    kv = make(nq, nkv, d, n_seq=4, max_seq=18, n_layers=2, fill=0x5a)
    led = ledger_for(kv, rng)
    w0 = led.weights.clone()
    width = (nq + 2 * nkv) * d
    wide = bf16(rng.standard_normal((rows, width + 24)) * 3)
    qn, kn = (bf16(1 + 0.3 * rng.standard_normal(d)) for _ in range(2)) if norm else (None, None)
    cache0 = kv.cache.clone()
    q = kv.append(1, B.Kv4Spans(spans), wide[:, :width], qn, kn, led)
    x = f64(wide[:, :width]).reshape(rows, nq + 2 * nkv, d)
    pos = np.concatenate([np.arange(p, p + r) for _, _, p, r in spans])
    angle = pos[:, None] * 1e6 ** (-2 * np.arange(d // 2) / d)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]

    def turned(y, w):
        if w is not None:
            y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + 1e-6) * f64(w)
        a, b = y[..., :d // 2], y[..., d // 2:]
        return np.concatenate([a * c - b * s, b * c + a * s], -1)

    want_q, want_k, want_v = turned(x[:, :nq], qn), turned(x[:, nq:nq + nkv], kn), x[:, nq + nkv:]
    size = np.abs(want_q).max(-1, keepdims=True)
    low, high = (f64(bf16(want_q + sign * 2.0 ** -19 * size)) for sign in (-1, 1))
    assert ((low <= f64(q)) & (f64(q) <= high)).all()
    pl, at = planes(kv), 0
    untouched = [torch.ones_like(p, dtype=torch.bool) for p in pl]
    for seq, n, p, r in spans:
        for side, want in ((0, want_k), (1, want_v)):
            codes = pl[side][1, seq, :, n:n + r].cpu().numpy()
            scales = pl[2 + side][1, seq, :, n:n + r].cpu().numpy()
            untouched[side][1, seq, :, n:n + r] = False
            untouched[2 + side][1, seq, :, n:n + r] = False
            if not r:
                continue
            codes = np.stack((codes & 15, codes >> 4), -1).reshape(nkv, r, d)
            got = R.values(codes, scales)
            ref = np.moveaxis(want[at:at + r], 1, 0)
            rc, rs = R.quantise(ref)
            same = got == R.values(rc, rs)
            if side == 1:
                assert same.all()
                continue
            # a key's code may differ only next to a boundary: within 2^-19 of the group's largest
            unit = 2.0 ** (scales.astype(float) - 127).repeat(32, -1).reshape(got.shape)
            a = np.abs(ref) / unit
            near = np.min([np.abs(a - m) for m in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5)], 0) <= 7 * 2.0 ** -19
            top = np.abs(ref).reshape(nkv, r, -1, 32).max(-1)
            edge = np.abs(top / 2.0 ** np.round(np.log2(top / 7)) / 7 - 1) < 2.0 ** -18
            assert (same | near | edge.repeat(32, -1).reshape(same.shape)).all()
            assert same.mean() > 0.999
        w, ps = led.weights[1, seq, :, n:n + r], led.positions[1, seq, :, n:n + r].cpu().numpy()
        assert (w == 0).all() and (ps == np.arange(p, p + r)).all()
        w0[1, seq, :, n:n + r] = 0
        at += r
    assert torch.equal(led.weights, w0)
    for p, p0, u in zip(pl, planes_of(kv, cache0), untouched):      # nothing else was written
        assert torch.equal(p[u], p0[u])


def planes_of(kv, cache):
    was, kv.cache = kv.cache, cache
    got = planes(kv)
    kv.cache = was
    return got


def test_the_codes_do_not_depend_on_how_rows_are_dealt():
    print("append: one call, three calls", flush=True)
    rng = np.random.default_rng(5)
    one, three = make(4, 2, 128, max_seq=40), make(4, 2, 128, max_seq=40)
    x = bf16(rng.standard_normal((33, 8 * 128)))
    n = bf16(1 + 0.1 * rng.standard_normal(128))
    q = one.append(0, B.Kv4Spans([(0, 0, 100, 33)]), x, n, n)
    parts = [three.append(0, B.Kv4Spans([(0, a, 100 + a, b - a)]), x[a:b], n, n) for a, b in ((0, 1), (1, 32), (32, 33))]
    assert torch.equal(q, torch.cat(parts))
    for a, b in zip(planes(one), planes(three)):
        assert torch.equal(a[0, 0, :, :33], b[0, 0, :, :33])


@pytest.mark.parametrize("nkv,d,rows", [(1, 64, 4100), (1, 128, 77), (2, 128, 2050), (3, 128, 1501), (8, 128, 1025), (5, 64, 33)])
def test_read(nkv, d, rows):
    """Rows that fill the chip (two a wave) and rows that do not, an odd number of them, in spans that do not start with the sequence."""
    print("read", nkv, d, rows, flush=True)
    rng = np.random.default_rng(rows)
    kv = make(nkv, nkv, d, n_seq=5, max_seq=rows + 9, n_layers=4)
    held = {(layer, seq): put(kv, layer, seq, rows + 9, rng) for layer in (1, 2, 3) for seq in (0, 3, 4)}
    spans = [(3, 9, 0, rows), (1, 5, 0, 0), (0, 0, 0, 1), (4, 7, 0, rows - rows % 2)]
    got = kv.read(1, 4, B.Kv4Spans(spans))
    for layer in (1, 2, 3):
        for side in (0, 1):
            want = np.concatenate([held[layer, seq][side][:, n:n + r] for seq, n, _, r in spans if r], 1).transpose(1, 0, 2)
            assert np.array_equal(f64(got[side][layer - 1]), want)


# ---- attend ----

@pytest.mark.parametrize("nq,nkv,d", [(1, 1, 128), (4, 2, 64), (10, 2, 128), (7, 1, 128), (16, 1, 64), (32, 2, 128)])
@pytest.mark.parametrize("spans", [
    [(0, 0, 0, 1)],                                      # the first token of a sequence
    [(2, 31, 31, 1)], [(2, 32, 32, 1)], [(1, 126, 9, 2)],  # ends of tiles
    [(1, 300, 300, 1), (0, 0, 5, 1), (2, 129, 129, 1)],  # ragged single tokens
    [(0, 7, 0, 3), (2, 500, 0, 0), (1, 61, 0, 2)],       # one without rows
    [(0, 0, 0, 9)], [(1, 119, 0, 9)], [(1, 121, 0, 40)], [(0, 0, 0, 33), (2, 255, 0, 65)],
])
def test_attend(nq, nkv, d, spans):
    print("attend", nq, nkv, d, spans, flush=True)
    rng = np.random.default_rng(len(spans) * 100 + nq)
    kv = make(nq, nkv, d, max_seq=523, n_layers=2, fill=0xff)      # slots that hold nothing read as NaN
    check_attend(kv, 1, spans, rng)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 6, 7, 12, 13, 26])
def test_attend_every_form(rows):
    """Across the switches between column tiles (16, 32, 64 columns) and to the chunk kernel, with and without weights, strided."""
    print("attend: 5 heads a kv head, rows", rows, flush=True)
    rng = np.random.default_rng(rows)
    kv = make(10, 2, 128, max_seq=1000)
    for with_ledger in (False, True):
        check_attend(kv, 0, [(1, 700 + rows, 0, rows)], rng, with_ledger, q_pad=40)


@pytest.mark.parametrize("d", [64, 128])
def test_attend_long_and_peaked(d):
    """A few thousand slots in many key ranges, and scores that leave one slot almost all the weight."""
    print("attend: long", d, flush=True)
    rng = np.random.default_rng(d)
    kv = make(4, 2, d, n_seq=2, max_seq=4500)
    for scale in (0.05, 2.0):
        check_attend(kv, 0, [(0, 4321, 0, 1)], rng, scale=scale)
        check_attend(kv, 0, [(1, 2111, 0, 41), (0, 77, 0, 3)], rng, scale=scale)


@pytest.mark.parametrize("nq,nkv,d", [(12, 2, 128), (4, 2, 64), (5, 5, 128)])
@pytest.mark.parametrize("rows", [1, 9])
def test_attend_where_ranges_begin(nq, nkv, d, rows):
    """Contexts that stay in one range without a ledger, and the first that do not; with a ledger they are cut, and joined beside the weights."""
    print("attend: one range or several", nq, nkv, d, rows, flush=True)
    rng = np.random.default_rng(nq + rows)
    kv = make(nq, nkv, d, n_seq=2, max_seq=640, fill=0xff)
    for held, ranges in ((rows, 1), (128, 1), (129, 1), (511, 1), (512, 1), (513, 5), (620, 5)):
        spans = [(1, held - rows, 0, rows), (0, 2, 0, rows)]
        assert kv.attend_plan(B.Kv4Spans(spans))[2][0] == ranges
        for with_ledger in (False, True):
            check_attend(kv, 0, spans, rng, with_ledger)


def test_attend_many_spans():
    print("attend: 64 spans", flush=True)
    rng = np.random.default_rng(9)
    kv = make(2, 2, 64, n_seq=70, max_seq=200)
    check_attend(kv, 0, [(69 - j, (j * 37) % 190, 0, 1 + j % 3) for j in range(64)], rng)


@pytest.mark.parametrize("n", [40, 64])
def test_attend_weights_with_and_without_room_for_scores(n):
    """Single tokens with a ledger, one of them on a long context: the scores of 40 x 40 heads x 3328 slots have room in the workspace (2^23 floats at
    most), those of 64 x 40 x 3328 do not."""
    print("attend: weights of", n, "spans", flush=True)
    rng = np.random.default_rng(n)
    kv = make(40, 8, 64, n_seq=64, max_seq=3300, max_rows=64, max_pos=64, fill=0xff)
    check_attend(kv, 0, [(5, 3299, 0, 1)] + [((6 + j) % 64, 7 * j % 130, 0, 1) for j in range(n - 1)], rng)


@pytest.mark.parametrize("rows", [1, 3, 50])
@pytest.mark.parametrize("side", ["k", "v"])
def test_a_group_without_numbers_reaches_the_rows_that_see_it_and_no_others(rows, side):
    print("attend: NaN in", side, rows, flush=True)
    rng = np.random.default_rng(rows)
    kv = make(4, 2, 128, max_seq=400)
    n = 210
    k, v = put(kv, 0, 0, n + rows, rng)
    pl = planes(kv)
    plane, ref = (pl[2], k) if side == "k" else (pl[3], v)
    codes = pl[0 if side == "k" else 1]
    q = bf16(rng.standard_normal((rows, 4, 128)) * 0.3)
    # an early slot (head 0, group 1: every row sees it); the chunk's own last slot (head 1, group 3: only the last row does)
    for head, slot, group in ((0, 17, 1), (1, n + rows - 1, 3)):
        plane[0, 0, head, slot, group] = 255
        codes[0, 0, head, slot, 16 * group:16 * group + 16] = 0
        ref[head, slot, 32 * group:32 * group + 32] = math.nan
    led = ledger_for(kv, rng)
    w0 = f64(led.weights)
    out = f64(kv.attend(0, B.Kv4Spans([(0, n, 0, rows)]), q, led))
    want, size, w = R.attention(f64(q), k, v, n)
    assert np.array_equal(np.isnan(out), np.isnan(want))
    fine = ~np.isnan(want)
    assert (np.abs(out - want)[fine] <= out_tol(want, size)[fine]).all()
    w0[0, 0, :, :n + rows] += w
    got = f64(led.weights)
    assert np.array_equal(np.isnan(got), np.isnan(w0))
    fine = ~np.isnan(w0)
    assert (np.abs(got - w0)[fine] <= WEIGHT_TOL * w0[fine]).all()


def test_a_query_without_numbers_stays_in_its_row_and_head():
    print("attend: NaN in q", flush=True)
    rng = np.random.default_rng(3)
    kv = make(4, 2, 128, max_seq=400)
    for rows in (2, 40):
        put(kv, 0, 0, 100 + rows, rng)
        q = bf16(rng.standard_normal((rows, 4, 128)) * 0.3)
        good = kv.attend(0, B.Kv4Spans([(0, 100, 0, rows)]), q)
        q[1, 2, 77] = math.nan
        bad = kv.attend(0, B.Kv4Spans([(0, 100, 0, rows)]), q)
        assert bad[1, 2].isnan().all()
        good[1, 2] = bad[1, 2] = 0
        assert torch.equal(good, bad)


@pytest.mark.parametrize("d,rows,context", [(64, 2, 40), (128, 2, 700), (128, 3, 513), (64, 4, 0), (128, 7, 60), (64, 7, 900), (128, 14, 300),
                                            (128, 30, 33), (64, 40, 500)])
@pytest.mark.parametrize("odd", [math.nan, math.inf])
def test_a_query_without_numbers_leaves_weights_of_slots_that_its_row_does_not_see(d, rows, context, odd):
    """In the first row and in one within: the weights of the slots that those rows see are no numbers, those of later rows' slots and of the other kv head are.
    Rows of two heads a kv head, in every form that sums up weights: from stored scores (up to 8 columns), beside the join, by columns in blocks."""
    print("attend: a query without numbers, weights", d, rows, context, odd, flush=True)
    rng = np.random.default_rng(rows + context)
    kv = make(4, 2, d, max_seq=context + rows + 3, fill=0xff)
    for bad in sorted({0, rows // 2}):
        k, v = put(kv, 0, 1, context + rows, rng)
        q = bf16(rng.standard_normal((rows, 4, d)) * 0.3)
        q[bad, 1, d - 3] = odd
        led = ledger_for(kv, rng)
        w0 = f64(led.weights)
        kv.attend(0, B.Kv4Spans([(1, context, 0, rows)]), q, led)
        q[bad, 1, d - 3] = math.nan                      # (an infinity times any key is none either: all of the row's scores are without numbers)
        w0[0, 1, :, :context + rows] += R.attention(f64(q), k, v, context)[2]
        got = f64(led.weights)
        assert np.isnan(w0).sum() == context + bad + 1
        assert np.array_equal(np.isnan(got), np.isnan(w0)), np.argwhere(np.isnan(got) != np.isnan(w0))[:5]
        fine = ~np.isnan(w0)
        assert (np.abs(got - w0)[fine] <= WEIGHT_TOL * w0[fine]).all()


def test_offsets_past_32_bits():
    """Planes of more than 4 GB: the last sequence of 40, its context at the end of its slots."""
    print("planes of 5 GB", flush=True)
    rng = np.random.default_rng(4)
    cap = 1 << 18
    kv = make(4, 8 // 2, 128, n_seq=80, max_seq=cap, max_rows=64, max_pos=cap)
    n = cap - 3
    pl = planes(kv)
    assert pl[0].numel() > 1 << 32
    for p in pl:                                         # all but the last slots: a neutral filling
        p[0, 79] = 0 if p.shape[-1] > 8 else 127
    x = bf16(rng.standard_normal((3, 12 * 128)))
    spans = B.Kv4Spans([(79, n, n, 3)])
    q = kv.append(0, spans, x)
    k, v = kv.read(0, 1, spans)
    codes, scales = R.quantise(f64(x).reshape(3, 12, 128)[:, 8:])
    assert np.array_equal(f64(v[0]), R.values(codes, scales))
    # keys of zeros score 0: slots before the chunk share one weight and have the value 0
    out, qq, kk, vv = f64(kv.attend(0, spans, q)), f64(q), f64(k[0]), f64(v[0])
    for i in range(3):
        for h in range(4):
            s = np.concatenate([[0.0], kk[:i + 1, h] @ qq[i, h] / math.sqrt(128)])
            e = np.exp(s - s.max()) * np.array([n] + [1] * (i + 1))
            want, size = e[1:] @ vv[:i + 1, h] / e.sum(), e[1:] @ np.abs(vv[:i + 1, h]) / e.sum()
            assert (np.abs(out[i, h] - want) <= out_tol(want, size) + 1e-12).all()


# ---- evict ----

def check_evict(kv, layers, spans, keep, recent, weights, positions, into):
    c = kv.cfg
    led = B.Kv4Ledger(torch.from_numpy(weights.copy()).cuda(), torch.from_numpy(positions.copy()).cuda())
    to = B.Kv4Ledger(torch.full_like(led.weights, -7.0), torch.full_like(led.positions, -7)) if into else led
    before = [p.cpu().numpy().copy() for p in planes(kv)]
    kv.evict(*layers, B.Kv4Spans(spans), keep, recent, led, to if into else None)
    after = [p.cpu().numpy() for p in planes(kv)]
    got_w, got_p = to.weights.cpu().numpy(), to.positions.cpu().numpy()
    want_w, want_p = (np.full_like(weights, -7), np.full_like(positions, -7)) if into else (weights.copy(), positions.copy())
    want = [b.copy() for b in before]
    for layer in range(*layers):
        for seq, n, pos, _ in spans:
            for h in range(c["n_kv_heads"]):
                src = R.evict(weights[layer, seq, h, :n], positions[layer, seq, h, :n], pos, keep, recent)
                m = len(src)
                want_w[layer, seq, h, :m], want_p[layer, seq, h, :m] = weights[layer, seq, h, src], positions[layer, seq, h, src]
                for w, b in zip(want, before):
                    w[layer, seq, h, :m] = b[layer, seq, h, src]
    assert np.array_equal(got_w, want_w, equal_nan=True)
    assert np.array_equal(got_p, want_p)
    for a, w in zip(after, want):
        assert np.array_equal(a, w)
    if into:
        assert np.array_equal(led.weights.cpu().numpy(), weights, equal_nan=True) and np.array_equal(led.positions.cpu().numpy(), positions)


def random_ledger(kv, spans, rng, kind):
    c = kv.cfg
    shape = (c["n_layers"], c["n_seq"], c["n_kv_heads"], c["max_seq"])
    w = np.exp(3 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "ties":
        w = rng.integers(0, 3, shape).astype(np.float32)
    if kind == "odd":                                    # every sort of number
        odd = np.array([0.0, -0.0, -1.5, math.inf, -math.inf, math.nan, 1e-45, 3.4e38, -1e-45, 1.0], dtype=np.float32)
        w = rng.choice(odd, shape)
    if kind == "equal":
        w[:] = 0.25
    p = np.zeros(shape, dtype=np.int32)
    for seq, n, pos, _ in spans:
        for layer in range(c["n_layers"]):
            for h in range(c["n_kv_heads"]):
                p[layer, seq, h, :n] = rng.permutation(max(n, pos))[:n] if pos >= n else rng.permutation(n)
    return w, p


@pytest.mark.parametrize("kind", ["spread", "ties", "odd", "equal"])
@pytest.mark.parametrize("d", [64, 128])
def test_evict(d, kind):
    print("evict", d, kind, flush=True)
    rng = np.random.default_rng(d)
    kv = make(4, 2, d, n_seq=4, max_seq=1100, n_layers=3)
    kv.cache.copy_(torch.from_numpy(rng.integers(0, 256, kv.cache.numel()).astype(np.uint8)))
    for spans, keep, recent in (([(1, 2, 2, 0)], 1, 0), ([(1, 2, 2, 0)], 1, 1), ([(0, 65, 65, 0), (2, 64, 90, 0), (3, 0, 0, 0)], 64, 13),
                                ([(3, 1099, 2000, 0), (0, 130, 130, 0), (2, 300, 300, 0)], 129, 64), ([(2, 1100, 1100, 0)], 1099, 1099),
                                ([(1, 1024, 1024, 0)], 3, 2), ([(0, 40, 40, 0)], 64, 64)):
        w, p = random_ledger(kv, spans, rng, kind)
        check_evict(kv, (0, 3), spans, keep, recent, w, p, into=False)
        check_evict(kv, (1, 2), spans, keep, recent, w, p, into=True)


@pytest.mark.parametrize("layers,n_seq,spans,keep", [
    (9, 4, [(1, 1100, 1100, 0), (0, 900, 2000, 0), (3, 1001, 1001, 0), (2, 770, 770, 0)], 769),    # 288 heads
    (2, 1, [(0, 768, 768, 0)], 700), (2, 1, [(0, 769, 769, 0)], 700), (2, 1, [(0, 2049, 2049, 0)], 64),
])
def test_evict_by_blocks_of_either_size(layers, n_seq, spans, keep):
    print("evict:", layers, "layers", spans, flush=True)
    rng = np.random.default_rng(keep)
    kv = make(8, 8, 64, n_seq=n_seq, max_seq=2050 if n_seq == 1 else 1100, n_layers=layers)
    kv.cache.copy_(torch.from_numpy(rng.integers(0, 256, kv.cache.numel()).astype(np.uint8)))
    for kind in ("spread", "ties"):
        w, p = random_ledger(kv, spans, rng, kind)
        check_evict(kv, (0, layers), spans, keep, keep // 5, w, p, into=kind == "ties")


def test_evict_long():
    print("evict: 40000 slots", flush=True)
    rng = np.random.default_rng(8)
    kv = make(2, 1, 64, n_seq=2, max_seq=40001)
    kv.cache.copy_(torch.from_numpy(rng.integers(0, 256, kv.cache.numel()).astype(np.uint8)))
    spans = [(1, 40001, 50000, 0), (0, 5, 5, 0)]
    for kind, keep, recent in (("spread", 20000, 3000), ("ties", 39000, 0), ("spread", 700, 700)):
        w, p = random_ledger(kv, spans, rng, kind)
        check_evict(kv, (0, 1), spans, keep, recent, w, p, into=keep == 700)


@pytest.mark.parametrize("n,keep", [(9000, 4111), (30001, 12345), (7000, 5800)])
def test_evict_long_into_another_ledger(n, keep):
    """Many moves of few heads (their own launch, some of its blocks without any), the ledger's entries written elsewhere."""
    print("evict: into another ledger", n, keep, flush=True)
    rng = np.random.default_rng(n)
    kv = make(2, 2, 64, n_seq=2, max_seq=n, n_layers=2)
    kv.cache.copy_(torch.from_numpy(rng.integers(0, 256, kv.cache.numel()).astype(np.uint8)))
    spans = [(1, n, 2 * n, 0), (0, keep + 3, keep + 3, 0)]
    w, p = random_ledger(kv, spans, rng, "spread")
    check_evict(kv, (0, 2), spans, keep, 100, w, p, into=True)


def test_evict_with_positions_that_repeat():
    """A ledger that no append wrote: exactly `keep` slots stay all the same."""
    print("evict: repeated positions", flush=True)
    rng = np.random.default_rng(2)
    kv = make(2, 1, 64, n_seq=1, max_seq=3000)
    kv.cache.copy_(torch.from_numpy(rng.integers(0, 256, kv.cache.numel()).astype(np.uint8)))
    w = rng.integers(0, 2, (1, 1, 1, 3000)).astype(np.float32)
    for p in (np.zeros_like(w, dtype=np.int32), rng.integers(-5, 5, w.shape).astype(np.int32), np.full(w.shape, 2 ** 31 - 1, dtype=np.int32)):
        check_evict(kv, (0, 1), [(0, 2999, 100, 0)], 1500, 200, w, p, into=False)


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
@pytest.mark.parametrize("n,other,keep,recent", [(131900, 131050, 131000, 999), (131073, 131072, 130500, 0), (140003, 90000, 70001, 5000), (262145, 70, 1, 1)])
def test_evict_past_the_slots_whose_bits_fit_a_block(n, other, keep, recent, kind):
    """More than 131072 slots, whose bits are in the workspace, moved by the block that selects and by blocks of their own, beside a sequence with fewer."""
    print("evict:", n, "and", other, "slots,", kind, flush=True)
    rng = np.random.default_rng(n + keep)
    kv = make(2, 1, 64, n_seq=3, max_seq=n)
    kv.cache.copy_(torch.from_numpy(rng.integers(0, 256, kv.cache.numel()).astype(np.uint8)))
    spans = [(2, n, n + 100, 0), (0, other, other, 0)]
    w, p = random_ledger(kv, spans, rng, kind)
    check_evict(kv, (0, 1), spans, keep, recent, w, p, into=kind == "spread")


@pytest.mark.parametrize("n,keep", [(30001, 12000), (30001, 29500), (24577, 64), (140003, 139700)])
def test_evict_long_with_positions_that_repeat(n, keep):
    """Slots alike in weight and position where the weights are read again for every digit: the first of them stay."""
    print("evict: repeated positions", n, keep, flush=True)
    rng = np.random.default_rng(n + keep)
    kv = make(2, 1, 64, n_seq=1, max_seq=n)
    kv.cache.copy_(torch.from_numpy(rng.integers(0, 256, kv.cache.numel()).astype(np.uint8)))
    w = rng.integers(0, 2, (1, 1, 1, n)).astype(np.float32)
    for p in (np.zeros_like(w, dtype=np.int32), rng.integers(-5, 5, w.shape).astype(np.int32), np.full(w.shape, 2 ** 31 - 1, dtype=np.int32)):
        check_evict(kv, (0, 1), [(0, n, 100, 0)], keep, min(keep, 200), w, p, into=False)


# ---- together ----

def test_a_context_is_thinned_and_goes_on():
    """Append, attend with a ledger, evict, append and attend again: the second attention is that of the slots that stayed."""
    print("append, attend, evict, attend", flush=True)
    rng = np.random.default_rng(6)
    nq, nkv, d = 6, 2, 128
    kv = make(nq, nkv, d, n_seq=2, max_seq=300, fill=0xff)
    led = ledger_for(kv, rng)
    x = bf16(rng.standard_normal((257, (nq + 2 * nkv) * d)))
    first = B.Kv4Spans([(1, 0, 0, 256)])
    q = kv.append(0, first, x[:256], ledger=led)
    kv.attend(0, first, q, led)
    w, p = led.weights[0, 1, :, :256].cpu().numpy(), led.positions[0, 1, :, :256].cpu().numpy()
    k, v = (f64(t[0]).transpose(1, 0, 2) for t in kv.read(0, 1, first))
    kv.evict(0, 1, B.Kv4Spans([(1, 256, 256, 0)]), 100, 30, led)
    src = [R.evict(w[h], p[h], 256, 100, 30) for h in range(nkv)]
    new = B.Kv4Spans([(1, 100, 256, 1)])
    q = kv.append(0, new, x[256:], ledger=led)
    kn, vn = (f64(t[0]).transpose(1, 0, 2) for t in kv.read(0, 1, new))
    k2 = np.stack([np.concatenate([k[h][src[h]], kn[h]]) for h in range(nkv)])
    v2 = np.stack([np.concatenate([v[h][src[h]], vn[h]]) for h in range(nkv)])
    out = f64(kv.attend(0, new, q, led))
    want, size, got_w = R.attention(f64(q), k2, v2, 100)
    assert (np.abs(out - want) <= out_tol(want, size)).all()
    before = np.concatenate([np.stack([w[h][src[h]] for h in range(nkv)]), np.zeros((nkv, 1))], 1)
    got = f64(led.weights[0, 1, :, :101])
    assert (np.abs(got - before - got_w) <= WEIGHT_TOL * (before + got_w)).all()
    assert (led.positions[0, 1, :, 100] == 256).all()


def test_streams():
    """Another stream than the cache's is refused, unless the caller named the stream; a named one is the one that runs."""
    print("streams", flush=True)
    rng = np.random.default_rng(7)
    kv = make(4, 2, 64)
    put(kv, 0, 0, 21, rng)
    q = bf16(rng.standard_normal((1, 4 * 64)))
    spans = B.Kv4Spans([(0, 20, 0, 1)])
    want = kv.attend(0, spans, q)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side), pytest.raises(B.StError) as e:
        kv.attend(0, spans, q)
    assert e.value.code == B.ST_EINVAL
    torch.cuda.synchronize()
    other = B.Kv4Cache(kv.cfg, kv.rope, cache=kv.cache, stream=side.cuda_stream)
    got = other.attend(0, spans, q)
    side.synchronize()
    assert torch.equal(got, want)


def test_what_a_cache_allocates_stays_with_its_stream():
    """Freed while its calls may still run, the memory of a cache on a named stream is not handed to another stream."""
    print("memory and streams", flush=True)
    side = torch.cuda.Stream()
    probe = make(4, 2, 64, max_seq=5000)
    kv = B.Kv4Cache(probe.cfg, probe.rope, stream=side.cuda_stream)
    was = {kv.cache.data_ptr(), kv._ws.data_ptr()}
    sizes = kv.cache.numel(), kv._ws.numel()
    del kv
    assert not was & {torch.empty(n, dtype=torch.uint8, device="cuda").data_ptr() for n in sizes}
    with torch.cuda.stream(side):
        again = B.Kv4Cache(probe.cfg, probe.rope)
    assert again.cache.data_ptr() in was


def test_a_captured_step_replays():
    """Append, attend with weights and eviction in a HIP graph, replayed with new inputs between eager work."""
    print("graph", flush=True)
    rng = np.random.default_rng(11)
    nq, nkv, d = 4, 2, 128
    side = torch.cuda.Stream()
    x = bf16(rng.standard_normal((2, (nq + 2 * nkv) * d)))
    spans = B.Kv4Spans([(0, 200, 200, 1), (1, 64, 64, 1)])
    end = B.Kv4Spans([(0, 201, 201, 0), (1, 65, 65, 0)])
    with torch.cuda.stream(side):
        kv = make(nq, nkv, d, max_seq=300)
        put(kv, 0, 0, 200, rng), put(kv, 0, 1, 64, rng)
        led = ledger_for(kv, rng)
        led.positions[:] = torch.arange(300, device="cuda", dtype=torch.int32)

        def step():
            q = kv.append(0, spans, x, ledger=led)
            out = kv.attend(0, spans, q, led)
            kv.evict(0, 1, end, 150, 20, led)
            return out

        start = kv.cache.clone(), led.weights.clone(), led.positions.clone()

        def reset():
            kv.cache.copy_(start[0]), led.weights.copy_(start[1]), led.positions.copy_(start[2])

        step()
        reset()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            out = step()
        for _ in range(4):
            reset()
            x.copy_(bf16(rng.standard_normal(x.shape)))
            want = step().clone()
            state = kv.cache.clone(), led.weights.clone(), led.positions.clone()
            reset()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            assert all(torch.equal(a, b) for a, b in zip((kv.cache, led.weights, led.positions), state))


def test_matrices_side_by_side():
    """Queries and outputs as columns of one matrix, and appended rows beside the queries they become."""
    print("one matrix", flush=True)
    rng = np.random.default_rng(12)
    nq, nkv, d = 4, 2, 64
    kv = make(nq, nkv, d, fill=0xff)
    w = (nq + 2 * nkv) * d
    both = torch.zeros(5, w + 2 * nq * d, dtype=torch.bfloat16, device="cuda")
    both[:, :w] = bf16(rng.standard_normal((5, w)))
    spans = B.Kv4Spans([(0, 0, 0, 2), (2, 0, 5, 3)])
    q = kv.append(0, spans, both[:, :w])
    both[:, w:w + nq * d] = q.flatten(1)
    out = both[:, w + nq * d:]
    kv.attend(0, spans, both[:, w:w + nq * d], out=out)
    assert torch.equal(out, kv.attend(0, spans, q).flatten(1))
    for bad in (both[:, w:w + nq * d], both[:, w + 8:w + 8 + nq * d]):
        with pytest.raises(B.StError) as e:
            kv.attend(0, spans, both[:, w:w + nq * d], out=bad)
        assert e.value.code == B.ST_EINVAL


def test_refusals_of_the_binding():
    print("refusals", flush=True)
    kv = make(4, 2, 64)
    one = B.Kv4Spans([(0, 3, 0, 1)])
    good = torch.zeros(1, 4 * 64, dtype=torch.bfloat16, device="cuda")
    wrong = [good.float(), good.cpu(), good[:, :64], torch.zeros(2, 256, dtype=torch.bfloat16, device="cuda"),
             torch.zeros(256, 1, dtype=torch.bfloat16, device="cuda").t()[:, ::2]]
    for q in wrong:
        with pytest.raises(B.StError) as e:
            kv.attend(0, one, q)
        assert e.value.code == B.ST_EINVAL
    unaligned = torch.zeros(1 + 256, dtype=torch.bfloat16, device="cuda")[1:].view(1, 256)
    with pytest.raises(B.StError):
        kv.attend(0, one, unaligned)
    with pytest.raises(B.StError):
        kv.append(0, one, torch.zeros(1, 8 * 64, dtype=torch.bfloat16, device="cuda"), good[0, :64], None)
    with pytest.raises(B.StError):
        B.Kv4Ledger(torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda"))
    shape = (1, 3, 2, 63)
    with pytest.raises(B.StError):
        kv.attend(0, one, good, B.Kv4Ledger(torch.zeros(shape, device="cuda"), torch.zeros(shape, dtype=torch.int32, device="cuda")))
    with pytest.raises(B.StError):
        B.Kv4Cache(kv.cfg, kv.rope[:5])
    assert kv.attend(0, B.Kv4Spans([]), good[:0]).shape == (0, 4, 64)
    assert kv.read(0, 1, B.Kv4Spans([(0, 5, 0, 0)]))[0].shape == (1, 0, 2, 64)
