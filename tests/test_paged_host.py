"""Host-only checks of the calls of the paged cache and of the verdict over drafts: sizes, plans, and refusals before anything touches a device."""
import ctypes as C
import os

import pytest
import torch

from paper_2504_12329_amd import binding as B

CFG = dict(n_layers=3, n_seq=5, n_q_heads=12, n_kv_heads=2, head_dim=128, n_pages=50, page_size=32, max_pages=30, max_rows=64, max_pos=2000, dtype=B.ST_BF16,
           rot_dim=128, rot_pairs=B.ST_PAIRS_HALVES, rms_eps=1e-6)
PTR = 0x10000                                             # never followed: every call below is refused or has nothing to do


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        from paper_2504_12329_amd import build
        build.build()
    return B.lib()


def config(**over):
    c = dict(CFG, **over)
    return B.st_paged_config(*(c[n] for n, _ in B.st_paged_config._fields_))


def sizes(L, c):
    a, b = C.c_size_t(), C.c_size_t()
    return L.st_paged_query_sizes(C.byref(c), C.byref(a), C.byref(b)), a.value, b.value


@pytest.fixture
def kv(L):
    _, cb, wb = sizes(L, config())
    h = C.c_void_p()
    assert L.st_paged_create(C.byref(config()), PTR, PTR, PTR, cb, PTR, wb, None, C.byref(h)) == B.ST_OK
    yield h
    L.st_paged_destroy(h)


def spans(*s):
    return (B.st_kv4_span * max(len(s), 1))(*s), len(s)


def tree(parent=PTR, depth=PTR, sees=PTR, words=1, width=1):
    return C.byref(B.st_draft_tree(parent, depth, sees, words, width))


def test_sizes(L):
    rc, cb, wb = sizes(L, config())
    assert rc == B.ST_OK and cb == 2 * 2 * 3 * 50 * 2 * 32 * 128 and wb > 0
    assert C.sizeof(B.st_paged_config) == 56 and C.sizeof(B.st_draft_tree) == 32 and C.sizeof(B.st_verify_config) == 16
    assert L.st_paged_query_sizes(C.byref(config()), None, None) == B.ST_OK
    rc, cb, _ = sizes(L, config(n_layers=64, n_pages=1 << 20, n_kv_heads=8, n_q_heads=40))
    assert rc == B.ST_OK and cb == 4 * 64 * (1 << 20) * 8 * 32 * 128        # past 32 bits


@pytest.mark.parametrize("over", [dict(n_layers=0), dict(n_seq=-1), dict(n_q_heads=0), dict(n_kv_heads=0), dict(n_pages=0), dict(max_pages=0), dict(max_rows=0), dict(max_pos=0),
                                  dict(head_dim=96), dict(head_dim=256), dict(n_kv_heads=5), dict(n_q_heads=34, n_kv_heads=2), dict(rms_eps=-1.0), dict(rms_eps=float("nan")),
                                  dict(rms_eps=float("inf")), dict(page_size=8), dict(page_size=48), dict(page_size=2048), dict(page_size=0), dict(max_pages=(1 << 19) + 1),
                                  dict(max_rows=(1 << 20) + 1), dict(dtype=2), dict(dtype=-1), dict(rot_dim=8), dict(rot_dim=-16), dict(rot_dim=144), dict(rot_pairs=2),
                                  dict(n_layers=60000, n_pages=2 ** 31 - 1), dict(n_q_heads=4100, n_kv_heads=4100)])
def test_bad_configs(L, over):
    rc, _, _ = sizes(L, config(**over))
    assert rc == B.ST_EINVAL and L.st_last_error()


def test_create(L):
    _, cb, wb = sizes(L, config())
    h, c = C.c_void_p(7), C.byref(config())
    assert L.st_paged_create(c, PTR, PTR, PTR, cb, PTR, wb, None, None) == B.ST_EINVAL
    for rope, table, cache, ws in ((None, PTR, PTR, PTR), (PTR, None, PTR, PTR), (PTR, PTR, None, PTR), (PTR, PTR, PTR, None), (PTR, PTR, PTR + 16, PTR),
                                   (PTR, PTR, PTR, PTR + 128), (PTR + 8, PTR, PTR, PTR), (PTR, PTR + 2, PTR, PTR)):
        assert L.st_paged_create(c, rope, table, cache, cb, ws, wb, None, C.byref(h)) == B.ST_EINVAL and h.value is None
    assert L.st_paged_create(c, PTR, PTR, PTR, cb - 1, PTR, wb, None, C.byref(h)) == B.ST_ENOMEM
    assert L.st_paged_create(c, PTR, PTR, PTR, cb, PTR, wb - 1, None, C.byref(h)) == B.ST_ENOMEM
    assert L.st_paged_create(None, PTR, PTR, PTR, cb, PTR, wb, None, C.byref(h)) == B.ST_EINVAL
    assert L.st_paged_create(C.byref(config(rot_dim=0)), None, PTR, PTR, cb, PTR, wb, None, C.byref(h)) == B.ST_OK   # no table where nothing rotates
    L.st_paged_destroy(h)
    L.st_paged_destroy(None)


BAD_SPANS = [([(5, 0, 0, 1)], B.ST_ERANGE), ([(-1, 0, 0, 1)], B.ST_ERANGE), ([(0, -1, 0, 1)], B.ST_ERANGE), ([(0, 960, 0, 1)], B.ST_ERANGE),
             ([(0, 0, 0, -1)], B.ST_ERANGE), ([(0, 1, -1, 1)], B.ST_ERANGE), ([(0, 2 ** 31 - 1, 0, 2 ** 31 - 1)], B.ST_ERANGE),
             ([(1, 0, 0, 1), (0, 0, 0, 1), (1, 5, 0, 1)], B.ST_EINVAL), ([(0, 0, 0, 65)], B.ST_ERANGE),
             ([(0, 0, 0, 40), (1, 0, 0, 25)], B.ST_ERANGE)]


@pytest.mark.parametrize("bad,code", BAD_SPANS)
def test_bad_spans(L, kv, bad, code):
    s, n = spans(*bad)
    for t in (None, tree()):
        assert L.st_paged_append(kv, 0, s, n, t, PTR, 2048, None, None, 2 * PTR, 1536) == code
        assert L.st_paged_attend(kv, 0, s, n, t, PTR, 1536, 1 << 30, 1536) == code
    assert L.st_paged_keep(kv, 0, 1, s, n, PTR, 4, PTR) == code


def test_append_refusals(L, kv):
    s, n = spans((0, 3, 1999, 1))
    ok = dict(layer=0, s=s, n=n, tree=None, qkv=PTR, stride=2048, qn=None, kn=None, q=1 << 30, qs=1536)

    def call(**over):
        a = dict(ok, **over)
        return L.st_paged_append(kv, a["layer"], a["s"], a["n"], a["tree"], a["qkv"], a["stride"], a["qn"], a["kn"], a["q"], a["qs"])

    late, m = spans((0, 3, 2000, 1))                      # past the rotation table
    two, k = spans((0, 3, 1999, 2))
    assert call(s=late, n=m) == call(s=late, n=m, tree=tree()) == call(s=two, n=k) == B.ST_ERANGE
    assert call(layer=3) == call(layer=-1) == B.ST_ERANGE
    assert call(tree=tree(depth=None)) == call(tree=tree(depth=PTR + 2)) == B.ST_EINVAL
    assert call(qkv=None) == call(qkv=PTR + 2) == call(stride=2040) == call(stride=2049) == B.ST_EINVAL
    assert call(q=None) == call(q=PTR + 8) == call(qs=1528) == call(qs=1537) == call(q=PTR) == B.ST_EINVAL
    assert call(qn=PTR) == call(kn=PTR) == call(qn=PTR, kn=PTR + 4) == B.ST_EINVAL
    assert call(n=65) == call(n=-1) == call(s=None) == B.ST_EINVAL
    assert L.st_paged_append(None, 0, s, n, None, PTR, 2048, None, None, 1 << 30, 1536) == B.ST_EINVAL


def test_attend_refusals(L, kv):
    s, n = spans((0, 3, 0, 1))
    assert L.st_paged_attend(None, 0, s, n, None, PTR, 1536, 1 << 30, 1536) == B.ST_EINVAL
    assert L.st_paged_attend(kv, 3, s, n, None, PTR, 1536, 1 << 30, 1536) == B.ST_ERANGE
    for q, qs, o, os_ in ((None, 1536, 1 << 30, 1536), (PTR, 1536, None, 1536), (PTR + 4, 1536, 1 << 30, 1536), (PTR, 1530, 1 << 30, 1536), (PTR, 1536, 1 << 30, 1535),
                          (PTR, 1536, PTR + 2, 1536), (PTR, 1536, PTR, 1536), (PTR, 1536, PTR + 16, 1536)):
        assert L.st_paged_attend(kv, 0, s, n, None, q, qs, o, os_) == B.ST_EINVAL
    for t, code in ((tree(sees=None), B.ST_EINVAL), (tree(sees=PTR + 4), B.ST_EINVAL), (tree(words=0), B.ST_EINVAL), (tree(words=17), B.ST_EINVAL), (tree(words=-1), B.ST_EINVAL)):
        assert L.st_paged_attend(kv, 0, s, n, t, PTR, 1536, 1 << 30, 1536) == code


def test_more_rows_than_bits(L):
    c = config(max_rows=2000)
    _, cb, wb = sizes(L, c)
    h = C.c_void_p()
    assert L.st_paged_create(C.byref(c), PTR, PTR, PTR, cb, PTR, wb, None, C.byref(h)) == B.ST_OK
    s, n = spans((0, 3, 0, 5), (1, 3, 0, 65))
    assert L.st_paged_attend(h, 0, s, n, tree(words=1), PTR, 1536, 1 << 30, 1536) == B.ST_ERANGE and b"bits" in L.st_last_error()
    L.st_paged_destroy(h)


def test_keep_refusals(L, kv):
    s, n = spans((0, 3, 0, 4))
    call = lambda lo=0, hi=3, s=s, n=n, path=PTR, stride=4, acc=PTR: L.st_paged_keep(kv, lo, hi, s, n, path, stride, acc)  # noqa: E731
    assert call(lo=-1) == call(hi=4) == call(lo=2, hi=1) == B.ST_ERANGE
    assert call(path=None) == call(acc=None) == call(path=PTR + 2) == call(acc=PTR + 1) == call(stride=-1) == B.ST_EINVAL
    assert L.st_paged_keep(None, 0, 1, s, n, PTR, 4, PTR) == B.ST_EINVAL


def test_calls_with_nothing_to_do(L, kv):
    none, n = spans((0, 3, 0, 0), (2, 0, 0, 0))
    for t in (None, tree()):
        assert L.st_paged_append(kv, 0, none, n, t, PTR, 2048, None, None, PTR, 1536) == B.ST_OK
        assert L.st_paged_attend(kv, 0, none, n, t, PTR, 1536, PTR, 1536) == B.ST_OK
    assert L.st_paged_attend(kv, 0, None, 0, None, PTR, 1536, PTR, 1536) == B.ST_OK
    assert L.st_paged_keep(kv, 0, 3, none, n, PTR, 4, PTR) == L.st_paged_keep(kv, 0, 3, None, 0, PTR, 4, PTR) == B.ST_OK
    some, m = spans((0, 3, 0, 2))
    assert L.st_paged_keep(kv, 1, 1, some, m, PTR, 4, PTR) == L.st_paged_keep(kv, 0, 3, some, m, PTR, 0, PTR) == B.ST_OK


def plan(L, c, s, n, with_tree=0):
    columns, blocks, ranges = C.c_int32(-1), C.c_int32(-1), (C.c_int32 * 64)(*[-1] * 64)
    rc = L.st_paged_attend_plan(C.byref(c), s, n, with_tree, C.byref(columns), C.byref(blocks), ranges)
    return rc, columns.value, blocks.value, list(ranges)[:max(n, 0)]


def test_attend_plan(L):
    c = config(n_q_heads=40, n_kv_heads=8, n_seq=64, max_pages=1 << 19, max_rows=1 << 16)
    assert plan(L, c, None, 0) == (B.ST_OK, 0, 0, [])
    assert plan(L, c, *spans((3, 9, 0, 0))) == (B.ST_OK, 0, 0, [0])
    assert plan(L, c, *spans((0, 0, 0, 1)))[1:] == (16, 8, [1])
    rc, columns, blocks, ranges = plan(L, c, *spans((0, 1 << 19, 0, 1)))
    assert rc == B.ST_OK and columns == 16 and 60 <= ranges[0] <= 64 and blocks == 8 * ranges[0]
    assert plan(L, c, *spans((0, 100, 0, 5)))[1] == 32 and plan(L, c, *spans((0, 100, 0, 7)))[1] == 128
    # a long span beside many short ones is cut
    assert max(plan(L, c, *spans((0, 16000, 0, 1), *((j, 200, 0, 1) for j in range(1, 64))))[3]) > 10
    assert L.st_paged_attend_plan(C.byref(c), *spans((0, 5, 0, 1)), 0, None, None, None) == B.ST_OK
    assert plan(L, config(head_dim=96), *spans((0, 0, 0, 1)))[0] == B.ST_EINVAL
    assert plan(L, c, *spans((0, 5, 0, 1024)), 1)[0] == B.ST_OK and plan(L, c, *spans((0, 5, 0, 1025)), 1)[0] == B.ST_ERANGE and plan(L, c, *spans((0, 5, 0, 1025)))[0] == B.ST_OK
    for bad, code in BAD_SPANS:
        assert plan(L, config(), *spans(*bad))[0] == code


def test_ranges_stay_within_what_the_workspace_holds(L):
    """At most 64 ranges of a span, and partial results for every row and head of the spans that are cut: those of twice 512 blocks."""
    for nq, nkv in ((1, 1), (12, 2), (40, 8), (16, 1), (4096, 256)):
        for max_rows in (1, 7, 64, 5000):
            c = config(n_layers=1, n_q_heads=nq, n_kv_heads=nkv, n_seq=64, max_pages=1 << 17, max_rows=max_rows)
            held = min(max_rows * nq * 64, 2 * 512 * 128)
            for n in (1, 3, 64):
                for rows in (1, 2, max_rows // n):
                    for length in (0, 31, 513, 4097, 1 << 21):
                        if rows < 1 or rows * n > max_rows:
                            continue
                        s = spans(*((j, length if j % 2 == 0 else length // 3, 0, rows) for j in range(n)))
                        rc, columns, blocks, ranges = plan(L, c, *s, with_tree=rows % 2)
                        cut = [r for r in ranges if r > 1]
                        assert rc == B.ST_OK and min(ranges) >= 1 and max(ranges) <= 64
                        assert blocks == sum(r * nkv * -(-rows * (nq // nkv) // columns) for r in ranges)
                        assert sum(cut) * rows * nq <= held, (nq, nkv, max_rows, n, rows, length)


# ---- the verdict ----

def vconfig(vocab=1000, dtype=B.ST_F32, max_rows=100, max_width=4):
    return B.st_verify_config(vocab, dtype, max_rows, max_width)


@pytest.fixture
def verifier(L):
    n = C.c_size_t()
    assert L.st_verify_query_sizes(C.byref(vconfig()), C.byref(n)) == B.ST_OK and n.value > 0
    h = C.c_void_p()
    assert L.st_verify_create(C.byref(vconfig()), PTR, n.value, None, C.byref(h)) == B.ST_OK
    yield h
    L.st_verify_destroy(h)


@pytest.mark.parametrize("over", [dict(vocab=0), dict(vocab=-1), dict(vocab=(1 << 24) + 1), dict(dtype=3), dict(dtype=-1), dict(max_rows=0), dict(max_rows=32768), dict(max_width=0),
                                  dict(max_width=65)])
def test_bad_verify_configs(L, over):
    assert L.st_verify_query_sizes(C.byref(vconfig(**over)), None) == B.ST_EINVAL


def test_verify_create(L):
    n, h = C.c_size_t(), C.c_void_p(7)
    assert L.st_verify_query_sizes(C.byref(vconfig()), C.byref(n)) == B.ST_OK
    c = C.byref(vconfig())
    assert L.st_verify_create(c, PTR, n.value, None, None) == L.st_verify_create(None, PTR, n.value, None, C.byref(h)) == B.ST_EINVAL
    assert L.st_verify_create(c, None, n.value, None, C.byref(h)) == L.st_verify_create(c, PTR + 64, n.value, None, C.byref(h)) == B.ST_EINVAL
    assert L.st_verify_create(c, PTR, n.value - 1, None, C.byref(h)) == B.ST_ENOMEM and h.value is None
    L.st_verify_destroy(None)
    assert L.st_verify_query_sizes(C.byref(vconfig(vocab=1 << 24, max_rows=32767, max_width=64)), C.byref(n)) == B.ST_OK and n.value > 2 ** 32


def test_verify_refusals(L, verifier):
    def call(rows=(5, 3), n=2, tree=None, heat=(1.0, 0.0), stride=5, ts=1000, ds=1000, draft=PTR, h=verifier, **p):
        a = {k: p.get(k, PTR) for k in ("tokens", "target", "accept", "sample", "path", "accepted", "next")}
        r = None if rows is None else (C.c_int32 * max(len(rows), 1))(*rows)
        t = None if heat is None else (C.c_float * max(len(heat), 1))(*heat)
        return L.st_verify_drafts(h, r, n, tree, a["tokens"], a["target"], ts, draft, ds, t, a["accept"], a["sample"], a["path"], stride, a["accepted"], a["next"])

    assert call(n=0) == B.ST_OK and call(n=-1) == call(n=65) == call(h=None) == B.ST_EINVAL
    assert call(rows=None) == call(heat=None) == B.ST_EINVAL
    assert call(rows=(0, 3)) == call(rows=(5, -1)) == call(rows=(1025, 1), stride=2000) == call(rows=(60, 50), stride=60) == call(stride=4) == B.ST_ERANGE
    for bad in (-1.0, float("nan"), float("inf")):
        assert call(heat=(1.0, bad)) == B.ST_EINVAL
    for k in ("tokens", "target", "accept", "sample", "path", "accepted", "next"):
        assert call(**{k: None}) == call(**{k: PTR + 2}) == B.ST_EINVAL
    assert call(accept=PTR + 4) == call(sample=PTR + 4) == call(draft=PTR + 2) == B.ST_EINVAL
    assert call(ts=999) == call(ds=999) == B.ST_EINVAL
    assert call(tree=tree(parent=None)) == call(tree=tree(parent=PTR + 2)) == call(tree=tree(width=0)) == call(tree=tree(width=5)) == B.ST_EINVAL


# ---- the binding ----

def test_draft_spans():
    s = B.DraftSpans([(0, 9, 9, 4), (1, 0, 5, 1), (2, 7, 7, 3)], [[-1, 0, 0, 1], [None], [7, 0, 1]], device="cpu")
    assert s.parent.tolist() == [-1, 0, 0, 1, -1, -1, 0, 1] and s.depth.tolist() == [0, 1, 1, 2, 0, 0, 1, 2] and s.width == 2 and s.rows == 8
    assert s.sees.tolist() == [[1], [3], [5], [11], [1], [1], [3], [7]]
    chain = B.DraftSpans([(0, 0, 0, 130)], [list(range(-1, 129))], device="cpu")
    bits = [sum((w & (2 ** 64 - 1)) << (64 * i) for i, w in enumerate(row)) for row in chain.sees.tolist()]
    assert bits == [2 ** (i + 1) - 1 for i in range(130)] and chain.depth.tolist() == list(range(130)) and chain.width == 1
    assert B.DraftSpans([], [], device="cpu").rows == 0


def test_the_same_trees_at_other_places():
    s = B.DraftSpans([(0, 9, 9, 3), (1, 0, 5, 1)], [[-1, 0, 0], [-1]], device="cpu")
    t = s.at([(4, 20, 25, 3), (2, 7, 7, 1)])
    assert t.spans == [(4, 20, 25, 3), (2, 7, 7, 1)] and t.rows == 4 and t.width == 2 and t.parent is s.parent and t.sees is s.sees and t.depth is s.depth
    assert s.spans == [(0, 9, 9, 3), (1, 0, 5, 1)]
    for bad in ([(0, 9, 9, 3)], [(0, 9, 9, 1), (1, 0, 5, 3)]):
        with pytest.raises(B.StError) as e:
            s.at(bad)
        assert e.value.code == B.ST_EINVAL


@pytest.mark.parametrize("parents", [[[-1, 0]], [[-1, 0, 0], [-1]], [[-1, 0, 2]], [[-1, 0, -1]], [[-1, 1, 0]]])
def test_bad_parents(parents):
    with pytest.raises(B.StError) as e:
        B.DraftSpans([(0, 0, 0, 3)], parents, device="cpu")
    assert e.value.code == B.ST_EINVAL


def test_trees_that_are_too_large():
    for parents in ([[-1] + [0] * 65], [list(range(-1, 1024))]):
        with pytest.raises(B.StError) as e:
            B.DraftSpans([(0, 0, 0, len(parents[0]))], parents, device="cpu")
        assert e.value.code == B.ST_ERANGE


def test_objects_that_need_a_gpu_say_so():
    table, rope = torch.zeros(5, 30, dtype=torch.int32), torch.zeros(2000, 64, 2)
    cfg = {k: v for k, v in CFG.items() if k not in ("dtype", "rot_pairs")}
    for over in (dict(), dict(dtype=torch.float32), dict(rot_pairs="thirds"), dict(page_size=17)):
        with pytest.raises(B.StError) as e:
            B.PagedCache(dict(cfg, **over), rope, table)
        assert e.value.code == B.ST_EINVAL
    for name in ("n_layers", "n_pages", "page_size", "max_pages", "max_rows", "max_pos", "rot_dim"):
        with pytest.raises(B.StError) as e:
            B.PagedCache(dict(cfg, **{name: 2 ** 32 + 16}), rope, table)
        assert e.value.code == B.ST_ERANGE
    with pytest.raises(B.StError):
        B.DraftVerifier(1000, 10, device="cpu")
    with pytest.raises(B.StError):
        B.DraftVerifier(1000, 10, dtype=torch.float64)
    with pytest.raises(B.StError) as e:
        B.DraftVerifier(2 ** 32 + 5, 10)
    assert e.value.code == B.ST_ERANGE
    with pytest.raises(B.StError):
        B.DraftSpans.of_tensors([(0, 0, 0, 3)], parent=torch.zeros(3, dtype=torch.int32))
