"""Host-only checks of the 4-bit cache's calls: sizes, and refusals before anything touches a device."""
import ctypes as C
import os

import pytest

from paper_2504_12329_amd import binding as B

CFG = dict(n_layers=3, n_seq=5, n_q_heads=12, n_kv_heads=2, head_dim=128, max_seq=1000, max_rows=64, max_pos=2000, rms_eps=1e-6)
PTR = 0x10000                                             # never followed: every call below is refused or has nothing to do


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        from paper_2504_12329_amd import build
        build.build()
    return B.lib()


def config(**over):
    c = dict(CFG, **over)
    return B.st_kv4_config(*(c[n] for n, _ in B.st_kv4_config._fields_))


def sizes(L, c):
    a, b = C.c_size_t(), C.c_size_t()
    return L.st_kv4_query_sizes(C.byref(c), C.byref(a), C.byref(b)), a.value, b.value


@pytest.fixture
def kv(L):
    _, cb, wb = sizes(L, config())
    h = C.c_void_p()
    assert L.st_kv4_create(C.byref(config()), PTR, PTR, cb, PTR, wb, None, C.byref(h)) == B.ST_OK
    yield h
    L.st_kv4_destroy(h)


def test_sizes(L):
    rc, cb, wb = sizes(L, config())
    slots = 3 * 5 * 2 * 1000
    assert rc == B.ST_OK and cb == 2 * slots * 64 + 2 * (-(-slots * 4 // 256) * 256) and wb > 0
    assert C.sizeof(B.st_kv4_config) == 36 and C.sizeof(B.st_kv4_span) == 16 and C.sizeof(B.st_kv4_ledger) == 16
    assert L.st_kv4_query_sizes(C.byref(config()), None, None) == B.ST_OK
    rc, cb, _ = sizes(L, config(n_layers=64, n_seq=64, n_q_heads=40, n_kv_heads=8, max_seq=1 << 17))
    assert rc == B.ST_OK and cb == 64 * 64 * 8 * (1 << 17) * 136        # past 32 bits


@pytest.mark.parametrize("over", [dict(n_layers=0), dict(n_seq=-1), dict(n_q_heads=0), dict(n_kv_heads=0), dict(max_seq=0), dict(max_rows=0),
                                  dict(max_pos=0), dict(head_dim=96), dict(head_dim=256), dict(n_kv_heads=5), dict(n_q_heads=34, n_kv_heads=2),
                                  dict(rms_eps=-1.0), dict(rms_eps=float("nan")), dict(rms_eps=float("inf")), dict(max_seq=(1 << 24) + 1),
                                  dict(max_rows=(1 << 20) + 1), dict(n_layers=60000, n_seq=60000, max_seq=1 << 24)])
def test_bad_configs(L, over):
    rc, _, _ = sizes(L, config(**over))
    assert rc == B.ST_EINVAL and L.st_last_error()


def test_create(L):
    _, cb, wb = sizes(L, config())
    h = C.c_void_p(7)
    c = C.byref(config())
    assert L.st_kv4_create(c, PTR, PTR, cb, PTR, wb, None, None) == B.ST_EINVAL
    for args in ((None, PTR, cb, PTR, wb), (PTR, None, cb, PTR, wb), (PTR, PTR, cb, None, wb), (PTR, PTR + 16, cb, PTR, wb),
                 (PTR, PTR, cb, PTR + 128, wb), (PTR + 8, PTR, cb, PTR, wb)):
        assert L.st_kv4_create(c, args[0], args[1], args[2], args[3], args[4], None, C.byref(h)) == B.ST_EINVAL
        assert h.value is None
    assert L.st_kv4_create(c, PTR, PTR, cb - 1, PTR, wb, None, C.byref(h)) == B.ST_ENOMEM
    assert L.st_kv4_create(c, PTR, PTR, cb, PTR, wb - 1, None, C.byref(h)) == B.ST_ENOMEM
    assert L.st_kv4_create(None, PTR, PTR, cb, PTR, wb, None, C.byref(h)) == B.ST_EINVAL
    L.st_kv4_destroy(None)


def spans(*s):
    return (B.st_kv4_span * max(len(s), 1))(*s), len(s)


BAD_SPANS = [([(5, 0, 0, 1)], B.ST_ERANGE), ([(-1, 0, 0, 1)], B.ST_ERANGE), ([(0, -1, 0, 1)], B.ST_ERANGE), ([(0, 1000, 0, 1)], B.ST_ERANGE),
             ([(0, 0, 0, -1)], B.ST_ERANGE), ([(0, 1, -1, 1)], B.ST_ERANGE), ([(0, 2 ** 31 - 1, 0, 2 ** 31 - 1)], B.ST_ERANGE),
             ([(1, 0, 0, 1), (0, 0, 0, 1), (1, 5, 0, 1)], B.ST_EINVAL), ([(0, 0, 0, 65)], B.ST_ERANGE),
             ([(0, 0, 0, 40), (1, 0, 0, 25)], B.ST_ERANGE)]


@pytest.mark.parametrize("bad,code", BAD_SPANS)
def test_bad_spans(L, kv, bad, code):
    s, n = spans(*bad)
    assert L.st_kv4_append(kv, 0, s, n, PTR, 2048, None, None, PTR, 1536, None) == code
    assert L.st_kv4_attend(kv, 0, s, n, PTR, 1536, PTR, 1536, None) == code


def test_append_refusals(L, kv):
    s, n = spans((0, 3, 1999, 1))
    ok = dict(layer=0, s=s, n=n, qkv=PTR, stride=2048, qn=None, kn=None, q=PTR, qs=1536, led=None)

    def call(**over):
        a = dict(ok, **over)
        return L.st_kv4_append(kv, a["layer"], a["s"], a["n"], a["qkv"], a["stride"], a["qn"], a["kn"], a["q"], a["qs"], a["led"])

    late, m = spans((0, 3, 2000, 1))                      # past the rotation table
    assert call(s=late, n=m) == B.ST_ERANGE
    assert call(layer=3) == call(layer=-1) == B.ST_ERANGE
    assert call(qkv=None) == call(qkv=PTR + 2) == call(stride=2040) == call(stride=2049) == B.ST_EINVAL
    assert call(q=None) == call(q=PTR + 8) == call(qs=1528) == call(qs=1537) == B.ST_EINVAL
    assert call(qn=PTR) == call(kn=PTR) == call(qn=PTR, kn=PTR + 4) == B.ST_EINVAL
    assert call(n=65) == call(n=-1) == call(s=None) == B.ST_EINVAL
    for led in (B.st_kv4_ledger(None, PTR), B.st_kv4_ledger(PTR, None), B.st_kv4_ledger(PTR + 2, PTR)):
        assert call(led=C.byref(led)) == B.ST_EINVAL
    assert L.st_kv4_append(None, 0, s, n, PTR, 2048, None, None, PTR, 1536, None) == B.ST_EINVAL


def test_attend_refusals(L, kv):
    s, n = spans((0, 3, 0, 1))
    assert L.st_kv4_attend(None, 0, s, n, PTR, 1536, PTR, 1536, None) == B.ST_EINVAL
    assert L.st_kv4_attend(kv, 3, s, n, PTR, 1536, PTR, 1536, None) == B.ST_ERANGE
    for q, qs, o, os_ in ((None, 1536, PTR, 1536), (PTR, 1536, None, 1536), (PTR + 4, 1536, PTR, 1536), (PTR, 1530, PTR, 1536),
                          (PTR, 1536, PTR, 1535), (PTR, 1536, PTR + 2, 1536)):
        assert L.st_kv4_attend(kv, 0, s, n, q, qs, o, os_, None) == B.ST_EINVAL


def test_matrices_that_share_memory(L, kv):
    s, n = spans((0, 3, 0, 2), (1, 0, 0, 3))
    attend = lambda q, qs, o, os_: L.st_kv4_attend(kv, 0, s, n, q, qs, o, os_, None)
    for q, qs, o, os_ in ((PTR, 1536, PTR, 1536), (PTR, 1536, PTR + 2 * 1528, 1536), (PTR + 16, 1536, PTR, 1536), (PTR, 4096, PTR + 2 * 4096, 4096),
                          (PTR, 4096, PTR + 2 * 1528, 4096), (PTR, 4096, PTR + 2 * 2568, 4096), (PTR + 2 * 2568, 4096, PTR, 4096),
                          (PTR, 3096, PTR + 2 * 1536, 3088), (PTR + 2 * (4 * 1536 + 1528), 1536, PTR, 1536)):
        assert attend(q, qs, o, os_) == B.ST_EINVAL and b"share" in L.st_last_error()
    assert L.st_kv4_append(kv, 0, s, n, PTR, 2048, None, None, PTR, 2048, None) == B.ST_EINVAL and b"share" in L.st_last_error()
    assert L.st_kv4_append(kv, 0, s, n, PTR, 2048, None, None, PTR + 2 * 2048, 1536, None) == B.ST_EINVAL and b"share" in L.st_last_error()


def test_evict_refusals(L, kv):
    led = B.st_kv4_ledger(PTR, PTR)
    s, n = spans((0, 300, 500, 0))

    def call(lo=0, hi=3, s=s, n=n, keep=100, recent=10, led=C.byref(led), into=None):
        return L.st_kv4_evict(kv, lo, hi, s, n, keep, recent, led, into)

    assert call(keep=0) == call(keep=-5) == call(recent=-1) == call(recent=101) == call(led=None) == B.ST_EINVAL
    assert call(lo=-1) == call(hi=4) == call(lo=2, hi=1) == B.ST_ERANGE
    rows, m = spans((0, 300, 500, 1))
    assert call(s=rows, n=m) == B.ST_EINVAL
    twice, m = spans((0, 300, 500, 0), (0, 300, 500, 0))
    assert call(s=twice, n=m) == B.ST_EINVAL
    assert call(into=C.byref(B.st_kv4_ledger(PTR, PTR + 4096))) == B.ST_EINVAL     # one array shared
    assert call(into=C.byref(B.st_kv4_ledger(None, PTR))) == B.ST_EINVAL
    size, base = 4 * 3 * 5 * 2 * 1000, 0x10000000
    far = C.byref(B.st_kv4_ledger(base, base + 64 * size))
    for off in (4, size - 4, -4, 4 - size):
        assert call(led=far, into=C.byref(B.st_kv4_ledger(base + off, base + 16 * size))) == B.ST_EINVAL
        assert call(led=far, into=C.byref(B.st_kv4_ledger(base + 16 * size, base + 64 * size + off))) == B.ST_EINVAL
    assert L.st_kv4_evict(None, 0, 1, s, n, 1, 0, C.byref(led), None) == B.ST_EINVAL


def test_read_refusals(L, kv):
    s, n = spans((0, 3, 0, 1))
    assert L.st_kv4_read(None, 0, 1, s, n, PTR, PTR) == B.ST_EINVAL
    assert L.st_kv4_read(kv, 0, 4, s, n, PTR, PTR) == L.st_kv4_read(kv, 2, 1, s, n, PTR, PTR) == B.ST_ERANGE
    assert L.st_kv4_read(kv, 0, 1, s, n, None, PTR) == L.st_kv4_read(kv, 0, 1, s, n, PTR, PTR + 8) == B.ST_EINVAL


def test_calls_with_nothing_to_do(L, kv):
    none, n = spans((0, 3, 0, 0), (2, 0, 0, 0))
    led = B.st_kv4_ledger(PTR, PTR)
    assert L.st_kv4_append(kv, 0, none, n, PTR, 2048, None, None, PTR, 1536, None) == B.ST_OK
    assert L.st_kv4_attend(kv, 0, none, n, PTR, 1536, PTR, 1536, C.byref(led)) == B.ST_OK
    assert L.st_kv4_attend(kv, 0, None, 0, PTR, 1536, PTR, 1536, None) == B.ST_OK
    assert L.st_kv4_read(kv, 0, 3, none, n, PTR, PTR) == B.ST_OK
    assert L.st_kv4_evict(kv, 1, 1, none, n, 5, 0, C.byref(led), None) == B.ST_OK
    assert L.st_kv4_evict(kv, 0, 3, None, 0, 5, 0, C.byref(led), None) == B.ST_OK


def plan(L, c, s, n, ledger=0):
    columns, blocks, ranges = C.c_int32(-1), C.c_int32(-1), (C.c_int32 * 64)(*[-1] * 64)
    rc = L.st_kv4_attend_plan(C.byref(c), s, n, ledger, C.byref(columns), C.byref(blocks), ranges)
    return rc, columns.value, blocks.value, list(ranges)[:max(n, 0)]


def test_attend_plan(L):
    c = config(n_q_heads=40, n_kv_heads=8, n_seq=64, max_seq=1 << 20, max_rows=1 << 16)
    assert plan(L, c, None, 0) == (B.ST_OK, 0, 0, [])
    assert plan(L, c, *spans((3, 9, 0, 0))) == (B.ST_OK, 0, 0, [0])
    rc, columns, blocks, ranges = plan(L, c, *spans((0, 1 << 19, 0, 1)))
    assert rc == B.ST_OK and columns == 16 and ranges == [64] and blocks == 8 * 64
    assert plan(L, c, *spans((0, 0, 0, 1)))[1:] == (16, 8, [1])
    assert plan(L, c, *spans((0, 100, 0, 20), (1, 0, 0, 0)))[1] == 32
    assert plan(L, c, *spans((0, 511, 0, 1), (1, 0, 0, 1)))[3] == [1, 1] and plan(L, c, *spans((0, 512, 0, 1), (1, 0, 0, 1)))[3] == [5, 1]
    assert plan(L, c, *spans((0, 511, 0, 1), (1, 0, 0, 1)), ledger=1)[3] == [4, 1]     # joined beside the weights
    assert plan(L, c, *spans((0, 0, 0, 1 << 16)))[1:] == (128, 8 * (1 << 16) * 5 // 128, [1])
    assert L.st_kv4_attend_plan(C.byref(c), *spans((0, 5, 0, 1)), 0, None, None, None) == B.ST_OK
    assert plan(L, config(head_dim=96), *spans((0, 0, 0, 1)))[0] == B.ST_EINVAL
    assert L.st_kv4_attend_plan(None, None, 0, 0, None, None, None) == B.ST_EINVAL
    for bad, code in BAD_SPANS:
        assert plan(L, config(), *spans(*bad))[0] == code


def test_ranges_stay_within_what_the_workspace_holds(L):
    """Wherever slots are cut into ranges: at most 512 blocks, 64 ranges of a span, and partial results for every row and head."""
    for nq, nkv in ((1, 1), (12, 2), (40, 8), (16, 1), (4096, 256)):
        for max_rows in (1, 7, 64, 5000):
            c = config(n_layers=1, n_q_heads=nq, n_kv_heads=nkv, n_seq=64, max_seq=1 << 22, max_rows=max_rows)
            held = min(max_rows * nq * 64, 512 * 128)
            for n in (1, 3, 64):
                for rows in (1, 2, max_rows // n):
                    for length in (0, 31, 4097, 1 << 21):
                        if rows < 1 or rows * n > max_rows:
                            continue
                        s = spans(*((j, length if j % 2 == 0 else length // 3, 0, rows) for j in range(n)))
                        rc, columns, blocks, ranges = plan(L, c, *s, ledger=rows % 2)
                        cut = [r for r in ranges if r > 1]
                        assert rc == B.ST_OK and min(ranges) >= 1 and max(ranges) <= 64
                        assert blocks == sum(r * nkv * -(-rows * (nq // nkv) // columns) for r in ranges)
                        assert not cut or (blocks <= 512 and sum(cut) * rows * nq <= held), (nq, nkv, max_rows, n, rows, length)


def test_evict_into_the_other_array_of_the_ledger(L, kv):
    """`into` may be the ledger or lie apart from it: its weights where the ledger's positions are, or the reverse, is refused as any other overlap."""
    s, n = spans((0, 300, 500, 0))
    size, base = 4 * 3 * 5 * 2 * 1000, 0x10000000
    led, far = B.st_kv4_ledger(base, base + 4 * size), base + 64 * size
    for off in (0, 4, size - 4, -4, 4 - size):
        for into in ((base + 4 * size + off, far), (far, base + off)):
            assert L.st_kv4_evict(kv, 0, 3, s, n, 100, 10, C.byref(led), C.byref(B.st_kv4_ledger(*into))) == B.ST_EINVAL
            assert b"overlap" in L.st_last_error()
    assert L.st_kv4_evict(kv, 0, 3, s, n, 100, 10, C.byref(led), C.byref(B.st_kv4_ledger(led.positions, led.weights))) == B.ST_EINVAL
    for off in (0, 4, 4 - size):                          # an `into` whose arrays share memory
        assert L.st_kv4_evict(kv, 0, 3, s, n, 100, 10, C.byref(led), C.byref(B.st_kv4_ledger(far, far + off))) == B.ST_EINVAL
    none = spans()
    for off in (size, -size):                             # side by side
        assert L.st_kv4_evict(kv, 0, 3, *none, 100, 10, C.byref(led), C.byref(B.st_kv4_ledger(base + 4 * size + off, far))) == B.ST_OK
