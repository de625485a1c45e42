"""Host-only checks of what the calls of the paged cache and of the verdict over drafts refuse at the ends of their ranges."""
import ctypes as C

import pytest

from paper_2504_12329_amd import binding as B

from .test_paged_host import L, PTR, verifier  # noqa: F401


@pytest.mark.parametrize("call,number", [("st_verify_drafts", C.c_float), ("st_verify_drafts64", C.c_double)])
def test_temperatures(L, verifier, call, number):  # noqa: F811
    """Of either width: refused where they are none, and looked at before anything else is (tokens are missing from every call)"""
    def code(heat, n=2):
        rows = (C.c_int32 * 64)(*[1] * 64)
        t = None if heat is None else (number * len(heat))(*heat)
        return getattr(L, call)(verifier, rows, n, None, None, PTR, 1000, None, 0, t, PTR, PTR, PTR, 1, PTR, PTR), L.st_last_error()
    for bad in (-1.0, float("nan"), float("inf"), -float("inf")):
        assert code([1.0, bad])[0] == B.ST_EINVAL and b"sequence 1: bad temperature" in code([1.0, bad])[1]
    for fine in (0.0, -0.0, 1e-45, 0.6, 3e38):
        assert code([fine, 1.0])[0] == B.ST_EINVAL and b"an array is NULL" in code([fine, 1.0])[1]
    assert code(None)[0] == B.ST_EINVAL and b"temperature is NULL" in code(None)[1]
    assert code([1.0] * 63 + [-1.0], 64)[1].startswith(b"sequence 63") and code([1.0] * 65, 65)[0] == B.ST_EINVAL and code([], 0)[0] == B.ST_OK
    if number is C.c_double:
        assert code([5e-324, 1.7e308])[1] == b"an array is NULL"


def test_positions_that_trees_need():
    trees = [[-1, 0, 1, 0, 2], [-1, 0, 0], [], [-1]]
    s = B.DraftSpans([(0, 9, 20, 5), (1, 0, 21, 3), (2, 0, 5, 0), (3, 7, 7, 1)], trees, device="cpu")
    assert s.positions == 24 and s.at([(0, 9, 5, 5), (1, 0, 8, 3), (2, 0, 30, 0), (4, 0, 3, 1)]).positions == 30
    assert B.DraftSpans([], [], device="cpu").positions == 0
