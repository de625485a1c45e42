"""The cache in pages where scores and positions are at their ends, against its definition in 64 bits (paged_ref).  Tolerances as in test_gpu_paged, where nothing else is
said."""
import numpy as np
import pytest
import torch

from paper_2504_12329_amd import binding as B

from . import paged_ref as R
from .test_gpu_paged import HALF, TYPES, check_append, contents, f64, make, random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [1, 3, 9, 40])
@pytest.mark.parametrize("sign", [1, -1])
def test_attend_scores_far_from_zero(dtype, d, rows, sign):
    """Scores of 2^16 to 2^33 (fp16), 2^83 (bf16) and more: the largest of them have the weight, those of one size share it.  Keys and queries are a number in all channels, so that every fp32 sum
    is exact (six bits times a power of two) and scores are equal or at least a 64th apart: nothing but the rounding of
    weights and outputs is left."""
    rng = np.random.default_rng(rows + d)
    kv, table = make(4, 2, d, dtype=dtype, n_pages=200, max_pages=60, n_seq=3)
    sizes = [2.0 ** e for e in ((7, 12, 15) if dtype is torch.float16 else (7, 12, 20, 40))]
    for size in sizes:
        for lens in ((0, 40, 700), (300, 17, 900 - rows)):
            spans = [(j, n, 0, rows) for j, n in enumerate(lens)]
            steps = torch.from_numpy(rng.integers(32, 64, (200, 1, 16, 1))).double() / 64    # several slots have the largest
            kv.cache[0, 0] = (sign * size * steps).expand(200, 2, 16, d).to(dtype).cuda()
            q = torch.full((rows * 3, 4, d), 2.0 ** 15 if dtype is torch.float16 else size, device="cuda").to(dtype)
            parents = [random_tree(rng, rows) for _ in spans]
            for plan, seen_of in ((B.Kv4Spans(spans), lambda j, i: range(i + 1)), (B.DraftSpans(spans, parents), lambda j, i: R.branch(parents[j], i))):
                got, at = f64(kv.attend(0, plan, q)), 0
                for j, (seq, length, _, n) in enumerate(spans):
                    k, v, there = contents(kv, table, seq, length + n)
                    for i in range(n):
                        seen = np.array([*range(length), *(length + x for x in seen_of(j, i))])
                        want, spread, total = R.attention(f64(q[at + i]), k, v, seen)
                        tol = (HALF[dtype] + 2.0 ** -15) * spread + HALF[dtype] * np.abs(want) + (2.0 ** -25 * (total + 1) if dtype is torch.float16 else 0)
                        assert (np.abs(got[at + i] - want) <= tol).all(), f"scores of {size * float(q[0, 0, 0]) * d ** 0.5:.3g}, span {j} row {i}"
                    at += n


@pytest.mark.parametrize("nats", [9.0, 14.0, 17.5, 20.0])
@pytest.mark.parametrize("nq,nkv,d,rows", [(4, 2, 64, 1), (4, 2, 128, 9), (4, 2, 64, 40), (12, 2, 128, 40)])
@pytest.mark.parametrize("length", [450, 3000])
def test_attend_one_slot_stands_above_many(nats, nq, nkv, d, rows, length):
    """fp16: many weights far below the largest one's 1 are together what the output consists of.  They are rounded at 2^-15 of where numbers of the type are (the largest is
    2^15): h of a weight, and 2^-40 below 2^-29; an output below 2^-14 by 2^-25."""
    rng = np.random.default_rng(rows)
    kv, table = make(nq, nkv, d, dtype=torch.float16, n_pages=220, max_pages=200, n_seq=1)
    kv.cache[0] = 0.0
    kv.cache[1] = 30 * (1 + kv.cache[1].double() / 8).half()
    page, slot = R.place(table, 220, 16, 0, 5)
    kv.cache[0, 0, page, :, slot] = torch.tensor(nats / d ** 0.5).half()
    kv.cache[1, 0, page, :, slot] = 0.0
    q = torch.ones(rows, nq, d, device="cuda").half()
    got, (k, v, _) = f64(kv.attend(0, B.Kv4Spans([(0, length, 0, rows)]), q)), contents(kv, table, 0, length + rows)
    for i in range(rows):
        want, size, total = R.attention(f64(q[i]), k, v, np.arange(length + i + 1))
        tol = (2.0 ** -11 + 2.0 ** -15) * size + 2.0 ** -11 * np.abs(want) + 2.0 ** -40 * total + 2.0 ** -25
        assert (np.abs(got[i] - want) <= tol).all(), f"row {i}: {(np.abs(got[i] - want) / tol).max()} of the tolerance"


def test_append_refuses_drafts_past_the_rotation_table():
    """As it does chains of as many rows; what the trees of a step need is known on the host"""
    rng = np.random.default_rng(2)
    kv, table = make(4, 2, 64, max_pos=100, n_seq=2)
    deep, wide = [-1, 0, 1, 0, 2], [-1, 0, 0]                                 # depths of 3 and 1
    check_append(kv, table, [(0, 3, 96, 5), (1, 0, 98, 3)], [deep, wide], True, rng)
    x = torch.randn(8, 8 * 64, device="cuda").bfloat16()
    was = kv.cache.clone()
    for spans in ([(0, 3, 97, 5), (1, 0, 98, 3)], [(0, 3, 96, 5), (1, 0, 99, 3)]):
        for plan in (B.DraftSpans(spans, [deep, wide]), B.DraftSpans([(0, 3, 0, 5), (1, 0, 0, 3)], [deep, wide]).at(spans)):
            with pytest.raises(B.StError, match="positions") as e:
                kv.append(0, plan, x)
            assert e.value.code == B.ST_ERANGE
    assert torch.equal(kv.cache, was)
    still, table = make(4, 2, 64, max_pos=100, n_seq=2, rot=0)                # nothing rotates, wherever it is
    trees = B.DraftSpans([(0, 3, 97, 5), (1, 0, 99, 3)], [deep, wide])
    q = still.append(0, trees, x)
    assert torch.equal(q.flatten(1), x[:, :256]) and torch.equal(q, still.append(0, trees.at([(0, 3, 0, 5), (1, 0, 0, 3)]), x))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nq,nkv,d,rows,length", [(4, 2, 64, 1, 0), (4, 2, 64, 5, 40), (12, 2, 128, 9, 3000), (12, 2, 128, 40, 300)])
def test_attend_rows_whose_scores_are_all_minus_infinity(dtype, nq, nkv, d, rows, length):
    """Zeros, and other heads and rows as they are"""
    kv, table = make(nq, nkv, d, dtype=dtype, n_pages=220, max_pages=200, n_seq=1)
    q = torch.randn(rows, nq, d, device="cuda").to(dtype).abs()
    q[rows // 2] = -q[rows // 2]                                              # its scores are all +infinity: NaN
    plan = B.Kv4Spans([(0, length, 0, rows)])
    want = kv.attend(0, plan, q)
    kv.cache[0, 0, :, 0, :, 3] = -float("inf")                                # of one kv head
    got = kv.attend(0, plan, q)
    others = [i for i in range(rows) if i != rows // 2]
    assert (got[others, :nq // nkv] == 0).all() and torch.equal(got[:, nq // nkv:], want[:, nq // nkv:])
    assert torch.isnan(got[rows // 2, :nq // nkv]).all() and torch.isfinite(want).all()
