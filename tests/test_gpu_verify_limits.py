"""The verdict over drafted tokens where its numbers are at their ends, against its definition in 64 bits (paged_ref.verify): rows, numbers and tokens are equal, as in
test_gpu_verify."""
import numpy as np
import pytest
import torch

from paper_2504_12329_amd import binding as B

from . import paged_ref as R
from .test_gpu_verify import TYPES, chains, check, random_tree

pytestmark = pytest.mark.gpu


# ---- logits that are large against the temperature ----

@pytest.mark.parametrize("name,value", [("fp32", None), ("fp32", -1e30), ("fp32", -1e20), ("bf16", None), ("bf16", -1e30), ("bf16", -1e20), ("fp16", None)])
@pytest.mark.parametrize("with_draft", [False, True])
def test_parts_of_a_row_that_are_masked_by_a_finite_number(name, value, with_draft):
    """value None: the type's lowest"""
    dtype = TYPES[name]
    low = torch.finfo(dtype).min if value is None else value
    rng = np.random.default_rng(1)

    def change(tokens, target, draft, accept, sample):
        target[:, 8192:24576] = low
        draft[:, 4096:12288] = low
        draft[:, ::2] = low
    for heats in ([1.0, 0.8, 0.7], [0.6, 0.9, 0.3], [0.1, 1.5, 0.0]):
        check(rng, [random_tree(rng, 7, 2) for _ in heats], 30011, heats, with_draft, dtype, change=change)
        check(rng, chains([3, 1, 5]), 30011, heats, with_draft, dtype, chain=True, change=change)


@pytest.mark.parametrize("top", ["lowest", -1e30, 1e30, 3e38])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("with_draft", [False, True])
def test_rows_whose_largest_logits_are_far_from_zero(top, dtype, with_draft):
    """Nothing is left but equal numbers, a few or all of a row: they share it"""
    top = torch.finfo(dtype).min if top == "lowest" else top
    rng = np.random.default_rng(2)

    def few(tokens, target, draft, accept, sample):
        target[:] = -float("inf")
        target[:, 77::2000] = top
        draft[:, 77::1000] = top

    def every(tokens, target, draft, accept, sample):
        target[::2], draft[1::2] = top, top
    for change in (few, every):
        for heats in ([1.0, 0.8], [0.7, 0.6], [2.5, 0.0]):
            check(rng, [random_tree(rng, 8, 3), random_tree(rng, 5, 1)], 9001, heats, with_draft, dtype, change=change)
            check(rng, chains([4, 2]), 9001, heats, with_draft, dtype, chain=True, change=change)


@pytest.mark.parametrize("T", [1e-9, 1e-12, 1e-17, 1e-18, 1e-20, 1e-30, 1.5e-45])
@pytest.mark.parametrize("with_draft", [False, True])
def test_temperatures_near_zero(T, with_draft):
    rng = np.random.default_rng(3)

    def shared(tokens, target, draft, accept, sample):          # many tokens have the largest logit
        target.clamp_(max=2.0)
        draft.clamp_(max=1.0)
    for change in (None, shared):
        for vocab in (50, 9000):
            check(rng, [random_tree(rng, 12, 3) for _ in range(3)], vocab, [T, 1.0, T], with_draft, change=change)
            check(rng, chains([1, 6]), vocab, [T, T], with_draft, chain=True, change=change)
            check(rng, chains([12, 6]), vocab, [T, 0.7], with_draft, torch.bfloat16, chain=True, change=change)


# ---- target and draft that agree ----

@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("vocab,masked", [(50, False), (9001, False), (9001, True)])
def test_nothing_is_left_of_a_distribution_less_itself(dtype, vocab, masked):
    """Drafts that cannot stay (no tokens), then others: what is left of p is empty, no draft after them stays, and the next token is drawn from p itself"""
    rng = np.random.default_rng(4)

    def change(tokens, target, draft, accept, sample):
        if masked:
            target[:, ::3] = -float("inf")
        draft.copy_(target)
        tokens[1:] = np.where(rng.random(len(tokens) - 1) < 0.5, -1, rng.integers(0, vocab, len(tokens) - 1))
        tokens[[1, 2, 3]] = -1
        accept[4::2] = 0.0
    for heats in ([1.0, 1.0], [0.5, 2.0]):
        got = check(rng, [[-1, 0, 0, 0], [-1, 0, 0, 1]], vocab, heats, True, dtype, change=change)
        assert got[0][0] == []
        check(rng, [random_tree(rng, 30, 5), random_tree(rng, 20, 4)], vocab, heats, True, dtype, change=change)
        check(rng, chains([4, 2]), vocab, heats, True, dtype, chain=True, change=change)
    for _ in range(10):
        check(rng, chains([4, 2, 12]), vocab, [1.0] * 3, True, dtype, chain=True, change=change)


@pytest.mark.parametrize("vocab", [9001, 30011])
@pytest.mark.parametrize("how", ["place", "shift"])
def test_the_same_distribution_from_other_numbers(vocab, how):
    """Rows that are cut into parts at other places, or logits that differ by one constant (multiples of 2^-8 up to 16: exactly)"""
    rng = np.random.default_rng(5)
    n = 16
    target = torch.from_numpy(np.round(rng.standard_normal((2 * n, vocab)) * 768) / 256).clamp_(-15, 15).float().cuda()
    wide = torch.zeros(2 * n, vocab + 7, device="cuda")
    draft = wide[:, 3:3 + vocab] if how == "place" else wide[:, :vocab]
    draft.copy_(target if how == "place" else target + 37.25)
    tokens, accept, sample = np.tile([0, -1], n), rng.random(2 * n), rng.random(n)
    v = B.DraftVerifier(vocab, 2 * n)
    c = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    path, counts, after = v.verify(B.Kv4Spans([(j, 0, 0, 2) for j in range(n)]), c(tokens).int(), target, 0.7, c(accept), c(sample), draft=draft)
    assert counts.tolist() == [0] * n
    x = target.double().cpu().numpy()
    want = [R.verify([-1, 0], tokens[:2], x[2 * j:2 * j + 2], x[2 * j:2 * j + 2], 0.7, accept[2 * j:2 * j + 2], sample[j])[1] for j in range(n)]
    assert after.tolist() == want


# ---- the temperature ----

@pytest.mark.parametrize("T", [0.6, 0.7, 0.8, 0.9, 1 / 3, 1e-3])
def test_the_temperature_is_not_rounded(T):
    """Random numbers half way between the borders that T and T rounded to 32 bits have: 5e-11 and more from either, at sums that are right to 1e-13"""
    rng = np.random.default_rng(6)
    near, vocab, n = float(np.float32(T)), 3000, 24
    x = np.float32(rng.standard_normal((2 * n, vocab)) * (3.0 if T > 0.1 else 0.01)).astype(np.float64)
    y = np.float32(x + 0.7 * (1.0 if T > 0.1 else 0.003) * rng.standard_normal(x.shape)).astype(np.float64)
    tokens, accept, sample = np.zeros(2 * n, dtype=np.int64), np.full(2 * n, 0.999), rng.random(n)
    for j in range(n):
        p, q, p32, q32 = (R.softmax(z[2 * j], t) for t in (T, near) for z in (x, y))
        if j % 3 == 0:                                           # the draft's verdict
            ratio, ratio32 = p / q, p32 / q32
            t = int(np.argmax(np.where(np.maximum(ratio, ratio32) < 1, np.abs(ratio - ratio32), 0)))
            assert abs(ratio[t] - ratio32[t]) > 1e-10
            tokens[2 * j + 1], accept[2 * j + 1] = t, (ratio[t] + ratio32[t]) / 2
        else:                                                    # the token after a draft that failed; j % 3 == 1: no token at all
            tokens[2 * j + 1] = -1
            left, left32 = (R.left_over(a, b) for a, b in ((p, q), (p32, q32)))
            sums, sums32 = np.cumsum(left), np.cumsum(left32)
            t = int(np.argmax(np.abs(sums - sums32)))
            assert abs(sums[t] - sums32[t]) > 1e-10
            sample[j] = (sums[t] + sums32[t]) / 2
    v = B.DraftVerifier(vocab, 2 * n)
    c = lambda z: torch.from_numpy(z).cuda()  # noqa: E731
    path, counts, after = v.verify(B.Kv4Spans([(j, 0, 0, 2) for j in range(n)]), c(tokens).int(), c(x).float(), T, c(accept), c(sample), draft=c(y).float())
    want = [R.verify([-1, 0], tokens[2 * j:2 * j + 2], x[2 * j:2 * j + 2], y[2 * j:2 * j + 2], T, accept[2 * j:2 * j + 2], sample[j]) for j in range(n)]
    assert [(path[j, :k].tolist(), t) for j, (k, t) in enumerate(zip(counts.tolist(), after.tolist()))] == want
    for j in range(0, n, 3):                                     # without draft logits, the border of a draft and of a token
        p, p32 = R.softmax(x[2 * j], T), R.softmax(x[2 * j], near)
        t = int(np.argmax(np.abs(p - p32)))
        assert abs(p[t] - p32[t]) > 1e-10
        tokens[2 * j + 1], accept[2 * j + 1] = t, (p[t] + p32[t]) / 2
    path, counts, after = v.verify(B.Kv4Spans([(j, 0, 0, 2) for j in range(n)]), c(tokens).int(), c(x).float(), T, c(accept), c(sample))
    want = [R.verify([-1, 0], tokens[2 * j:2 * j + 2], x[2 * j:2 * j + 2], None, T, accept[2 * j:2 * j + 2], sample[j]) for j in range(n)]
    assert [(path[j, :k].tolist(), t) for j, (k, t) in enumerate(zip(counts.tolist(), after.tolist()))] == want


@pytest.mark.parametrize("T", [5e-324, 1e-300, 1e-100, 1e-45, 1e38, 1e100, 1.7e308])
@pytest.mark.parametrize("with_draft", [False, True])
def test_temperatures_past_32_bits(T, with_draft):
    """Below them the largest logits share a row, above them all of its tokens do"""
    rng = np.random.default_rng(7)

    def change(tokens, target, draft, accept, sample):
        target[::2].clamp_(max=1.0)
        draft[1::2].clamp_(max=1.0)
        target[:, 5:9] = -float("inf")
    with np.errstate(over="ignore"):
        check(rng, [random_tree(rng, 12, 3) for _ in range(3)], 9000, [T, 1.0, T], with_draft, change=change)
        check(rng, chains([5, 2]), 9000, [T, 0.0], with_draft, chain=True, change=change)


# ---- many parts of a row ----

@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("pad,offset", [(0, 0), (2, 1), (1, 5)])
def test_rows_of_several_large_parts(dtype, with_draft, pad, offset):
    """512 parts of 8192 logits and more: the form of the sums that large calls take; rows of four parts that start and end inside one"""
    rng = np.random.default_rng(8 + offset)

    def change(tokens, target, draft, accept, sample):
        target[3, 8000:17000], target[5, 24570] = -float("inf"), float("nan")
        draft[7, 16380:] = -float("inf")
    trees = [random_tree(rng, n, 3) for n in ((30, 24, 25) if with_draft else (60, 50, 48))]
    check(rng, trees, 30011, [1.0, 0.7, 1.3], with_draft, dtype, pad=pad, offset=offset)
    check(rng, trees, 30011, [0.0, 0.5, 0.0], with_draft, dtype, pad=pad, offset=offset, change=change)
    if dtype is torch.bfloat16:
        check(rng, chains([len(p) for p in trees]), 30011, [0.6, 1.0, 0.0], with_draft, dtype, chain=True, pad=pad, offset=offset)


@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("vocab,rows", [(300001, (3, 2)), (1100003, (3, 2))])
def test_rows_of_more_parts_than_a_wave_has_lanes(with_draft, vocab, rows):
    """The smaller vocabulary: 147 small parts, 74 of the draw; the larger: 135 large parts, 269 of the draw"""
    rng = np.random.default_rng(vocab)
    dtype = torch.float32 if vocab < 1 << 20 else torch.bfloat16

    def late(tokens, target, draft, accept, sample):            # all that has a weight lies behind the first 64 parts
        target[:, :vocab - 20000] = -float("inf")
    for change in (None, late):
        for heats in ([1.0, 0.7], [0.0, 1.0]):
            check(rng, chains(rows), vocab, heats, with_draft, dtype, chain=True, change=change, offset=1)
            check(rng, [[-1, 0, 0], [-1, 0]], vocab, heats, with_draft, dtype, change=change)


@pytest.mark.parametrize("with_draft", [False, True])
def test_a_token_in_each_part(with_draft):
    """The token is found in whichever part it is, and the parts before it count"""
    rng = np.random.default_rng(9)
    vocab, at = 300001, [0, 4095, 4096, 65535, 262143, 262144, 266239, 266240, 300000]

    def change(tokens, target, draft, accept, sample):
        target.fill_(-float("inf"))
        target[:, at] = 0.0
        draft.fill_(0.0)
        tokens[:] = 1
        sample[:] = (np.arange(len(sample)) + 0.5) / len(at)
    got = check(rng, chains([2] * len(at)), vocab, [1.0] * len(at), with_draft, chain=True, change=change)
    assert [t for _, t in got] == at
