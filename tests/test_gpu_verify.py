"""The verdict over drafted tokens on the GPU against its definition in 64 bits (paged_ref.verify): rows, numbers and tokens are equal.  Both sides compute in 64 bits, so
that they could only differ where a random number lies within some 1e-13 of a verdict's border; the inputs are fixed by their seeds."""
import numpy as np
import pytest
import torch

from paper_2504_12329_amd import binding as B

from . import paged_ref as R

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def random_tree(rng, rows, width):
    p, free = [-1], [width]
    for i in range(1, rows):
        at = int(rng.choice([k for k in range(i) if free[k] > 0]))
        free[at] -= 1
        free.append(width)
        p.append(at)
    return p


def inputs(rng, parents, vocab, T, with_draft, near=0.7, spread=3.0):
    """(tokens, target, draft) of one sequence: drafts as they come about, drawn from the draft's distribution or its best ones"""
    rows = len(parents)
    target = rng.standard_normal((rows, vocab)) * spread
    draft = target + near * rng.standard_normal((rows, vocab))
    tokens = np.zeros(rows, dtype=np.int64)
    for i in range(rows):
        after = [c for c in range(rows) if c and parents[c] == i]
        best = np.argsort(-draft[i])
        for k, c in enumerate(after):
            tokens[c] = rng.choice(vocab, p=R.softmax(draft[i], T)) if with_draft and T > 0 else best[k % vocab]
    return tokens, target, draft


def check(rng, trees, vocab, heats, with_draft, dtype=torch.float32, chain=False, width=None, change=None, pad=0, offset=0):
    first = np.cumsum([0] + [len(p) for p in trees])
    parts = [inputs(rng, p, vocab, T, with_draft) for p, T in zip(trees, heats)]
    tokens = np.concatenate([x[0] for x in parts])
    logits = [torch.full((first[-1], vocab + pad + offset), 9.0, dtype=dtype, device="cuda")[:, offset:offset + vocab] for _ in range(2)]
    for k in (0, 1):
        logits[k].copy_(torch.from_numpy(np.concatenate([x[1 + k] for x in parts])))
    accept, sample = rng.random(first[-1]), rng.random(len(trees))
    if change:
        change(tokens, logits[0], logits[1], accept, sample)
    spans = [(j, 0, 0, len(p)) for j, p in enumerate(trees)]
    plan = B.Kv4Spans(spans) if chain else B.DraftSpans(spans, trees)
    if width is not None:
        plan = B.DraftSpans.of_tensors(spans, parent=plan.parent, width=width)
    v = B.DraftVerifier(vocab, int(first[-1]) + 3, max_width=1 if chain else max(plan.width, 2), dtype=dtype)
    v._ws.fill_(255)
    c = lambda x, t: torch.from_numpy(x).to(t).cuda()  # noqa: E731
    path, accepted, after = v.verify(plan, c(tokens, torch.int32), logits[0], heats if len(set(heats)) > 1 else heats[0], c(accept, torch.float64), c(sample, torch.float64),
                                     draft=logits[1] if with_draft else None)
    t64, d64 = (x.double().cpu().numpy() for x in logits)
    got = []
    for j, p in enumerate(trees):
        a, b = first[j], first[j + 1]
        want, token = R.verify(p, tokens[a:b], t64[a:b], d64[a:b] if with_draft else None, heats[j], accept[a:b], sample[j], width or 64)
        n = int(accepted[j])
        assert (path[j, :n].tolist(), int(after[j])) == (want, token), f"sequence {j}, temperature {heats[j]}"
        assert (path[j, n:] == -1).all()
        got.append((want, token))
    return got


def chains(rows):
    return [list(range(-1, n - 1)) for n in rows]


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("vocab", [1, 2, 17, 1000, 8191, 8192, 8193, 30011])
def test_chains(dtype, with_draft, vocab):
    rng = np.random.default_rng(vocab)
    for rows in ((1,), (2, 1, 6), (5, 21, 3, 9)):
        for heats in ([1.0] * len(rows), [0.0] * len(rows), [(0.6, 0.0, 2.5, 1.0)[j] for j in range(len(rows))]):
            check(rng, chains(rows), vocab, heats, with_draft, dtype, chain=True)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("vocab,width", [(2, 3), (40, 2), (40, 8), (9001, 3), (20000, 5)])
def test_trees(dtype, with_draft, vocab, width):
    rng = np.random.default_rng(vocab + width)
    ends = []
    for rows in ((1,), (2, 4), (30, 17, 8), (65, 2)):
        trees = [random_tree(rng, r, width) for r in rows]
        for heats in ([1.0] * len(rows), [(0.7, 0.0, 1.5)[j] for j in range(len(rows))]):
            ends += check(rng, trees, vocab, heats, with_draft, dtype)
    assert any(len(p) > 1 for p, _ in ends) and any(len(p) == 0 for p, _ in ends)


@pytest.mark.parametrize("with_draft", [False, True])
def test_many_sequences_and_long_trees(with_draft):
    rng = np.random.default_rng(5)
    check(rng, [random_tree(rng, 1 + j % 5, 3) for j in range(64)], 300, [(1.0, 0.0, 0.5)[j % 3] for j in range(64)], with_draft)
    check(rng, [random_tree(rng, 1024, 64), chains([1024])[0], random_tree(rng, 700, 2)], 100, [1.0, 0.8, 0.0], with_draft)


@pytest.mark.parametrize("with_draft", [False, True])
def test_wide_rows(with_draft):
    """64 rows after one, most of them failing"""
    rng = np.random.default_rng(6)

    def change(tokens, target, draft, accept, sample):
        accept[:60] = 1 - 1e-9
    check(rng, [[-1] + [0] * 64, [-1] + [0] * 64], 500, [1.0, 1.0], with_draft, change=change)
    check(rng, [[-1] + [0] * 64], 5, [1.0], with_draft, change=change)                    # more drafts than tokens: the same ones again


@pytest.mark.parametrize("with_draft", [False, True])
def test_width_bounds_the_drafts_that_are_tried(with_draft):
    rng = np.random.default_rng(7)
    for width in (1, 2, 3):
        check(rng, [random_tree(rng, 40, 6) for _ in range(6)], 50, [1.0] * 6, with_draft, width=width)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("vocab,pad,offset", [(8193, 0, 1), (8193, 0, 0), (20000, 3, 5), (777, 8, 3)])
def test_rows_that_start_anywhere(dtype, with_draft, vocab, pad, offset):
    rng = np.random.default_rng(vocab + pad)
    check(rng, [random_tree(rng, 12, 3) for _ in range(3)], vocab, [1.0, 0.0, 0.7], with_draft, dtype, pad=pad, offset=offset)


def test_target_and_draft_that_start_at_different_places():
    rng = np.random.default_rng(8)
    tree, vocab = random_tree(rng, 20, 3), 9000
    tokens, target, draft = inputs(rng, tree, vocab, 1.0, True)
    accept, sample = rng.random(20), rng.random(1)
    a = torch.from_numpy(target).float().cuda()
    b = torch.zeros(20, vocab + 7, device="cuda")[:, 3:3 + vocab]
    b.copy_(torch.from_numpy(draft))
    v = B.DraftVerifier(vocab, 20, max_width=3)
    c = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    path, n, after = v.verify(B.DraftSpans([(0, 0, 0, 20)], [tree]), c(tokens).int(), a, 1.0, c(accept), c(sample), draft=b)
    want = R.verify(tree, tokens, a.double().cpu().numpy(), b.double().cpu().numpy(), 1.0, accept, sample[0])
    assert (path[0, :int(n)].tolist(), int(after)) == want


@pytest.mark.parametrize("with_draft", [False, True])
def test_infinities_and_nan(with_draft):
    rng = np.random.default_rng(9)
    inf, nan = float("inf"), float("nan")

    def masked(tokens, target, draft, accept, sample):          # tokens that are forbidden
        target[:, ::2] = -inf
        draft[:, 1::3] = -inf

    def nothing(tokens, target, draft, accept, sample):
        target[2], target[5] = -inf, -inf
        draft[9] = -inf

    def spoiled(tokens, target, draft, accept, sample):
        target[1, 77], target[4, 8500], draft[8, 0], target[12, 3] = nan, inf, nan, -inf

    trees = [random_tree(rng, 9, 2), chains([9])[0]]
    for change in (masked, nothing, spoiled):
        for heats in ([1.0, 1.0], [0.0, 0.5], [0.0, 0.0]):
            check(rng, trees, 9000, heats, with_draft, change=change)
    check(rng, chains([3, 3]), 9000, [1.0, 0.0], with_draft, chain=True, change=lambda k, t, d, a, s: t.fill_(nan))
    one = lambda k, t, d, a, s: (t.fill_(-inf), t[:, 8200].fill_(2.0))  # noqa: E731
    assert all(token == 8200 for _, token in check(rng, chains([3, 3]), 9000, [1.0, 0.0], with_draft, chain=True, change=one))


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("vocab,offset", [(9000, 0), (4099, 3), (16, 0)])
def test_few_tokens_are_allowed(dtype, with_draft, vocab, offset):
    """Nine tokens of ten forbidden to the target, others to the draft, and drafts that mostly fail, side by side"""
    rng = np.random.default_rng(vocab)

    def change(tokens, target, draft, accept, sample):
        for x, part in ((target, 0.9), (draft, 0.5)):
            out = rng.random(tuple(x.shape)) < part
            out[:, vocab // 2] = False
            x.masked_fill_(torch.from_numpy(out).cuda(), -float("inf"))
        tokens[1::2] = vocab // 2 + np.arange(len(tokens[1::2])) % (vocab - vocab // 2)
        accept[:] = 1 - (1 - accept) / 16
    ends = check(rng, [random_tree(rng, n, 5) for n in (40, 25, 12)], vocab, [1.0, 0.6, 1.5], with_draft, dtype, offset=offset, change=change)
    ends += check(rng, chains([6, 9, 3]), vocab, [1.0, 0.6, 1.5], with_draft, dtype, chain=True, offset=offset, change=change)
    assert any(len(p) == 0 for p, _ in ends)


@pytest.mark.parametrize("with_draft", [False, True])
def test_random_numbers_at_their_ends(with_draft):
    rng = np.random.default_rng(10)
    for u in (0.0, 1 - 2.0 ** -53):
        for x in (0.0, 1 - 2.0 ** -53, 0.5):
            def change(tokens, target, draft, accept, sample):
                accept[:], sample[:] = u, x
                target[:, :5] = -float("inf")                   # neither the first nor the last token has a weight
                target[:, -5:] = -float("inf")
            check(rng, [random_tree(rng, 15, 3), chains([5])[0]], 9000, [1.0, 0.6], with_draft, change=change)


def test_the_same_distribution_keeps_every_first_draft():
    rng = np.random.default_rng(11)
    for vocab in (50, 9000):
        got = check(rng, chains([20, 7]), vocab, [1.0, 0.7], True, chain=True, change=lambda k, t, d, a, s: d.copy_(t))
        assert [len(p) for p, _ in got] == [19, 6]


def test_ties_go_to_the_lowest_token():
    rng = np.random.default_rng(12)

    def change(tokens, target, draft, accept, sample):
        target.clamp_(max=1.0)
        tokens[1::2] = target.double().argmax(1).cpu().numpy()[0]
    for dtype in TYPES.values():
        check(rng, [random_tree(rng, 12, 3) for _ in range(3)], 20000, [0.0] * 3, False, dtype, change=change)


@pytest.mark.parametrize("with_draft", [False, True])
def test_tokens_outside_the_vocabulary_do_not_stay(with_draft):
    rng = np.random.default_rng(13)

    def change(tokens, target, draft, accept, sample):
        tokens[1::3], tokens[2::5] = -1, 900
        accept[::2] = 0.0
    check(rng, [random_tree(rng, 30, 3) for _ in range(4)], 900, [1.0, 0.5, 0.0, 2.0], with_draft, change=change)


def test_rows_that_follow_none_are_not_reached():
    rng = np.random.default_rng(14)
    v = B.DraftVerifier(100, 6, max_width=4)
    target = torch.zeros(6, 100, device="cuda")
    parent = torch.tensor([0, 0, 5, -7, 2 ** 31 - 1, 2], dtype=torch.int32, device="cuda")   # row 2 follows a later one; only row 1 is in the tree
    plan = B.DraftSpans.of_tensors([(0, 0, 0, 6)], parent=parent, width=4)
    zeros = torch.zeros(6, dtype=torch.float64, device="cuda")
    path, n, after = v.verify(plan, torch.arange(6, dtype=torch.int32, device="cuda"), target, 1.0, zeros, torch.full((1,), 0.5, dtype=torch.float64, device="cuda"))
    assert path.tolist() == [[1, -1, -1, -1, -1, -1]] and n.tolist() == [1] and after.tolist() == [50]


def test_tokens_that_stay_are_distributed_as_the_targets():
    """One draft after a row, then the token after it or in its place: over many random numbers every token comes as often as the target has it.  40000 draws of a token of
    probability p: off by at most 5 sqrt(p (1 - p) / 40000) but once in two million, for each of 2 x 12 tokens."""
    rng = np.random.default_rng(15)
    vocab, draws = 12, 40000
    target, draft = rng.standard_normal(vocab) * 1.5, rng.standard_normal(vocab) * 1.5
    p, q = R.softmax(target, 0.8), R.softmax(draft, 0.8)
    for tree in ([-1, 0], [-1, 0, 0, 0]):
        rows, counts, done = len(tree), np.zeros(vocab), 0
        v = B.DraftVerifier(vocab, 64 * rows, max_width=3)
        plan = B.DraftSpans([(j, 0, 0, rows) for j in range(64)], [tree] * 64)
        lt = torch.from_numpy(np.tile(target, (64 * rows, 1))).float().cuda()
        ld = torch.from_numpy(np.tile(draft, (64 * rows, 1))).float().cuda()
        tokens, firsts = [], []
        while done < draws:
            k = rng.choice(vocab, p=q, size=64 * rows)
            t = torch.from_numpy(k).int().cuda()
            a, s = (torch.from_numpy(rng.random(m)).cuda() for m in (64 * rows, 64))
            path, n, after = v.verify(plan, t, lt, 0.8, a, s, draft=ld)
            tokens.append(torch.where(n > 0, t.view(64, rows).gather(1, path[:, :1].clamp(min=0).long())[:, 0], after))
            done += 64
        counts = torch.bincount(torch.cat(tokens), minlength=vocab).cpu().numpy() / done
        assert (np.abs(counts - p) <= 5 * np.sqrt(p * (1 - p) / done)).all(), (tree, counts, p)


def test_the_same_call_twice_and_a_handle_of_another_size():
    rng = np.random.default_rng(16)
    trees = [random_tree(rng, 20, 3) for _ in range(3)]
    a = check(rng, trees, 5000, [1.0] * 3, True)
    rng = np.random.default_rng(16)
    trees = [random_tree(rng, 20, 3) for _ in range(3)]
    assert check(rng, trees, 5000, [1.0] * 3, True) == a
