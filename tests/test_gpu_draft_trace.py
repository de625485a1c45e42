"""Drafts, verdicts and kept branches over paged caches, as a whole: texts grow by what the large model itself would have written.

Tolerance: the large model reads the finished text once more, in one chunk on a cache of its own; a greedy token's logit lies within twice the bound for two evaluations of a
bf16 model's logits (LOGIT_TOL of the largest) of the largest."""
import pytest
import torch

from paper_2504_12329_amd import draft_trace, synth

from .gpu_common import LOGIT_TOL

pytestmark = pytest.mark.gpu


def models(n_seq, max_rows=64, same=False):
    cfg = synth.model_config("tiny_large", 400)
    weights = synth.make_weights(cfg, 5, device="cuda")
    large, again = (draft_trace.PagedModel("tiny_large", 5, n_seq, 400, r, weights=weights) for r in (max_rows, 200))
    small = draft_trace.PagedModel("tiny_large", 5, n_seq, 400, max_rows, weights=weights) if same else draft_trace.PagedModel("tiny_small", 3, n_seq, 400, max_rows)
    return small, large, again


@pytest.mark.parametrize("widths", [[1], [1, 1, 1, 1, 1], [3, 2, 1], [4, 4]])
@pytest.mark.parametrize("same", [False, True])
def test_greedy_rounds_write_what_the_large_model_would(widths, same):
    prompts = [synth.make_prompt(n, 1024, 40 + n).tolist() for n in (37, 5, 90)]
    small, large, again = models(3, same=same)
    job = draft_trace.Drafting(small, large, prompts, widths, 0.0)
    grown = [0, 0, 0]
    for _ in range(12):
        grown = [a + b for a, b in zip(grown, job.round())]
    assert [len(t) - len(p) for t, p in zip(job.texts, prompts)] == grown and all(t[:len(p)] == p for t, p in zip(job.texts, prompts))
    assert large.len == [len(t) - 1 for t in job.texts] == small.len
    if same:
        assert min(grown) > 12                                # drafts of the model itself stay
    from paper_2504_12329_amd import binding as B
    for s, (text, p) in enumerate(zip(job.texts, prompts)):
        logits = again.forward(torch.tensor(text[:-1], device="cuda"), B.Kv4Spans([(s, 0, 0, len(text) - 1)]))
        for i in range(len(p), len(text)):
            row = logits[i - 1]
            assert row[text[i]] >= row.max() - 2 * LOGIT_TOL * row.abs().max(), f"sequence {s}, token {i}"


@pytest.mark.parametrize("widths", [[1, 1, 1], [2, 2, 1]])
def test_drawn_rounds(widths):
    prompts = [synth.make_prompt(n, 1024, n).tolist() for n in (3, 64)]
    small, large, _ = models(2, same=True)
    job = draft_trace.Drafting(small, large, prompts, widths, 0.8)
    grown = [job.round() for _ in range(10)]
    assert all(1 <= g <= len(widths) + 1 for r in grown for g in r)
    assert large.len == [len(t) - 1 for t in job.texts] and all(0 <= x < 1024 for t in job.texts for x in t)
    assert sum(map(sum, grown)) > 20                           # drafts from the same distribution stay, but for rounding

    again = draft_trace.Drafting(*models(2, same=True)[:2], prompts, widths, 0.8)
    for _ in range(10):
        again.round()
    assert again.texts == job.texts                            # the same seeds, the same texts


def test_the_command(capsys):
    draft_trace.main("--small tiny_small --large tiny_large --layers 0 --sequences 2 --prompt 20 --tokens 12 --widths 2 1".split())
    assert "tokens a round and sequence" in capsys.readouterr().out
