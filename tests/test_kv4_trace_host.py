"""The trace's contexts on the CPU, with the models' passes replaced."""
import torch

from paper_2504_12329_amd import kv4_trace


def context(max_rows, seen):
    m = kv4_trace.Context.__new__(kv4_trace.Context)
    m.max_rows = max_rows

    def forward(x, rows):
        seen.append(list(rows))
        assert x.shape[0] == sum(rows) and max(rows) <= max_rows
        return 2 * x
    m.forward = forward
    return m


def test_prefill_gives_back_every_row_of_sequences_of_unequal_length():
    for rows in ([5], [30, 5, 17], [8, 8], [1, 0, 16], [3, 24]):
        seen, x = [], torch.arange(sum(rows) * 4.0).view(-1, 4)
        assert torch.equal(context(8, seen).prefill(x, rows), 2 * x), rows
        assert [sum(r) for r in zip(*seen)] == rows


def test_prefill_without_rows():
    seen = []
    assert context(8, seen).prefill(torch.zeros(0, 4), [0, 0]).shape == (0, 4) and not seen
