"""The trees of the draft trace, on the CPU."""
from paper_2504_12329_amd import draft_trace


def test_trees():
    assert draft_trace.parents_of([]) == ([-1], [0, 1])
    assert draft_trace.parents_of([1, 1, 1]) == ([-1, 0, 1, 2], [0, 1, 2, 3, 4])
    assert draft_trace.parents_of([3, 2]) == ([-1, 0, 0, 0, 1, 1, 2, 2, 3, 3], [0, 1, 4, 10])
