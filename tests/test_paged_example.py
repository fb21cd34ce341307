"""CPU checks of how examples/paged_answer.py makes block lists from evidence spans."""
import pytest
import torch

from examples.paged_answer import span_blocks


def plain(starts, span_len, page, last, top):
    named = [0, last, max(last - 1, 0)] + [b for s in starts if s >= 0 for b in range(s // page, min((s + span_len - 1) // page, last) + 1)]
    kept = sorted(list(dict.fromkeys(named))[:top])
    return kept + [-1] * (top - len(kept))


@pytest.mark.parametrize("starts,span_len,page,last,top", [
    ([0, 192, 576, 1280, 1920, 2112], 64, 64, 47, 12),            # whole blocks: one each
    ([10, 200, 600, 1300, 1950, 2150], 64, 64, 47, 12),           # two each, more than there is room for: the worst spans' are left out
    ([2990, 5, -1, -1], 40, 64, 46, 8),                           # no such span; a span that ends with the context
    ([-1, -1], 64, 64, 9, 5),
    ([0], 16, 64, 0, 4),                                          # a context of one block
    ([100, 90, 400], 300, 16, 60, 32),
])
def test_lists_keep_the_first_and_the_newest_blocks(starts, span_len, page, last, top):
    got = span_blocks(torch.tensor(starts), span_len, page, last, top, "cpu").tolist()
    assert got == plain(starts, span_len, page, last, top)
    assert 0 in got and last in got
