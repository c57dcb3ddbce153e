"""Pins for the oracle's slots where a sequence of a batch sits a step out."""
import numpy as np
import pytest

import oracle

TABLE = np.array([[7, 3, -1], [9, -1, -1], [2, -1, -1]], dtype=np.int32)
ACCEPTED = np.array([[2, 5, -1], [-1, -1, -1], [0, -1, -1]])


def test_a_sequence_that_sits_out_gains_nothing():
    r = oracle.cache_slots([31, 16, 5], [2, -1, 1], ACCEPTED, [4, 5, 6], 3, TABLE, 8, 16, 12)
    assert r["status"] == 0 and r["free_count"] == 2 and r["context_len"].tolist() == [34, 16, 7]
    assert r["start"].tolist() == [0, 3, 3, 5] and r["page_start"].tolist() == [0, 1, 1, 1]
    assert r["slot"].tolist() == [3 * 16 + 15, 6 * 16, 6 * 16 + 1, 2 * 16 + 5, 2 * 16 + 6] + [-1] * 7
    assert r["source"].tolist() == [0, 3, 6, 16, 17] + [-1] * 7
    assert r["block_table"].tolist() == [[7, 3, 6], [9, -1, -1], [2, -1, -1]]


@pytest.mark.parametrize("add,accepted", [([2, -2, 1], ACCEPTED), ([2, -1, 1], None)])
def test_other_negative_lengths_are_refused(add, accepted):
    assert oracle.cache_slots([31, 16, 5], add, accepted, [4, 5, 6], 3, TABLE, 8, 16, 12)["status"] == 1
