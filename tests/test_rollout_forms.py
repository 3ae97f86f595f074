"""Pins of the rollout step's plain forms (no GPU)."""
import numpy as np

from oracle import rollout


def test_pages_form_serves_who_needs_no_page_after_pages_ran_out():
    """By hand: two pages are left; request 0 takes one, request 2 wants three,
    request 3 has room in the pages that it holds."""
    table = np.array([[0, -1, -1, -1], [1, -1, -1, -1], [2, -1, -1, -1], [3, 4, -1, -1]], np.int32)
    o = rollout.pages_extend([16, 3, 16, 20], [1, 1, 1, 2], [1, 5, 40, 3], [7, 8, 9], 2, table, 16,
                             60)
    assert o["error"] and o["taken"] == 1
    assert o["kv_len"].tolist() == [17, 8, 16, 23] and o["held"].tolist() == [2, 1, 1, 2]
    assert o["slots"].tolist() == [112] + [16 + x for x in range(3, 8)] + [-1] * 40 \
        + [68, 69, 70] + [-1] * 11
