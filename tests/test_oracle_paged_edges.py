"""The paged oracle at the ends of the types, by hand-worked cases and against the plain definition."""
import numpy as np
import pytest

from oracle import paged

INF = np.inf
KEPT = float(np.float32(3e38))


@pytest.mark.parametrize("q,lo,hi,want", [
    ([2.0, 1.0], [-INF, -1.0], [3.0, 1.0], 7.0),            # a key of -inf in a column where q is positive: the others of the page still count
    ([-2.0, 1.0], [-3.0, -1.0], [INF, 1.0], 7.0),
    ([2.0, 1.0], [-1.0, -1.0], [INF, 1.0], INF),
    ([-2.0, 1.0], [-INF, -1.0], [1.0, 1.0], INF),
    ([2.0, 1.0], [-INF, -1.0], [-INF, 1.0], -INF),          # every key of the page is -inf there
    ([0.0, 1.0], [-INF, -1.0], [INF, 1.0], 1.0),            # 0 times an infinity counts as 0
    ([0.0, 0.0], [-INF, -1.0], [INF, 1.0], 0.0),
    ([INF, 1.0], [0.0, -1.0], [0.0, 1.0], 1.0),
    ([2.0, 1.0], [INF, -1.0], [-INF, 1.0], INF),            # no number in the column at all: the page is kept
    ([2.0, 1.0], [-INF, -1.0], [-INF, INF], KEPT),          # infinities of both signs meet
    ([np.nan, 1.0], [-1.0, -1.0], [1.0, 1.0], KEPT),
])
def test_page_score_at_the_ends(q, lo, hi, want):
    assert paged.page_score_any(np.array([q]), np.array([lo, hi]), 1.0) == want
    # a second row that scores less changes nothing
    if want > 0:
        assert paged.page_score_any(np.array([q, [0.0, 0.0]]), np.array([lo, hi]), 1.0) == want


def test_page_score_any_is_page_score():
    g = np.random.default_rng(3)
    for _ in range(20):
        q, rows = g.standard_normal((3, 16)), g.standard_normal((5, 16))
        edge = paged.bounds(rows)
        assert abs(paged.page_score_any(q, edge, 0.3) - paged.page_score(q, edge, 0.3)[0]) < 1e-12
