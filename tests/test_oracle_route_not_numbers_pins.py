"""Pins for the oracle's router where active logits are not numbers: a token with one counts and shows it."""
import numpy as np
import pytest

from oracle import route as orc

NAN, INF = np.nan, np.inf


@pytest.mark.parametrize("row", [[NAN] * 4, [NAN, -INF, NAN, -INF], [-INF, -INF, -INF, NAN], [NAN, 1, 2, -INF]])
def test_a_token_with_a_nan_is_not_an_empty_one(row):
    x = np.array([row, [0.0, 1, 2, 3], [-INF] * 4])
    route, p, counts, loss = orc.route_topk(x, 2)
    barred = np.array(row) == -INF
    assert np.isnan(p[0, ~barred]).all() and not p[0, barred].any()
    numbers = [b for b in range(4) if np.isfinite(row[b])]
    assert route[0].tolist() == [1 if b in sorted(numbers, key=lambda b: -row[b])[:2] else 0 for b in range(4)]
    assert counts[4] == 2 and np.isnan(loss)
    assert not p[2].any() and not route[2].any()                 # all barred: nothing
    d = orc.route_backward(p, counts, np.ones((3, 4)), 1.0)
    assert np.isnan(d[0, ~barred]).all() and np.array_equal(d[0, barred], np.zeros(barred.sum()))
    assert np.isfinite(d[1]).all() and not d[2].any()


def test_one_branch():
    route, p, counts, loss = orc.route_topk(np.array([[NAN], [2.0]]), 1)
    assert np.isnan(p[0, 0]) and p[1, 0] == 1 and route.tolist() == [[0], [1]] and counts.tolist() == [1, 2] and np.isnan(loss)


def test_nothing_but_nans_has_no_finite_loss():
    route, p, counts, loss = orc.route_topk(np.full((3, 2), NAN), 1)
    assert np.isnan(p).all() and not route.any() and counts.tolist() == [0, 0, 3] and np.isnan(loss)


def test_padding_and_inactive_branches_hide_theirs():
    x = np.array([[NAN, 0.0, 1.0], [NAN, NAN, NAN]])
    route, p, counts, loss = orc.route_topk(x, 1, active=[0, 1, 1], real=[1, 0])
    assert np.isfinite(p).all() and counts.tolist() == [0, 0, 1, 1] and np.isfinite(loss)
