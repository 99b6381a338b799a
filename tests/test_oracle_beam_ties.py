"""Pins of the oracle's order of candidates of one value: of a beam by logit, equal ones the lower token first; between beams the
lower beam first. No test here touches a GPU."""
import numpy as np

from oracle import step_oracle as so


def test_logits_that_a_score_hides():
    for score in (-1e30, 1e30):
        s, p, t = so.beam_select(np.array([[1.0, 1.5, 2.0, 0.0]]), np.array([[score]]), 4)
        assert t.tolist() == [[2, 1, 0, 3]] and p.tolist() == [[0] * 4] and s.tolist() == [[score] * 4]


def test_beams_of_one_value():
    x = np.array([[1.0, 2.0, 2.0], [9.0, -np.inf, 3.0]])
    s, p, t = so.beam_select(x, np.full((1, 2), -1e30), 6, None, 1)
    assert p.tolist() == [[0, 0, 0, 1, 1, -1]] and t.tolist() == [[1, 2, 0, 0, 2, 1]]
    s, p, t = so.beam_select(x, np.full((1, 2), -1e30), 6, np.array([[False, True]]), 1)
    assert p.tolist() == [[0, 0, 0, 1, -1, -1]] and t.tolist() == [[1, 2, 0, 1, 1, 1]]


def test_logits_too_small_to_show():
    x = np.zeros((1, 6))
    x[0, [1, 4]] = [1e-30, 2e-30]
    assert so.beam_select(x, np.zeros((1, 1)), 6)[2].tolist() == [[4, 1, 0, 2, 3, 5]]
