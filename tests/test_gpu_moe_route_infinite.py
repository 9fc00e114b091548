"""Biases that force an expert or forbid it, beside each other in a group."""
import numpy as np
import pytest

from tests.test_gpu_moe_route import inputs, run

pytestmark = pytest.mark.gpu

INF = np.inf


@pytest.mark.parametrize("sigmoid", (False, True))
def test_infinities_of_both_signs_in_a_group(sigmoid):
    """Groups of two: a forced expert and a forbidden one, two forbidden ones, two of finite scores each.  The first has no sum and comes last."""
    x, w, _ = inputs(3, 5, 8, 128)
    bias = np.array([INF, -INF, -INF, -INF, 0, 0, 0, 0], dtype=np.float32)
    score = lambda top: run(x, w, 2 * top, bias=bias, sigmoid=sigmoid, groups=4, top_groups=top, normalise=False)[0]  # noqa: E731
    two, three, four = score(2), score(3), score(4)
    assert (np.sort(two, axis=1) == [4, 5, 6, 7]).all()
    assert np.array_equal(three[:, :4], two) and (three[:, 4:] == [2, 3]).all()
    assert (four[:, 0] == 0).all() and np.array_equal(four[:, 1:5], two) and (four[:, 5:] == [1, 2, 3]).all()


def test_a_forced_expert_beside_finite_ones():
    x, w, _ = inputs(4, 5, 9, 128)
    bias = np.array([0, 0, 0, -INF, 0, INF, 0, 0, 0], dtype=np.float32)
    ids = run(x, w, 3, bias=bias, groups=3, top_groups=1, normalise=False)[0]
    assert (ids == [5, 4, 3]).all()
