"""Pins of the float64 definition in oracle/learner.py: singular values go through the polynomials, singular vectors stay."""
import numpy as np
import pytest

from oracle import learner

QUINTIC = (3.4445, -4.7750, 2.0315)


@pytest.mark.parametrize("m,n", [(1, 1), (5, 5), (4, 9), (9, 4), (1, 6)])
@pytest.mark.parametrize("coefficients", [[QUINTIC] * 5, [(1.5, -0.5, 0.0)] * 3, [(2.0, 0.0, 0.0)], [(1.0, 1.0, 1.0), QUINTIC]])
def test_singular_values(m, n, coefficients):
    x = np.random.default_rng(m * 10 + n).standard_normal((m, n))
    u, t, v = np.linalg.svd(x, full_matrices=False)
    t = t / (np.linalg.norm(t) + 1e-7)
    for a, b, c in coefficients:
        t = a * t + b * t ** 3 + c * t ** 5
    assert np.allclose(learner.orthogonalise(x, coefficients), u * t @ v)


def test_limits():
    # the cubic's fixed point: a matrix with orthonormal rows; the transpose of a matrix gives the transpose of the result; scale does not matter
    x = np.random.default_rng(0).standard_normal((6, 8))
    y = learner.orthogonalise(x, [(1.5, -0.5, 0.0)] * 40)
    assert np.allclose(y @ y.T, np.eye(6))
    assert np.allclose(learner.orthogonalise(x.T, [QUINTIC] * 5), learner.orthogonalise(x, [QUINTIC] * 5).T)
    assert np.allclose(learner.orthogonalise(x * 1e5, [QUINTIC] * 5, eps=0.0), learner.orthogonalise(x, [QUINTIC] * 5, eps=0.0))
    assert (learner.orthogonalise(np.zeros((3, 4)), [QUINTIC] * 5) == 0).all()
