"""Plain float64 definition of a learner's update with its singular values pushed towards one.  Pinned by singular value decompositions in
tests/test_oracle_orthogonalise.py."""
import numpy as np


def orthogonalise(x, coefficients, eps=1e-7):
    """x [m,n], coefficients [steps][3] -> the result, float64."""
    x = np.asarray(x, np.float64)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / (np.sqrt((x ** 2).sum()) + eps)
    for a, b, c in coefficients:
        gram = x @ x.T
        x = a * x + (b * gram + c * gram @ gram) @ x
    return x.T if tall else x
