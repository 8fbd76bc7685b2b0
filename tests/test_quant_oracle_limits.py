"""The 8-bit values' definition for blocks with elements that are not finite."""
import numpy as np

from oracle import operators_oracle as oo


def test_elements_that_are_not_finite_leave_the_others_their_scale():
    x = np.array([0.1, -3.0, np.inf, 7.0, np.nan, -np.inf])
    finite = np.isfinite(x)
    q = oo.quantise_block(x)
    assert np.isnan(q[~finite]).all() and np.array_equal(q[finite], oo.quantise_block(x[finite]))
    assert np.isnan(oo.quantise_block(np.full(3, np.inf))).all()
    w = np.zeros((130, 130))
    w[:] = np.linspace(-1, 1, 130)
    clean = oo.quantise_weight(w)
    w[3, 5] = np.inf
    q = oo.quantise_weight(w)
    assert np.isnan(q[3, 5]) and np.isnan(q).sum() == 1 and np.array_equal(np.delete(q, 5, 1), np.delete(clean, 5, 1))
