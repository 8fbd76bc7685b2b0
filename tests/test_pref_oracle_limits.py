"""The preference loss's definition at the ends of its range."""
import numpy as np

from oracle import operators_oracle as oo

LOWEST = float(np.finfo(np.float32).min)


def test_rows_without_a_larger_logit_are_uniform():
    z = np.full((2, 5), LOWEST)
    l, _ = oo.row_logp(z, [0, 3])
    assert np.allclose(l, -np.log(5), rtol=1e-15)
    r = oo.preference(z, [0, 3], [0, 1, 2], [0], [(0.5, 0.0, 0.0)])
    assert np.allclose(r["dz"][0], -0.25 * (np.eye(5)[0] - 0.2)) and np.allclose(r["dz"][1], 0.25 * (np.eye(5)[3] - 0.2))


def test_terms_without_weight_have_no_part_in_a_loss():
    z = np.array([[0.0, -np.inf, 1.0], [0.5, 0.0, 0.0]])
    for smoothing, targets, want in ((0.0, [0, 1], None), (0.0, [1, 0], np.inf), (1.0, [1, 0], 0.0)):
        r = oo.preference(z, targets, [0, 1, 2], [0], [(0.5, smoothing, 0.0)])
        if want is not None:
            assert r["loss"][0] == want
        assert np.isfinite(r["dz"]).all()
    r = oo.preference(z[::-1], [0, 1], [0, 1, 2], [0], [(0.5, 0.0, 0.0)])        # the rejected sequence cannot be: nothing is left to lose
    assert r["margin"][0] == np.inf and r["loss"][0] == 0.0
