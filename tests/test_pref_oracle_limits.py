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
