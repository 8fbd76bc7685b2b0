"""Sequences of probability 0 (a counted target's logit is minus infinity: a masked vocabulary): infinite margins, and losses that only the terms with
a weight have a part in."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from operator_util import HALF_ULP, values, within
from test_gpu_pref import Case

pytestmark = pytest.mark.gpu

SMOOTHING = [0.0, 1.0, 0.0, 1.0, 0.25]
# which sequence of the adapter's first pair has probability 0, and what that makes of its loss and margin
CHOSEN, REJECTED = 0, 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [300, 2500])
@pytest.mark.parametrize("side", [CHOSEN, REJECTED])
def test_terms_without_weight_have_no_part(dtype, V, side):
    rng = np.random.default_rng(3)
    N = len(SMOOTHING)
    lens, owner = [3, 4] * (2 * N), [i for i in range(N) for _ in range(2)]
    T = sum(lens)
    z, targets = values(rng, (T, V), dtype, 2.0), rng.integers(0, V, T)
    gone = [14 * i + 3 * side + 1 for i in range(N)]              # a row of the adapter's first pair
    for t in gone:
        z[t, targets[t]] = -np.inf
    c = Case(dtype, V, lens, owner, [(0.5, a, 0.0) for a in SMOOTHING], ref=False, z=z, targets=targets).run()
    margin, loss, logp = c.margin.host()[0], c.loss.host()[0], c.logp.host()[0]
    sign = 1.0 if side == REJECTED else -1.0
    assert np.all(margin[0::2] == sign * np.inf) and np.isfinite(margin[1::2]).all()
    assert np.all(logp[side::4] == -np.inf)
    for i, a in enumerate(SMOOTHING):
        m = margin[2 * i + 1].astype(float)
        other = ((1 - a) * np.logaddexp(0, -m) + a * np.logaddexp(0, m)) / 2
        weight = a if side == REJECTED else 1 - a                 # of the term that is infinite
        want = np.inf if weight > 0 else other
        assert c.want["loss"][i] == pytest.approx(want, rel=1e-4), i
        assert loss[i] == pytest.approx(want, rel=2.0 ** -20), i
    # the gradient: sigma is 0 or 1
    got, w = c.dz.host(), c.want
    assert np.isfinite(got).all()
    k = np.abs(np.repeat(w["coef"], lens))
    p = np.exp(np.where(np.isfinite(z), z, -1e30) - w["lse"][:, None])
    p[np.arange(T), targets] += 1.0
    within(got, w["dz"], HALF_ULP[dtype] * np.abs(w["dz"]) * 1.01 + 2.0 ** -12 * k[:, None] * p, "dz")


def test_likelihood_of_an_impossible_sequence():
    """The likelihood term has its weight: infinite with it, and no part without."""
    rng = np.random.default_rng(4)
    z, targets = values(rng, (14, 90), "f32", 2.0), rng.integers(0, 90, 14)
    z[1, targets[1]] = z[8, targets[8]] = -np.inf
    c = Case("f32", 90, [3, 4, 3, 4], [0, 1], [(0.5, 1.0, 0.0), (0.5, 1.0, 0.3)], ref=False, z=z, targets=targets).run()
    loss = c.loss.host()[0]
    assert loss[0] == 0.0 and loss[1] == np.inf and np.array_equal(c.want["loss"], [0.0, np.inf])
