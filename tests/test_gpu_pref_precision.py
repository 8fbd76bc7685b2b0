"""What a row's log-probability and gradient keep of their precision: under shifts of the row, of masks of the type's lowest value, and summed over
long sequences."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from operator_util import stream, values, within
from paper_2604_05426_amd import binding as ml
from test_gpu_pref import PARAMS, Case

pytestmark = pytest.mark.gpu

LOWEST = {"bf16": float(torch.finfo(torch.bfloat16).min), "f32": float(np.finfo(np.float32).min)}


def results(c):
    """Outputs of both forwards and the backward of a case."""
    c.run()
    out = [t.host() for t in (c.logp, c.margin, c.loss, c.dz)]
    ml.multi_lora_pref_logp(c.pref, c.d_z, c.ld, c.d_t, c.logp, c.ws, row_logp=c.row, stream=stream())
    return out + [c.row.host(), c.logp.host()]


@pytest.mark.parametrize("dtype,grid,shifts", [("f32", 2.0 ** -6, (1000.0, -1000.0, 2.0 ** 16)), ("bf16", 0.5, (64.0, -64.0))])
@pytest.mark.parametrize("V", [700, 20000])
def test_a_shifted_row_is_the_same_row(dtype, grid, shifts, V):
    """Logits on a grid that the type holds around the shift too: the differences in a row are the same numbers, so every result is, bit for bit."""
    rng = np.random.default_rng(1)
    lens, owner = [9, 4, 6, 7], [0, 1]
    z = np.round(np.clip(rng.standard_normal((26, V)) * 1.5, -7, 7) / grid) * grid
    targets = rng.integers(0, V, 26)
    base = Case(dtype, V, lens, owner, PARAMS, z=z, targets=targets)
    want = results(base)
    base.check().check_logp()
    for s in shifts:
        moved = z + s
        c = Case(dtype, V, lens, owner, PARAMS, z=moved, targets=targets)
        assert np.array_equal(c.d_z.double().cpu().numpy(), moved)
        c.d_ref = base.d_ref
        for a, b in zip(results(c), want):
            assert np.array_equal(a, b), s


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [300, 40000])
def test_rows_of_the_lowest_value(dtype, V):
    """A row whose every logit is the type's lowest value is uniform: log-probability -log V, gradient k ([target] - 1 / V)."""
    rng = np.random.default_rng(2)
    z = values(rng, (8, V), dtype, 2.0)
    z[3], z[6] = LOWEST[dtype], LOWEST[dtype]
    c = Case(dtype, V, [4, 4], [0], PARAMS, z=z, targets=rng.integers(0, V, 8))
    row = results(c)[4][0]
    u = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}[dtype]
    for t in (3, 6):
        assert c.want["row"][t] == pytest.approx(-np.log(V), rel=1e-12)
        assert abs(row[t] + np.log(V)) <= 2.0 ** -21 * np.log(V)
        within(c.dz.host()[t], c.want["dz"][t], 1.01 * u * np.abs(c.want["dz"][t]) + 2.0 ** -18 * np.abs(c.want["coef"][t // 4]) / V + 2.0 ** -18 * np.abs(c.want["dz"][t]), "dz")
