"""What a row's log-probability and gradient keep of their precision: under shifts of the row, of masks of the type's lowest value, and summed over
long sequences."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from operator_util import HALF_ULP, stream, values, within
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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_ten_parts(dtype):
    """A vocabulary of 151936: ten parts a row, whose sums are joined in two groups of eight."""
    Case(dtype, 151936, [2, 3, 1, 2], [0, 1], PARAMS, ld=151936 + 24).run().check().check_logp()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [300, 20000])
def test_masked_entries_within_bounds_that_are_numbers(dtype, V):
    """A third of the vocabulary at minus infinity, a third at the lowest value: probability and gradient 0 there, and the others' as without them."""
    rng = np.random.default_rng(4)
    z, live = values(rng, (12, V), dtype, 2.0), V // 3
    targets = rng.integers(0, live, 12)
    targets[[0, 7]] = -100
    z[:, live:2 * live], z[:, 2 * live:] = -np.inf, LOWEST[dtype]
    z[0], z[7] = np.nan, np.inf
    c = Case(dtype, V, [6, 6], [1], PARAMS, z=z, targets=targets).run()
    got, w = c.dz.host(), c.want
    assert np.all(got[[0, 7]] == 0.0) and np.all(got[:, live:] == 0.0) and np.all(w["dz"][:, live:] == 0.0)
    rows = [t for t in range(12) if t not in (0, 7)]
    p = np.exp(z[rows, :live] - w["lse"][rows][:, None])
    p[np.arange(10), targets[rows]] += 1.0
    k = np.abs(np.repeat(w["coef"], 6))[rows]
    want = w["dz"][rows][:, :live]
    bound = HALF_ULP[dtype] * np.abs(want) * 1.01 + 2.0 ** -12 * k[:, None] * p
    assert np.isfinite(bound).all()
    within(got[rows][:, :live], want, bound, "dz")
    bare = Case(dtype, live, [6, 6], [1], PARAMS, ref=False, z=np.where(np.isfinite(z[:, :live]), z[:, :live], 0.0), targets=targets)
    assert np.allclose(bare.want["row"], w["row"], rtol=1e-13, atol=1e-13)
    ml.multi_lora_pref_logp(c.pref, c.d_z, c.ld, c.d_t, c.logp, c.ws, row_logp=c.row, stream=stream())
    within(c.row.host()[0], w["row"], 2.0 ** -19 + 2.0 ** -24 * np.abs(w["row"]), "row_logp")
