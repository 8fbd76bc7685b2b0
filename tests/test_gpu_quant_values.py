"""Values that the 8-bit products have to keep in their places: infinities and NaN in the weight, the largest and smallest scales, and fp32 rows that different
tiles take."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from operator_util import values
from oracle import operators_oracle as oo
from paper_2604_05426_amd.workloads import round_to_bf16
from test_gpu_quant import Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [5, 300])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_infinities_and_nans_of_the_weight_stay_in_their_row_and_column(dtype, T, bad):
    """W[r, c] makes column c of Y and column r of dX (the element's row of W) NaN; every other output has the bits it had."""
    rng = np.random.default_rng(1)
    k, n = 300, 270
    X, W, dY = values(rng, (T, k), dtype), values(rng, (k, n), dtype, 0.02), values(rng, (T, n), dtype, 0.01)
    places = [(5, 9), (131, 200), (299, 269)]
    for at in places:
        W[at] = 0.0                                   # not its block's largest magnitude, whose scale stays
    clean = Layer(dtype, T, k, n, X=X, W=W, dY=dY).run().check()
    y, dx = clean.Y.host(), clean.dX.host()
    dirty = W.copy()
    for at in places:
        dirty[at] = bad
    got = Layer(dtype, T, k, n, X=X, W=dirty, dY=dY).run()
    rows, cols = [a for a, _ in places], [b for _, b in places]
    gy, gdx = got.Y.host(), got.dX.host()
    assert np.isnan(gy[:, cols]).all() and np.isnan(gdx[:, rows]).all()
    assert np.array_equal(np.delete(gy, cols, 1), np.delete(y, cols, 1))
    assert np.array_equal(np.delete(gdx, rows, 1), np.delete(dx, rows, 1))


def test_weight_of_nothing_finite():
    """A block without a finite element has no magnitude: its outputs are NaN, its neighbours' are theirs."""
    rng = np.random.default_rng(2)
    X, W, dY = values(rng, (20, 256), "bf16"), values(rng, (256, 256), "bf16", 0.02), values(rng, (20, 256), "bf16", 0.01)
    clean = Layer("bf16", 20, 256, 256, X=X, W=W, dY=dY).run()
    y, dx = clean.Y.host(), clean.dX.host()
    W = W.copy()
    W[:128, 128:] = np.inf
    got = Layer("bf16", 20, 256, 256, X=X, W=W, dY=dY).run()
    assert np.isnan(got.Y.host()[:, 128:]).all() and np.array_equal(got.Y.host()[:, :128], y[:, :128])
    assert np.isnan(got.dX.host()[:, :128]).all() and np.array_equal(got.dX.host()[:, 128:], dx[:, 128:])


SCALES = [-127, -126, -125, 0, 118, 119, 120]


def codes(e):
    """Every 8-bit value times 2^e that fp32 holds, 128 of them, the largest one such that 2^e is the block's scale."""
    tab = oo.e4m3_values()
    if e == 120:
        tab = np.minimum(tab, 240.0)                  # above, 2^120 times the value passes the largest fp32 number
    row = np.concatenate([tab, [tab[-1]]]) * 2.0 ** e
    assert np.array_equal(row, row.astype(np.float32).astype(float))
    return row


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_largest_and_smallest_scales(dtype):
    """All 8-bit values through products with the identity, as activations and as the weight, under the scales at both ends of their range.  A scale below
    2^-126 has values that the result's type holds as denormal numbers or, flushed, as zeros."""
    def near(got, want):
        keep = np.abs(want) >= 2.0 ** -126
        assert np.array_equal(got[keep], want[keep])
        assert np.all(np.abs(got[~keep] - want[~keep]) <= 2.0 ** -126)

    X = np.array([codes(e) * (-1) ** i for i, e in enumerate(SCALES)])
    if dtype == "bf16":
        X = round_to_bf16(X.astype(np.float32)).astype(float)             # (its numbers end at 2^-133)
    L = Layer(dtype, len(SCALES), 128, 128, X=X, W=np.eye(128), dY=X).run()
    want = oo.quantise_rows(X)
    near(L.Y.host(), want)
    near(L.dX.host(), want)
    for e in SCALES:
        W = np.zeros((128, 128))
        W[:, 0] = codes(e)
        W[0, :] = codes(e)[::-1]
        W[0, 0] = codes(e)[127]
        if dtype == "bf16":
            W = round_to_bf16(W.astype(np.float32)).astype(float)
        L = Layer(dtype, 128, 128, 128, X=np.eye(128), W=W, dY=np.eye(128)).run()
        want = oo.quantise_weight(W)
        near(L.Y.host(), want)
        near(L.dX.host(), want.T)


def test_a_single_precision_row_does_not_depend_on_the_tile():
    """Row counts by which the products take each of the three fp32 kernels."""
    rng = np.random.default_rng(11)
    k, n = 700, 2100
    X, dY, W = values(rng, (2050, k), "f32"), values(rng, (2050, n), "f32", 0.01), values(rng, (k, n), "f32", 0.02)
    many = Layer("f32", 2050, k, n, X=X, W=W, dY=dY).run()
    y, dx = many.Y.host(), many.dX.host()
    for a, b in ((5, 6), (100, 133), (300, 500), (1000, 2000)):
        few = Layer("f32", b - a, k, n, X=X[a:b], W=W, dY=dY[a:b]).run()
        assert np.array_equal(y[a:b], few.Y.host()) and np.array_equal(dx[a:b], few.dX.host()), (a, b)
