"""Parameter gradients of block edges over many adapters, some of them without rows."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2604_05426_amd import binding as ml
from test_gpu_edge import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate", ["shared", "adapter"])
def test_shared_gains_of_more_adapters_than_a_work_group_has_threads(dtype, gate):
    """Gains (and a gate) that 300 adapters share: their sums in two rounds of 256."""
    rng = np.random.default_rng(7)
    Case(dtype, [int(x) for x in rng.integers(0, 4, 299)] + [5], 72, gains="shared", gate=gate).run()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gains,gate", [("shared", "shared"), ("shared", "adapter"), ("adapter", "shared")])
def test_accumulates_into_shared_gradients(dtype, gains, gate):
    c = Case(dtype, [60, 0, 3, 50], 136, gains=gains, gate=gate).run()
    c.backward(flags=ml.FLAG_ACCUM_GRADS, fill=3.0)
    c.check_backward(base=3.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("flags", [0, ml.FLAG_ACCUM_GRADS])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_gradients_of_adapters_without_rows_whatever_their_parameters(dtype, flags, bad):
    """An adapter without rows has gradients of zero (added to what is there, with the flag) also where its gate, gain or scale is not finite."""
    c = Case(dtype, [20, 0, 7, 0], 80, gains="adapter")
    c.dev["gate"][1, 3] = bad
    c.dev["post"][3, 5] = bad
    c.dev["scale"][3] = bad
    c.forward()
    c.backward(flags=flags, fill=3.0 if flags else float("nan"))
    for name, out in c.g.items():
        got = out.host()
        got = got.T if name == "d_scale" else got
        assert np.all(got[[1, 3]] == (3.0 if flags else 0.0)), name
        assert np.isfinite(got).all(), name
