"""Margins and losses of sequences of thousands of rows: a small difference of large sums, which keeps whatever every row is off by in the same direction.

Tolerance: a row's log-probability is off by the rounding of its sum of exponentials, whose error is without direction and below 2^-23 (rms), and by what the
exponential is off by on average, below 2^-27.  Over the rows of a pair the first adds up with the square root of their number (six times that
here), the second with the difference of the two sequences' rows."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from operator_util import DT, ML, stream, within
from paper_2604_05426_amd import binding as ml

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1601, 3301, 33000])
@pytest.mark.parametrize("chosen,rejected", [(8200, 7100), (15000, 900), (900, 15000)])
def test_margin_and_loss(dtype, V, chosen, rejected):
    scale = 1 if V < 20000 else 4
    chosen, rejected = chosen // scale, rejected // scale
    T, beta = chosen + rejected, 0.5
    gen = torch.Generator(device="cuda").manual_seed(V + chosen)
    z = (torch.randn((T, V), generator=gen, device="cuda") * 2.0).to(DT[dtype])
    targets = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    rows = torch.arange(T, device="cuda")
    z[rows, targets.long()] = (z[rows, targets.long()].float() + 8.0 + torch.randn(T, generator=gen, device="cuda")).to(DT[dtype])
    row = torch.cat([torch.log_softmax(p.double(), 1).gather(1, t[:, None])[:, 0] for p, t in zip(z.split(1024), targets.long().split(1024))]).cpu().numpy()
    logp = np.array([row[:chosen].sum(), row[chosen:].sum()])
    ref = (logp + [2.0, -1.5]).astype(np.float32).astype(np.float64)
    pref = ml.Preference(ML[dtype], T, V, [0], [0, chosen, T], [(beta, 0.1, 0.0)], stream())
    ws = torch.empty(pref.workspace_bytes(), dtype=torch.uint8, device="cuda")
    out = {k: torch.full((n,), float("nan"), device="cuda") for k, n in (("logp", 2), ("margin", 1), ("loss", 1), ("row", T))}
    ml.multi_lora_pref_fwd(pref, z, V, targets, torch.from_numpy(ref.astype(np.float32)).cuda(), out["logp"], out["margin"], out["loss"], ws, stream())
    margin = beta * ((logp[0] - ref[0]) - (logp[1] - ref[1]))
    pair = 6 * 2.0 ** -23 * np.sqrt(T) + 2.0 ** -27 * abs(chosen - rejected)
    loss = 0.9 * np.logaddexp(0, -margin) + 0.1 * np.logaddexp(0, margin)
    within(out["margin"].cpu().numpy(), margin, beta * pair + 2.0 ** -24 * abs(margin), "margin")
    within(out["loss"].cpu().numpy(), loss, beta * pair + 2.0 ** -23 * abs(loss), "loss")
    within(out["logp"].cpu().numpy(), logp, 2.0 ** -24 * np.abs(logp) + 6 * 2.0 ** -23 * np.sqrt(T) + 2.0 ** -27 * T, "logp")
    ml.multi_lora_pref_logp(pref, z, V, targets, out["logp"], ws, row_logp=out["row"], stream=stream())
    within(out["row"].cpu().numpy(), row, 8 * 2.0 ** -23 + 2.0 ** -24 * np.abs(row), "row_logp")
