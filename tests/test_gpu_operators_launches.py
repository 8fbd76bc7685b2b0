"""The operators on so many rows that their work groups do not fit one launch (2^32 work items a dimension).  Tensors are filled and compared on the device in
slices; rows around the launches' ends and the last ones are compared with the definitions."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from operator_util import HALF_ULP, plan, stream, within
from oracle import operators_oracle as oo
from paper_2604_05426_amd import binding as ml

pytestmark = pytest.mark.gpu


def test_dropout():
    """2^25 + 7 rows of 1032 columns, two rows a work group of 256: 2^24 + 4 work groups; in place, a last job of a few rows."""
    T, cols, last = (1 << 25) + 7, 1032, 5
    X = torch.empty((T, cols), dtype=torch.bfloat16, device="cuda")
    X[:] = (torch.arange(cols, device="cuda") % 61 + 1).to(torch.bfloat16)
    p = plan("bf16", [0, T - last, T])
    print(f"[case] dropout T={T}", flush=True)
    ml.multi_lora_dropout(p, ml.Dropout([(0.25, 5), (0.5, 6)]), cols, X, X, counter=9, stream=stream())
    torch.cuda.synchronize()
    row = (np.arange(cols) % 61 + 1).astype(float)
    for first in (0, 1 << 23, (1 << 24) - 2, 1 << 24, 1 << 25, T - last - 3):
        n = min(4, T - last - first)
        words = oo.philox([np.tile(np.arange(cols // 8), n), np.repeat(np.arange(first, first + n), cols // 8), np.full(n * cols // 8, 9), np.zeros(n * cols // 8)], [5, 0])
        numbers = np.stack([(words[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF) for j in range(8)], axis=-1).reshape(n, cols)
        want = np.where(numbers >= oo.threshold(0.25), row * (4 / 3), 0.0)
        within(X[first:first + n].double().cpu().numpy(), want, HALF_ULP["bf16"] * np.abs(want) * (1 + 2.0 ** -8) + 3 * 2.0 ** -24 * np.abs(want), first)
    want = np.where(oo.keep_mask(last, cols, 0.5, 6, 9), 2.0 * row, 0.0)
    assert np.array_equal(X[T - last:].double().cpu().numpy(), want)
    # every row has been worked on: none kept all of its columns
    whole = 0
    for part in X.split(1 << 22):
        whole += int((part != 0).all(1).sum())
    assert whole == 0
    p.destroy()


@pytest.mark.parametrize("d", [1, 8])
def test_edge(d):
    """2^29 + 5 rows, eight a work group of 64 would be 2^26 + 1 work groups."""
    T, last = (1 << 29) + 5, 3
    line = (torch.arange(1 << 20, device="cuda") % 253 - 126).to(torch.bfloat16)
    h, dx = (torch.empty((T, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t, flip in ((h, 1), (dx, -1)):
        flat = t.view(-1)
        for at in range(0, T * d, 1 << 20):
            piece = flat[at:at + (1 << 20)]
            piece.copy_(line[:len(piece)] if flip > 0 else line.flip(0)[:len(piece)])
    gain = torch.linspace(0.5, 1.5, 2 * d, device="cuda").to(torch.bfloat16).view(2, d)
    x, dh = torch.full((T, d), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, d), 9.0, dtype=torch.bfloat16, device="cuda")
    stats = torch.empty((2, T), device="cuda")
    e = ml.Edge(d, pre_gain=gain, pre_ld=d, pre_eps=0.5)
    p = plan("bf16", [0, T - last, T])
    print(f"[case] edge T={T} d={d}", flush=True)
    ml.multi_lora_edge_fwd(p, e, h, None, None, x, stats, stream())
    ml.multi_lora_edge_bwd(p, e, h, None, stats, dx, None, dh, None, None, stream=stream())
    torch.cuda.synchronize()
    f = lambda t: t.double().cpu().numpy()
    for first in (0, 1 << 22, (1 << 25) - 5, 1 << 28, (1 << 29) - 500, T - last - 9, T - last):
        rows = slice(first, min(first + 1000, T if first == T - last else T - last))
        g = f(gain[1 if first == T - last else 0])
        a, b = f(h[rows]), f(dx[rows])
        r = 1 / np.sqrt((a ** 2).mean(1, keepdims=True) + 0.5)
        want = a * r * g
        within(f(x[rows]), want, HALF_ULP["bf16"] * np.abs(want) * 1.01 + 2.0 ** -18 * np.abs(want), (first, "x"))
        m = (g * b * a * r).mean(1, keepdims=True)
        want = r * (g * b - a * r * m)
        mag = r * (np.abs(g * b) + np.abs(a * r) * (np.abs(g * b * a * r)).mean(1, keepdims=True))
        within(f(dh[rows]), want, HALF_ULP["bf16"] * np.abs(want) * 1.01 + 2.0 ** -18 * mag, (first, "dh"))
    assert not any(bool((part == 9.0).any()) for part in x.split(1 << 26))          # written everywhere (|x| is below 1.5 sqrt(d))
    assert bool(torch.isfinite(stats[1]).all())
    p.destroy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quant(dtype):
    """2^27 + 100 rows, eight a work group of 256 as they are rounded: 2^24 + 13 work groups.  Operands -2 .. 2: every sum is exact."""
    T, k, n = (1 << 27) + 100, 8, 4
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(1)
    units = lambda *shape: torch.randint(-2, 3, shape, generator=gen, device="cuda", dtype=torch.int8).to(dt)
    X, dY, W = units(T, k), units(T, n), units(k, n)
    kind = ml.BF16 if dtype == "bf16" else ml.F32
    p = ml.Plan(kind, T, k, n, [], [], [0], stream=stream())
    w8 = torch.empty(ml.multi_lora_quant_bytes(k, n), dtype=torch.uint8, device="cuda")
    ws = torch.empty(ml.multi_lora_quant_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    Y, dX = torch.full((T, n), 99.0, dtype=dt, device="cuda"), torch.full((T, k), 99.0, dtype=dt, device="cuda")
    print(f"[case] 8-bit products T={T} {dtype}", flush=True)
    ml.multi_lora_quant_weight(kind, k, n, W, w8, stream())
    ml.multi_lora_quant_fwd(p, X, w8, Y, ws, stream())
    ml.multi_lora_quant_bwd(p, dY, w8, dX, ws, stream())
    torch.cuda.synchronize()
    w = W.float()
    for a, b, c, d in zip(X.split(1 << 24), Y.split(1 << 24), dY.split(1 << 24), dX.split(1 << 24)):
        assert torch.equal(b.float(), sum(a[:, i:i + 1].float() * w[i] for i in range(k)))
        assert torch.equal(d.float(), sum(c[:, i:i + 1].float() * w[:, i] for i in range(n)))
    p.destroy()
