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
