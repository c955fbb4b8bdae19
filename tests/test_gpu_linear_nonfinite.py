"""GPU: NaN and infinities in the operands of dass_linear and its gradient appear where the formulas have them, and nowhere else."""
import math

import pytest
import torch

import linear_reference as ref
from test_gpu_linear import _backward, _forward, _make, _saved

pytestmark = pytest.mark.gpu

# few rows, small f32 blocks, tiles, split k, both products in one launch and not; dense and by expert
SIZES = [(3, 128, 136, 0), (40, 136, 200, 3), (150, 200, 144, 0), (700, 2056, 264, 5), (1030, 576, 520, 0), (1500, 136, 200, 6)]


def _at(T, offsets, row):
    """The expert of a row."""
    return next(e for e, lo, hi in ref.spans(T, offsets) if lo <= row < hi)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("T,d_in,d_out,E", SIZES)
def test_nan_passes_every_activation(gpu_device, T, d_in, d_out, E, act, dtype):
    """A NaN in X is NaN in the whole row of pre and out; a NaN in pre is NaN in dX's row, in dW's row and in dbias, and in dmul."""
    p = _make(T, d_in, d_out, dtype, E=E)
    clean, clean_pre = _forward(p, act, dtype)
    row, col = T - 2, d_out - 3
    q = dict(p, X=p["X"].clone())
    q["X"][row, 5] = math.nan
    others = torch.arange(T, device="cuda") != row
    for got, want in zip(_forward(q, act, dtype), (clean, clean_pre)):
        assert bool(got[row].isnan().all()) and torch.equal(got[others], want[others])
    if act == "none":
        return
    pre, dout = _saved(p, dtype)
    clean = _backward(p, act, pre, dtype, dout=dout)
    pre[row, col] = math.nan
    got = _backward(p, act, pre, dtype, dout=dout)
    e = _at(T, p["offsets"], row)
    dW, dbias = (got["dW"][e], got["dbias"][e]) if E else (got["dW"], got["dbias"])
    assert bool(got["dX"][row].isnan().all()) and bool(dW[col].isnan().all()) and bool(dbias[col].isnan()) and bool(got["dmul"][row, col].isnan())
    for name, t in got.items():     # and in nothing else
        n = {"dX": d_in, "dW": d_in, "dbias": 1, "dmul": 1}[name]
        assert int(t.isnan().sum()) == n, name
        keep = ~t.isnan()
        assert torch.equal(t[keep], clean[name][keep]), name
