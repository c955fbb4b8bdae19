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


def _kind(t):
    """0: finite, 1 and -1: the infinities, 2: NaN."""
    return torch.where(t.isnan(), 2.0, torch.where(t.isinf(), t.sign(), torch.zeros_like(t))).to(torch.int8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "none"])
@pytest.mark.parametrize("T,d_in,d_out,E", SIZES + [(1, 64, 72, 0), (4, 1000, 4096, 0), (2048, 72, 8, 0), (250, 1032, 64, 9), (4096, 16, 8, 0), (4099, 64, 72, 0),
                                                     (5000, 16, 24, 5)])
def test_infinities_in_gradients(gpu_device, T, d_in, d_out, E, act, dtype):
    """Infinite elements of W, X and dout, one or two of either sign in a sum, meet g whatever parts it is kept in; with act
    none the powers of 2 in mul leave g a bf16 number, whose second part would be 0."""
    for seed, where in enumerate(("W", "X", "dout", "all")):
        p = _make(T, d_in, d_out, dtype, E=E, seed=seed)
        pre, dout = _saved(p, dtype)
        p["mul"] = torch.exp2(torch.randint(-3, 3, dout.shape, device="cuda").float()).to(dout.dtype)
        row = T - 1
        e = _at(T, p["offsets"], row)
        W = p["W"][e] if E else p["W"]
        if where in ("W", "all"):
            W[5, 7], W[1, 9], W[6, 9] = math.inf, -math.inf, math.inf
        if where in ("X", "all"):
            p["X"][row, 11] = -math.inf
            p["X"][max(0, T - 3), 3] = p["X"][row, 3] = math.inf
        if where in ("dout", "all"):
            dout[row, 2] = -math.inf
        got = _backward(p, act, pre, dtype, names=("dX", "dW", "dbias"), dout=dout)
        want = ref.linear_grad(dout, p["X"], p["W"], p["offsets"], act, pre, p["mul"])
        for name, t in got.items():
            value = want[name][0].reshape(t.shape)
            if (name, where) in (("dX", "W"), ("dW", "X")) or where in ("dout", "all"):
                assert not bool(value.isfinite().all()), "the case has an infinity"
            assert torch.equal(_kind(t.double()), _kind(value)), f"{name}, {where}"
