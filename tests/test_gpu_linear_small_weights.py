"""GPU: bf16 gradients of narrow layers with many rows, whose dW has few elements, against float64.

Tolerances as in test_gpu_linear.py.  For dW g is two bf16 numbers, off by at most 2^-16 of g; for dX it is rounded once."""
import math

import pytest
import torch

import linear_reference as ref
from test_gpu_linear import V, _backward, _make, _saved, _u, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,mul", [("silu", True), ("none", True), ("gelu_erf", False)])
@pytest.mark.parametrize("T,d_in,d_out,E", [(2051, 8, 8, 0), (4096, 8, 16, 0), (4096, 64, 64, 0), (4100, 1000, 8, 0), (65536, 8, 8, 0), (9000, 64, 128, 0),
                                            (4096, 32, 24, 9), (20000, 8, 64, 16), (3000, 16, 8, 40)])
def test_small_weights_keep_more_of_g(gpu_device, T, d_in, d_out, E, act, mul):
    p = _make(T, d_in, d_out, "bf16", E=E, tail=7 if E else 0, mul=mul)
    pre, dout = _saved(p, "bf16")
    want = ref.linear_grad(dout, p["X"], p["W"], p["offsets"], act, pre, p["mul"])
    longest = max(hi - lo for _, lo, hi in ref.spans(T, p["offsets"]))
    u, first = _u(torch.bfloat16), {}
    for names in (("dX", "dW", "dbias"), ("dW",), ("dX",)):
        got = _backward(p, act, pre, "bf16", names=names, dout=dout)
        for name, K, g_off in (("dX", d_out, u), ("dW", longest, 2.0 ** -16 + 8 * V)):
            if name in got:
                value, A, R = want[name]
                tol = u * value.abs() + (g_off + 4 * math.sqrt(2 * K) * V) * A + (2.0 ** -20 * R if act != "none" else 0)
                _within(got[name].reshape(value.shape), value, tol, f"{name} of {T} x {d_in} -> {d_out}, {E} experts")
    if p["W"].numel() < 2048:
        return
    # In the whole: an element differs from the formula's value rounded once where that lies within its error e of a border, by
    # one step, at most 2^-7 of the value v: the squares of the differences add up to 2 |e| 2^-7 |v| each in the mean, in all at most
    # 2^-6 ||e|| ||v||; two steps of elements of four times the root mean square v cover the chance of it.  g's second rounding and the f32 sums are of
    # either sign, so ||e|| is at most 2^-16 and sqrt(2 K) v of the root of the terms' squares.  (g in one part: 0.0026 of ||v||.)
    dW, value = _backward(p, act, pre, "bf16", names=("dW",), dout=dout)["dW"].double(), want["dW"][0]
    squares = torch.stack([(want["g"][lo:hi] ** 2).t().contiguous() @ p["X"][lo:hi].double() ** 2 for _, lo, hi in ref.spans(T, p["offsets"])])
    v2 = float((value ** 2).sum())
    e = (2.0 ** -16 + math.sqrt(2 * longest) * V) * math.sqrt(float(squares.sum())) + (2.0 ** -20 * float(torch.linalg.vector_norm(want["dW"][2])) if act != "none" else 0)
    most = 2.0 ** -6 * e * math.sqrt(v2) + 2 * (2.0 ** -7 * 4) ** 2 * v2 / value.numel()
    assert float(((dW - value.to(torch.bfloat16).double()) ** 2).sum()) <= most
