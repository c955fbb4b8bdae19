"""The linear layer with its epilogue, its gradients, and the sort of tokens by expert, in float64 from their formulas
(tests only; shares nothing with the library).  Beside each value stands the sum of its terms' magnitudes, from which
the tests derive their tolerances."""
import math

import torch

ACTS = ("none", "silu", "gelu_tanh", "gelu_erf", "relu")


def act(x, name):
    if name == "silu":
        return x / (1 + torch.exp(-x))
    if name == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    if name == "gelu_erf":
        return 0.5 * x * torch.special.erfc(-x / math.sqrt(2))
    return torch.clamp(x, min=0) if name == "relu" else x


def slope(x, name):
    if name == "silu":
        s = 1 / (1 + torch.exp(-x))
        return s + x * s * (1 - s)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        th = torch.tanh(c * (x + 0.044715 * x ** 3))
        return 0.5 * (1 + th) + 0.5 * x * (1 - th ** 2) * c * (1 + 3 * 0.044715 * x ** 2)
    if name == "gelu_erf":
        return 0.5 * torch.special.erfc(-x / math.sqrt(2)) + x * torch.exp(-x ** 2 / 2) / math.sqrt(2 * math.pi)
    return (x > 0).to(x.dtype) if name == "relu" else torch.ones_like(x)


def spans(T, offsets):
    """(expert, lo, hi) of the rows of each expert; one span of all rows without offsets."""
    if offsets is None:
        return [(0, 0, T)]
    o = [int(v) for v in offsets.cpu()]
    return [(e, o[e], o[e + 1]) for e in range(len(o) - 1)]


def _mm(a, b):
    return torch.matmul(a, b.contiguous())


def linear(X, W, offsets=None, bias=None, act_name="none", mul=None, residual=None):
    """(pre, out, sum of |x w| + |bias|) for the rows of experts; NaN elsewhere."""
    T, d_out = X.shape[0], W.shape[-2]
    stack = (W if offsets is not None else W[None]).double()
    pre = torch.full((T, d_out), math.nan, dtype=torch.float64, device=X.device)
    size = torch.full_like(pre, math.nan)
    for e, lo, hi in spans(T, offsets):
        x, wt = X[lo:hi].double(), stack[e].t()
        pre[lo:hi], size[lo:hi] = _mm(x, wt), _mm(x.abs(), wt.abs())
        if bias is not None:
            b = bias.reshape(len(stack), d_out)[e].double()
            pre[lo:hi] += b
            size[lo:hi] += b.abs()
    out = act(pre, act_name)
    if mul is not None:
        out = out * mul.double()
    if residual is not None:
        out = out + residual.double()
    return pre, out, size


def linear_grad(dout, X, W, offsets=None, act_name="none", pre=None, mul=None):
    """dict of g, |dout mul|, and (value, sum of |terms|, sum of |terms| with |dout mul| for g) of dX, dW, dbias; dmul."""
    T, d_out = dout.shape
    stack = (W if offsets is not None else W[None]).double()
    raw = dout.double() * (mul.double() if mul is not None else 1)
    g = raw * slope(pre.double(), act_name) if act_name != "none" else raw
    X64 = X.double()

    def dx(u, w):
        r = torch.full((T, w.shape[-1]), math.nan, dtype=torch.float64, device=u.device)
        for e, lo, hi in spans(T, offsets):
            r[lo:hi] = _mm(u[lo:hi], w[e])
        return r

    def dw(u, x):
        return torch.stack([_mm(u[lo:hi].t().contiguous(), x[lo:hi]) for _, lo, hi in spans(T, offsets)])

    def db(u):
        return torch.stack([u[lo:hi].sum(0) for _, lo, hi in spans(T, offsets)])

    a, r = g.abs(), raw.abs()
    return {"g": g, "raw": r,
            "dX": (dx(g, stack), dx(a, stack.abs()), dx(r, stack.abs())),
            "dW": tuple(t.reshape(W.shape) for t in (dw(g, X64), dw(a, X64.abs()), dw(r, X64.abs()))),
            "dbias": (db(g), db(a), db(r)),
            "dmul": None if pre is None else dout.double() * act(pre.double(), act_name)}


def sort(ids, E):
    """(offsets, order, place) by a plain loop over the pairs."""
    flat = [int(v) for v in ids.reshape(-1).cpu()]
    order, place, offsets = [-1] * len(flat), [-1] * len(flat), [0]
    row = 0
    for e in range(E):
        for pair, v in enumerate(flat):
            if v == e:
                order[row], place[pair] = pair, row
                row += 1
        offsets.append(row)
    as_int = lambda v: torch.tensor(v, dtype=torch.int32)
    return as_int(offsets), as_int(order), as_int(place).reshape(ids.shape)
