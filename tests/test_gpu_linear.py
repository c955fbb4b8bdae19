"""GPU parity: dass_linear and dass_linear_backward against float64.

Tolerances, derived from the arithmetic.  u = 2^-8 (bf16) or 2^-24 (f32) is half a step of the stored type, v = 2^-24 that of
the f32 sums.  With A the sum of a product's |terms|, K its length:
  sums      K f32 roundings of partial sums, each at most v A, that add like a random walk: sqrt(K) v A; a factor of
            4 covers the extremes of a few million of them (K v A is the worst case that never comes)
  act       its value is off by less than 2^-21 |pre| (the hardware's exponential and reciprocal, the rational erf: 2e-7),
            its slope by 2^-20, and it passes the error of pre on with a slope of at most 1.13
  rounding  u of the value for each output, and u of every term of dX and dW for g, which is rounded to bf16
            where there is an activation or mul (in f32 g carries a few v of its own: 8 v covers them)
These are worst cases but for the random walk.  Where the rounding of the output is all there is, the error over u |value| is
uniform in [0, 1 / m] for a significand m in [1, 2): in the mean 0.5 E[1 / m], between 0.5 ln 2 = 0.35 (m uniform) and
0.5 / (2 ln 2) = 0.36 (its logarithm uniform).  Every other term only widens the bound, so the mean is asked to stay
below 0.45; a systematic error (a lost slab of k, a wrong row) is near 1 or beyond everywhere.
"""
import math

import pytest
import torch

import paper_2405_01943_amd as dass

import linear_reference as ref
from gpu_helpers import padded

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
V = 2.0 ** -24


def _u(dt):
    return torch.finfo(dt).eps / 2


def _within(got, want, tol, what):
    keep = ~torch.isnan(want)
    e = (got.double() - want).abs()[keep] / (tol[keep] + 1e-300)
    worst = float(e.max()) if e.numel() else 0.0
    assert worst <= 1.0, f"{what}: worst error / tolerance = {worst:.3f}"
    if e.numel() > 1000:
        assert float(e.mean()) < 0.45, what


def _offsets(T, E, gen, tail):
    """E ragged experts over the first T - tail rows, some of them empty."""
    cuts = torch.sort(torch.randint(0, T - tail + 1, (E - 1,), generator=gen)).values if E > 1 else torch.empty(0, dtype=torch.int64)
    return torch.cat([torch.tensor([0]), cuts, torch.tensor([T - tail])]).to(torch.int32)


def _make(T, d_in, d_out, dtype, E=0, tail=0, pad=0, seed=0, bias=True, mul=True, residual=True):
    g = torch.Generator().manual_seed(seed + 31 * T + 7 * d_in + d_out)
    dt = DT[dtype]

    def rnd(*shape, std=1.0):
        t = (torch.randn(shape, generator=g) * std).to(dt).cuda()
        return padded(t, pad) if pad and t.dim() == 2 else t

    W = rnd(max(E, 1) * d_out, d_in, std=1.0 / math.sqrt(d_in))
    if E:
        W = W.unflatten(0, (E, d_out))
    p = {"X": rnd(T, d_in), "W": W, "bias": None, "mul": rnd(T, d_out) if mul else None,
         "residual": rnd(T, d_out) if residual else None,
         "offsets": _offsets(T, E, g, tail).cuda() if E else None}
    if bias:
        p["bias"] = rnd(E * d_out).reshape(E, d_out).contiguous() if E else rnd(d_out)
    return p


def _blank(T, n, dtype, pad=0):
    t = torch.full((T, n), 3.0, dtype=DT[dtype], device="cuda")
    return padded(t, pad) if pad else t


def _forward(p, act, dtype, pad=0, keep=True):
    T, d_out = p["X"].shape[0], p["W"].shape[-2]
    out, pre = _blank(T, d_out, dtype, pad), _blank(T, d_out, dtype, pad) if keep else None
    dass.linear(p["X"], p["W"], out, act=act, bias=p["bias"], mul=p["mul"], residual=p["residual"], pre_out=pre,
                offsets=p["offsets"])
    torch.cuda.synchronize()
    return out, pre


def _check_forward(p, act, out, pre, dtype, what):
    dt, K = DT[dtype], p["X"].shape[1]
    want_pre, want, A = ref.linear(p["X"], p["W"], p["offsets"], p["bias"], act, p["mul"], p["residual"])
    sums = 4 * math.sqrt(K) * V * A
    m = p["mul"].double().abs() if p["mul"] is not None else torch.ones_like(A)
    terms = m * (ref.act(want_pre, act).abs() + 1) + (p["residual"].double().abs() if p["residual"] is not None else 0)
    tol = _u(dt) * want.abs() + 1.14 * m * sums + (m * 2.0 ** -21 * want_pre.abs() if act != "none" else 0) + 4 * V * terms
    _within(out, want, tol, what)
    if pre is not None:
        _within(pre, want_pre, _u(dt) * want_pre.abs() + 1.01 * sums, what + " pre")
    rows = torch.isnan(want[:, 0])
    assert torch.all(out[rows] == 3.0) and (pre is None or torch.all(pre[rows] == 3.0)), "rows of no expert"


# one row to a few hundred, odd ones; row lengths that are no multiples of a tile or a slab
SIZES = [(1, 64, 64), (1, 4096, 264), (2, 8, 8), (7, 1000, 72), (16, 264, 1000), (17, 520, 136), (33, 72, 520), (64, 2048, 96),
         (65, 328, 264), (130, 192, 320), (300, 256, 688), (513, 136, 264), (1030, 576, 520)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d_in,d_out", SIZES)
def test_linear_sizes(gpu_device, T, d_in, d_out, dtype):
    p = _make(T, d_in, d_out, dtype)
    out, pre = _forward(p, "silu", dtype)
    _check_forward(p, "silu", out, pre, dtype, f"{T} x {d_in} -> {d_out}")


# Larger grids: together, and with SIZES, they take every kernel: in bf16 the tiles of 256 x 256, 128 x 256 and 128 x 128, k whole
# and split (2 to 16 shares), and the short 128 x 128, in f32 the tiles, whole and split, and both sizes of blocks, for the
# product and both gradients
LARGE = [("bf16", 4224, 136, 4104, 0), ("bf16", 4100, 2056, 2056, 0), ("bf16", 2050, 264, 2056, 0), ("bf16", 5000, 264, 8200, 0),
         ("bf16", 8200, 520, 1032, 0), ("bf16", 4096, 1032, 4104, 0), ("bf16", 130, 4104, 1032, 0), ("bf16", 9000, 264, 4104, 5),
         ("bf16", 9000, 4104, 264, 5), ("bf16", 12000, 136, 264, 3), ("bf16", 700, 2056, 264, 5), ("f32", 4100, 264, 1032, 0),
         ("f32", 4100, 1032, 264, 0), ("f32", 9000, 132, 132, 0), ("f32", 9000, 132, 260, 3),
         ("bf16", 2050, 4104, 2056, 0), ("bf16", 4100, 4104, 136, 0), ("bf16", 1000, 72, 4104, 3), ("bf16", 520, 4104, 4104, 0),
         ("f32", 4096, 264, 1000, 0), ("f32", 4096, 1000, 264, 0), ("f32", 260, 1000, 4096, 0), ("f32", 1000, 6152, 1000, 0),
         ("f32", 1000, 1000, 6152, 0), ("f32", 6152, 1000, 1000, 0)]


@pytest.mark.parametrize("dtype,T,d_in,d_out,E", LARGE)
def test_linear_large(gpu_device, dtype, T, d_in, d_out, E):
    p = _make(T, d_in, d_out, dtype, E=E, tail=31 if E else 0)
    out, pre = _forward(p, "silu", dtype)
    _check_forward(p, "silu", out, pre, dtype, f"{T} x {d_in} -> {d_out}")


@pytest.mark.parametrize("dtype,T,d_in,d_out,E", LARGE)
def test_linear_backward_large(gpu_device, dtype, T, d_in, d_out, E):
    p = _make(T, d_in, d_out, dtype, E=E, tail=31 if E else 0)
    pre, dout = _saved(p, dtype)
    got = _backward(p, "silu", pre, dtype, dout=dout)
    _check_backward(p, "silu", pre, dout, got, dtype, f"{T} x {d_in} -> {d_out}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("bias,mul,residual,keep", [(0, 0, 0, 0), (1, 0, 0, 1), (0, 1, 0, 0), (0, 0, 1, 0), (1, 1, 1, 1)])
@pytest.mark.parametrize("T", [5, 200])
def test_linear_epilogues(gpu_device, T, act, bias, mul, residual, keep, dtype):
    p = _make(T, 200, 144, dtype, bias=bias, mul=mul, residual=residual, pad=8)
    out, pre = _forward(p, act, dtype, pad=8, keep=keep)
    _check_forward(p, act, out, pre, dtype, act)
    for t in (out, pre):
        if t is not None:
            assert torch.all(t._base[:, 144:] == 7.0)   # nothing written past a row's end


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,tail", [(1, 8, 0), (2, 2, 1), (16, 8, 0), (40, 3, 5), (129, 5, 0), (260, 1, 3), (400, 70, 9), (1500, 6, 77)])
def test_linear_by_expert(gpu_device, T, E, tail, dtype):
    p = _make(T, 136, 200, dtype, E=E, tail=tail, seed=E)
    out, pre = _forward(p, "gelu_tanh", dtype)
    _check_forward(p, "gelu_tanh", out, pre, dtype, f"{T} rows, {E} experts")


def test_linear_many_experts(gpu_device):
    p = _make(700, 64, 64, "bf16", E=1000, tail=3)
    out, pre = _forward(p, "none", "bf16")
    _check_forward(p, "none", out, pre, "bf16", "1000 experts")


def test_linear_in_place(gpu_device):
    """out may be the residual or the other branch itself."""
    for T in (3, 150):
        p = _make(T, 128, 192, "bf16")
        out, _ = _forward(p, "silu", "bf16", keep=False)
        for name in ("residual", "mul"):
            q = dict(p, **{name: p[name].clone()})
            dass.linear(q["X"], q["W"], q[name], act="silu", bias=q["bias"], mul=q["mul"], residual=q["residual"])
            assert torch.equal(q[name].view(torch.int16), out.view(torch.int16)), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linear_large_values(gpu_device, dtype):
    """Pre-activations far out on both sides: the activations are 0 or the value itself, never NaN."""
    for act in ref.ACTS:
        p = _make(40, 64, 64, dtype, mul=False, residual=False)
        p["X"] *= 1e12
        out, pre = _forward(p, act, dtype)
        assert bool(torch.isfinite(out.float()).all()), act
        _check_forward(p, act, out, pre, dtype, act)
        grads = _backward(p, act, pre, dtype, names=("dX", "dW"), dout=torch.ones_like(out))
        assert all(bool(torch.isfinite(t.float()).all()) for t in grads.values()), act


# -------------------------------------------------------------------- gradients --
def _backward(p, act, pre, dtype, names=("dX", "dW", "dbias", "dmul"), dout=None, pad=0):
    T, d_in, d_out = p["X"].shape[0], p["X"].shape[1], p["W"].shape[-2]
    E = p["W"].shape[0] if p["offsets"] is not None else 0
    g = {}
    if "dX" in names:
        g["dX"] = _blank(T, d_in, dtype, pad)
    if "dW" in names:
        g["dW"] = _blank(max(E, 1) * d_out, d_in, dtype, pad)
        if E:
            g["dW"] = g["dW"].unflatten(0, (E, d_out))
    if "dbias" in names:
        g["dbias"] = torch.full((E, d_out) if E else (d_out,), 3.0, dtype=DT[dtype], device="cuda")
    if "dmul" in names and p["mul"] is not None:
        g["dmul"] = _blank(T, d_out, dtype, pad)
    dass.linear_backward(dout, p["X"], p["W"], act=act, pre=pre, mul=p["mul"], offsets=p["offsets"], **g)
    torch.cuda.synchronize()
    return g


def _check_backward(p, act, pre, dout, got, dtype, what):
    dt = DT[dtype]
    T, d_out = dout.shape
    want = ref.linear_grad(dout, p["X"], p["W"], p["offsets"], act, pre, p["mul"])
    rounded = act != "none" or p["mul"] is not None
    g_off = (_u(dt) if dt == torch.bfloat16 else 8 * V) if rounded else 0.0
    longest = max(hi - lo for _, lo, hi in ref.spans(T, p["offsets"]))
    for name, K in (("dX", d_out), ("dW", longest), ("dbias", longest)):
        if name not in got:
            continue
        value, A, R = want[name]
        walk = 4 * math.sqrt(max(K, 1)) * V
        keep_g = (4 * V if name == "dbias" else g_off) if rounded else 0.0
        tol = _u(dt) * value.abs() + (keep_g + walk) * A + (2.0 ** -20 * R if act != "none" else 0)
        _within(got[name].reshape(value.shape), value, tol, f"{what} {name}")
        rows = torch.isnan(value[:, 0]) if name == "dX" else None
        if rows is not None:
            assert torch.all(got[name][rows] == 3.0), "rows of no expert"
    if "dmul" in got:
        inside = torch.zeros(T, dtype=torch.bool, device=dout.device)
        for _, lo, hi in ref.spans(T, p["offsets"]):
            inside[lo:hi] = True
        w = torch.where(inside[:, None], want["dmul"], math.nan)
        tol = _u(dt) * w.abs() + dout.double().abs() * (2.0 ** -21 * pre.double().abs() + 1e-37) + 2 * V * w.abs()
        _within(got["dmul"], w, tol, f"{what} dmul")
        assert torch.all(got["dmul"][~inside] == 3.0), "rows of no expert"


def _saved(p, dtype, seed=5):
    """A pre-activation and an output gradient as a training step has them."""
    g = torch.Generator().manual_seed(seed)
    shape = (p["X"].shape[0], p["W"].shape[-2])
    return ((torch.randn(shape, generator=g) * 1.5).to(DT[dtype]).cuda(), (torch.randn(shape, generator=g) * 0.1).to(DT[dtype]).cuda())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d_in,d_out", SIZES + [(2100, 264, 328)])
def test_linear_backward_sizes(gpu_device, T, d_in, d_out, dtype):
    p = _make(T, d_in, d_out, dtype)
    pre, dout = _saved(p, dtype)
    got = _backward(p, "silu", pre, dtype, dout=dout)
    _check_backward(p, "silu", pre, dout, got, dtype, f"{T} x {d_in} -> {d_out}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("mul", [False, True])
def test_linear_backward_epilogues(gpu_device, act, mul, dtype):
    p = _make(150, 200, 144, dtype, mul=mul, pad=8)
    pre, dout = _saved(p, dtype)
    got = _backward(p, act, pre, dtype, dout=dout, pad=8)
    _check_backward(p, act, pre, dout, got, dtype, act)
    assert torch.all(got["dX"]._base[:, 200:] == 7.0) and torch.all(got["dW"]._base[:, 200:] == 7.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,tail", [(1, 8, 0), (2, 2, 1), (16, 8, 0), (129, 5, 0), (260, 1, 3), (400, 70, 9), (1500, 6, 77)])
def test_linear_backward_by_expert(gpu_device, T, E, tail, dtype):
    p = _make(T, 136, 200, dtype, E=E, tail=tail, seed=E)
    pre, dout = _saved(p, dtype)
    got = _backward(p, "gelu_erf", pre, dtype, dout=dout)
    _check_backward(p, "gelu_erf", pre, dout, got, dtype, f"{T} rows, {E} experts")
    empty = [e for e, lo, hi in ref.spans(T, p["offsets"]) if lo == hi]
    assert torch.all(got["dW"][empty] == 0) and torch.all(got["dbias"][empty] == 0)


@pytest.mark.parametrize("dtype,T,d_in,d_out,E", LARGE[:19] + [("bf16", *size, 0) for size in SIZES])
def test_linear_backward_one_by_one(gpu_device, dtype, T, d_in, d_out, E):
    """Each product in a call of its own: both together may share a launch."""
    p = _make(T, d_in, d_out, dtype, E=E, tail=31 if E else 0)
    pre, dout = _saved(p, dtype)
    for names in (("dX",), ("dW", "dbias")):
        _check_backward(p, "silu", pre, dout, _backward(p, "silu", pre, dtype, names=names, dout=dout), dtype, f"{T} x {d_in} -> {d_out}")


@pytest.mark.parametrize("names", [("dX",), ("dW",), ("dbias",), ("dmul",), ("dX", "dbias"), ("dW", "dmul")])
def test_linear_backward_parts(gpu_device, names):
    """Each gradient alone has the bits that it has among the others."""
    p = _make(90, 136, 72, "bf16")
    pre, dout = _saved(p, "bf16")
    whole, part = (_backward(p, "silu", pre, "bf16", names=n, dout=dout) for n in (("dX", "dW", "dbias", "dmul"), names))
    assert sorted(part) == sorted(names)
    for name in names:
        assert torch.equal(part[name].view(torch.int16), whole[name].view(torch.int16)), name


@pytest.mark.parametrize("act", ref.ACTS)
def test_linear_gradients_against_differences(gpu_device, act):
    """f32 gradients against central differences of the float64 forward pass, along random directions.  A step of 1e-5
    leaves 1e-9 of the value; the kernels' own error is about 1e-6 of the sum of the terms' magnitudes."""
    p = _make(37, 40, 24, "f32", E=3, tail=2)
    g = torch.Generator().manual_seed(8)
    dout = torch.randn((37, 24), generator=g).cuda()
    _, pre = _forward(p, act, "f32")
    got = _backward(p, act, pre, "f32", dout=dout)
    rows = p["offsets"][-1].item()

    def loss(**moved):
        q = {n: (p[n].double() if p[n].dtype == torch.float32 else p[n]) for n in ("X", "W", "bias", "mul", "residual", "offsets")}
        q.update(moved)
        out = ref.linear(q["X"], q["W"], q["offsets"], q["bias"], act, q["mul"], q["residual"])[1]
        return float((out[:rows] * dout[:rows].double()).sum())

    for name, grad in (("X", "dX"), ("W", "dW"), ("bias", "dbias"), ("mul", "dmul")):
        base = p[name].double()
        step = torch.randn(base.shape, generator=g, dtype=torch.float64).cuda()
        want = (loss(**{name: base + 1e-5 * step}) - loss(**{name: base - 1e-5 * step})) / 2e-5
        terms = got[grad].double() * step
        if grad in ("dX", "dmul"):
            terms = terms[:rows]
        assert abs(float(terms.sum()) - want) <= 1e-5 * float(terms.abs().sum()) + 1e-8, name


def test_linear_repeats_bit_for_bit(gpu_device):
    p = _make(700, 520, 264, "bf16", E=5, tail=11)
    pre, dout = _saved(p, "bf16")
    first = _forward(p, "silu", "bf16"), _backward(p, "silu", pre, "bf16", dout=dout)
    again = _forward(p, "silu", "bf16"), _backward(p, "silu", pre, "bf16", dout=dout)
    for a, b in zip([*first[0], *first[1].values()], [*again[0], *again[1].values()]):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
