"""GPU: what dass_linear, its gradient and the experts' rows must not touch, and matrices of more than 2^31 elements."""
import math

import pytest
import torch

import paper_2405_01943_amd as dass
from paper_2405_01943_amd import binding

import linear_reference as ref
from test_gpu_linear import DT, V, _backward, _check_backward, _check_forward, _forward, _make, _saved, _u, _within

pytestmark = pytest.mark.gpu

# grids of every kernel by expert: few rows, the four tiles, whole and split, and f32's
BY_EXPERT = [("bf16", 40, 136, 200, 3), ("bf16", 1500, 136, 200, 6), ("bf16", 9000, 264, 4104, 5), ("bf16", 9000, 4104, 264, 5),
             ("bf16", 700, 2056, 264, 5), ("bf16", 1000, 72, 4104, 3), ("bf16", 8200, 1032, 2056, 2), ("f32", 40, 136, 200, 3),
             ("f32", 1500, 132, 260, 6), ("f32", 4096, 264, 1000, 2)]


def _wide_nan(t, pad=8):
    """The same rows, with NaN between them."""
    big = torch.full((t.shape[0], t.shape[1] + pad), math.nan, dtype=t.dtype, device=t.device)
    big[:, :t.shape[1]] = t
    return big[:, :t.shape[1]]


def _all_bytes(n):
    return torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")


def _run(p, pre, dout, E):
    """Output, kept sums and all gradients, with workspaces of exactly the stated size, all bits set."""
    T, d_in, d_out, dt = p["X"].shape[0], p["X"].shape[1], p["W"].shape[-2], p["X"].dtype
    got = {n: torch.full((T, d_out), 3.0, dtype=dt, device="cuda") for n in ("out", "pre_out", "dmul")}
    got["dX"] = torch.full((T, d_in), 3.0, dtype=dt, device="cuda")
    got["dW"] = torch.full((E, d_out, d_in), 3.0, dtype=dt, device="cuda")
    got["dbias"] = torch.full((E, d_out), 3.0, dtype=dt, device="cuda")
    dass.linear(p["X"], p["W"], got["out"], act="silu", bias=p["bias"], mul=p["mul"], residual=p["residual"], pre_out=got["pre_out"],
                offsets=p["offsets"], workspace=_all_bytes(dass.linear_workspace_bytes(T, d_in, d_out, dt, E)))
    dass.linear_backward(dout, p["X"], p["W"], act="silu", pre=pre, mul=p["mul"], offsets=p["offsets"],
                         workspace=_all_bytes(dass.linear_backward_workspace_bytes(T, d_in, d_out, dt, E)),
                         **{n: got[n] for n in ("dX", "dW", "dbias", "dmul")})
    torch.cuda.synchronize()
    return got


@pytest.mark.parametrize("dtype,T,d_in,d_out,E", BY_EXPERT)
def test_rows_of_no_expert_and_gaps_are_not_read(gpu_device, dtype, T, d_in, d_out, E):
    """NaN before the first expert's rows, behind the last one's, between all rows and in the workspace changes no bit."""
    p = _make(T, d_in, d_out, dtype, E=E, tail=9)
    pre, dout = _saved(p, dtype)
    p["offsets"][0] = min(5, int(p["offsets"][1]))
    lo, hi = int(p["offsets"][0]), int(p["offsets"][-1])
    clean = _run(p, pre, dout, E)
    q = dict(p)
    for name in ("X", "mul", "residual"):
        q[name] = _wide_nan(p[name])
        q[name][:lo] = q[name][hi:] = math.nan
    bad = [_wide_nan(t) for t in (pre, dout)]
    for t in bad:
        t[:lo] = t[hi:] = math.nan
    q["W"] = _wide_nan(p["W"].reshape(E * d_out, d_in)).unflatten(0, (E, d_out))
    got = _run(q, *bad, E)
    for name, want in clean.items():
        assert torch.equal(got[name], want), name
        assert bool(torch.isfinite(want.float()).all()), name


@pytest.mark.parametrize("dtype,T,d_in,d_out,E", BY_EXPERT)
def test_an_expert_of_nan_leaves_the_others(gpu_device, dtype, T, d_in, d_out, E):
    p = _make(T, d_in, d_out, dtype, E=E)
    pre, dout = _saved(p, dtype)
    clean = _run(p, pre, dout, E)
    o = [int(v) for v in p["offsets"].cpu()]
    e = max(range(E), key=lambda x: o[x + 1] - o[x])
    p["X"][o[e]:o[e + 1]] = math.nan
    dout[o[e]:o[e + 1]] = math.inf
    p["W"][e] = math.nan
    got = _run(p, pre, dout, E)
    for name, want in clean.items():
        by_expert = name in ("dW", "dbias")
        for x in range(E):
            part = (lambda t: t[x]) if by_expert else (lambda t: t[o[x]:o[x + 1]])
            if x != e:
                assert torch.equal(part(got[name]), part(want)), name
    assert bool(torch.isnan(got["out"][o[e]:o[e + 1]].float()).all())


@pytest.mark.parametrize("bounds", [(0, 100, 50, 200), (0, 300, 300, 0), (-7, 60, 5000, 90), (50, 40, 30, 20)])
def test_strange_offsets_stay_inside(gpu_device, bounds):
    """Bounds that fall or lie outside: the call ends, writes no row outside the matrices, and the well-formed spans hold."""
    for dtype in ("bf16", "f32"):
        p = _make(200, 136, 200, dtype, E=3)
        pre, dout = _saved(p, dtype)
        p["offsets"] = torch.tensor(bounds, dtype=torch.int32, device="cuda")
        for T in (200, 16):
            part = {n: (t[:T] if n in ("X", "mul", "residual") else t) for n, t in p.items()}
            _run(part, pre[:T], dout[:T], 3)


@pytest.mark.parametrize("names", [("dX",), ("dW",), ("dbias",), ("dX", "dbias"), ("dW", "dmul"), ("dX", "dW"), ("dW", "dbias")])
@pytest.mark.parametrize("E", [0, 3])
def test_small_f32_gradients_in_any_company(gpu_device, E, names):
    """The parts of the one launch of a small f32 gradient: each alone and with others has the same bits."""
    p = _make(90, 136, 72, "f32", E=E, tail=4 if E else 0)
    pre, dout = _saved(p, "f32")
    whole, part = (_backward(p, "silu", pre, "f32", names=n, dout=dout) for n in (("dX", "dW", "dbias", "dmul"), names))
    for name in names:
        assert torch.equal(part[name].view(torch.int32), whole[name].view(torch.int32)), name


@pytest.mark.parametrize("names", [("dX", "dW"), ("dX",), ("dW",)])
@pytest.mark.parametrize("T,d_in,d_out,E", [(1, 128, 128, 0), (1, 4096, 264, 0), (2, 128, 8192, 0), (4, 1000, 4096, 0), (40, 136, 200, 3),
                                            (150, 64, 104, 0), (2048, 72, 8, 0), (250, 1032, 64, 9), (1, 2056, 14336, 5), (65, 64, 72, 0), (3, 136, 14336, 0), (33, 200, 5000, 4)])
def test_gradients_of_few_elements_keep_more_of_g(gpu_device, T, d_in, d_out, E, names):
    """Up to 16384 elements of g, or of a g with up to 8192 of dX, are two bf16 numbers: rounded twice they are off by at most 2^-8 of 2^-8."""
    p = _make(T, d_in, d_out, "bf16", E=E, tail=min(T - 1, 3) if E else 0)
    pre, dout = _saved(p, "bf16")
    got = _backward(p, "silu", pre, "bf16", names=names, dout=dout)
    want = ref.linear_grad(dout, p["X"], p["W"], p["offsets"], "silu", pre, p["mul"])
    longest = max(hi - lo for _, lo, hi in ref.spans(T, p["offsets"]))
    for name, K in (("dX", d_out), ("dW", longest)):
        if name in got:
            value, A, R = want[name]
            # the result's rounding; g's two and 4 in f32; 4 sqrt(2 K) for the sum over both parts; the slope's own error
            tol = _u(torch.bfloat16) * value.abs() + (2.0 ** -16 + 8 * V + 4 * math.sqrt(2 * K) * V) * A + 2.0 ** -20 * R
            _within(got[name].reshape(value.shape), value, tol, f"{name} of {T} x {d_in} -> {d_out}, {E} experts")


# ------------------------------------------------------- beyond 2^31 elements --
FAR = 300      # the last rows, all that is compared


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linear_of_a_long_matrix(gpu_device, dtype):
    T, d = 131072 + 77, 16392
    dt = DT[dtype]
    p = {"X": torch.randn((T, d), dtype=dt, device="cuda"), "W": (torch.randn((16, d), device="cuda") / math.sqrt(d)).to(dt), "bias": None,
         "mul": None, "residual": None, "offsets": None}
    assert p["X"].numel() > 2 ** 31
    out, _ = _forward(p, "none", dtype, keep=False)
    far = {**p, "X": p["X"][-FAR:]}
    _check_forward(far, "none", out[-FAR:], None, dtype, "the last rows")
    # all but the last rows without a gradient: dW is theirs
    dout = torch.zeros((T, 16), dtype=dt, device="cuda")
    dout[-FAR:] = torch.randn((FAR, 16), device="cuda").to(dt)
    got = _backward(p, "none", None, dtype, names=("dX", "dW"), dout=dout)
    got["dX"] = got["dX"][-FAR:].clone()
    # the zeros of the other rows add nothing, so the error is that of the last rows' sum
    _check_backward(far, "none", None, dout[-FAR:], got, dtype, "the last rows")


def test_linear_of_long_weights(gpu_device):
    E, d_out, d_in = 5, 16384, 32768
    X, W = torch.randn((40, d_in), device="cuda").bfloat16(), torch.empty((E, d_out, d_in), dtype=torch.bfloat16, device="cuda")
    assert W.numel() > 2 ** 31
    for e in range(E):
        W[e].normal_(0, 1 / math.sqrt(d_in))
    p = {"X": X, "W": W, "bias": None, "mul": None, "residual": None,
         "offsets": torch.tensor([0, 0, 2, 2, 2, 40], dtype=torch.int32, device="cuda")}
    out, _ = _forward(p, "none", "bf16", keep=False)
    dout = torch.randn((40, d_out), device="cuda").bfloat16()
    got = _backward(p, "none", None, "bf16", names=("dX", "dW"), dout=dout)
    for e, lo, hi in ((1, 0, 2), (4, 2, 40)):
        one = {**p, "X": X[lo:hi], "W": W[e], "offsets": None}
        _check_forward(one, "none", out[lo:hi], None, "bf16", f"expert {e}")
        _check_backward(one, "none", None, dout[lo:hi], {"dX": got["dX"][lo:hi], "dW": got["dW"][e]}, "bf16", f"expert {e}")
    for e in (0, 2, 3):
        assert not got["dW"][e].any()


def test_rows_beyond_31_bits(gpu_device):
    T, k, d = 70000, 4, 8192
    X = torch.randn((T, d), device="cuda").bfloat16()
    ids = torch.randint(0, 8, (T, k), device="cuda")
    offsets, order, place = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (9, T * k, T * k))
    place = place.view(T, k)
    dass.expert_sort(ids, 8, offsets, order, place)
    rows = torch.empty((T * k, d), dtype=torch.bfloat16, device="cuda")
    assert rows.numel() > 2 ** 31
    dass.expert_gather(X, place, rows)
    w = torch.rand((T, k), device="cuda")
    out = torch.empty_like(X)
    dass.expert_combine(rows, place, out, weights=w)
    dY, dw = torch.empty_like(rows), torch.empty_like(w)
    dass.expert_combine_backward(X, rows, place, w, dY, dw)
    some = torch.cat([torch.randint(0, T, (500,), device="cuda"), (order[-200:] // k).long()])    # among them the owners of the last rows
    for j in range(k):
        at = place[some, j].long()
        assert torch.equal(rows[at], X[some])
        assert torch.equal(dY[at], (w[some, j, None] * X[some].float()).bfloat16())
    want = (w[some].double().sum(1, keepdim=True)) * X[some].double()
    # k products and sums in f32, rounded once: each off by half a step of a sum that is no larger than the result
    assert bool(((out[some].double() - want).abs() <= (_u(torch.bfloat16) + 2 * k * 2.0 ** -24) * want.abs()).all())
    dots = (X[some].double() ** 2).sum(1, keepdim=True)
    assert bool(((dw[some].double() - dots).abs() <= d * 2.0 ** -24 * dots).all())


def test_a_workspace_of_another_streams_blocks_is_not_taken(gpu_device):
    """A block that the current stream's kernels may still use is not handed to a call on a second stream."""
    side, device = torch.cuda.Stream(), torch.device("cuda", torch.cuda.current_device())
    first = binding._scratch(3 << 20, device)
    at = first.data_ptr()
    del first
    second = binding._scratch(3 << 20, device, side)
    assert second.data_ptr() != at
    assert binding._scratch(3 << 20, device).data_ptr() == at
