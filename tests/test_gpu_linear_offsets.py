"""GPU: offsets that lie outside 0 .. T or fall.  Every output and workspace lies between guards, which nothing may change."""
import pytest
import torch

import paper_2405_01943_amd as dass

import linear_reference as ref
from test_gpu_linear import _check_backward, _check_forward, _make, _saved

pytestmark = pytest.mark.gpu

GUARD, FILL = 300, 3.0     # rows on either side: more than a tile has


class Guarded:
    """A contiguous matrix of FILL between guards of 7."""

    def __init__(self, shape, dtype):
        n = 1
        for s in shape:
            n *= s
        pad = GUARD * shape[-1]
        self.big = torch.full((n + 2 * pad,), 7.0, dtype=dtype, device="cuda")
        self.big[pad:pad + n] = FILL
        self.pad, self.t = pad, self.big[pad:pad + n].view(shape)

    def check(self, what):
        assert bool((self.big[:self.pad] == 7.0).all()) and bool((self.big[-self.pad:] == 7.0).all()), f"{what}: written outside"


def _workspace(n):
    big = torch.full((n + 2 * 65536,), 0x5A, dtype=torch.uint8, device="cuda")
    return big, big[65536:65536 + n]


def _run(p, pre, dout, E, offsets):
    T, d_in, d_out, dt = p["X"].shape[0], p["X"].shape[1], p["W"].shape[-2], p["X"].dtype
    shapes = {"out": (T, d_out), "pre_out": (T, d_out), "dmul": (T, d_out), "dX": (T, d_in), "dW": (E, d_out, d_in), "dbias": (E, d_out)}
    g = {n: Guarded(s, dt) for n, s in shapes.items()}
    spaces = [_workspace(dass.linear_workspace_bytes(T, d_in, d_out, dt, E)), _workspace(dass.linear_backward_workspace_bytes(T, d_in, d_out, dt, E))]
    dass.linear(p["X"], p["W"], g["out"].t, act="silu", bias=p["bias"], mul=p["mul"], residual=p["residual"], pre_out=g["pre_out"].t, offsets=offsets,
                workspace=spaces[0][1])
    dass.linear_backward(dout, p["X"], p["W"], act="silu", pre=pre, mul=p["mul"], offsets=offsets, workspace=spaces[1][1],
                         **{n: g[n].t for n in ("dX", "dW", "dbias", "dmul")})
    torch.cuda.synchronize()
    for name, x in g.items():
        x.check(name)
    for big, inside in spaces:
        assert bool((big[:65536] == 0x5A).all()) and bool((big[65536 + inside.numel():] == 0x5A).all()), "written outside a workspace"
    return {n: x.t for n, x in g.items()}


# tiles of every kind, k whole and split, few rows, both parts of a gradient in one launch and not, g in one part and in two
SIZES = [("bf16", 200, 136, 200), ("bf16", 16, 136, 200), ("bf16", 3, 72, 64), ("bf16", 1500, 264, 520), ("bf16", 700, 2056, 264), ("bf16", 4099, 40, 64),
         ("f32", 200, 136, 200), ("f32", 16, 136, 200), ("f32", 4096, 264, 1000)]


def _cuda(bounds):
    return torch.tensor(bounds, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,T,d_in,d_out", SIZES)
def test_bounds_outside_count_as_the_nearest_inside(gpu_device, dtype, T, d_in, d_out):
    far = 2 ** 31 - 1
    for bounds in ((-7, T // 3, T // 2, T + 5), (-far, -3, 0, T), (T // 4, T // 2, T + 1, far), (T // 3, T // 3, 2 * T // 3, 2 * T // 3), (far, far, far, far), (-9, -8, -7, -6)):
        p = _make(T, d_in, d_out, dtype, E=3)
        pre, dout = _saved(p, dtype)
        inside = [min(max(b, 0), T) for b in bounds]
        got, want = (_run(p, pre, dout, 3, _cuda(b)) for b in (bounds, inside))
        for name in want:
            assert torch.equal(got[name], want[name]), f"{name}, {bounds}"
        # and those are right; rows of no expert keep what they held (both checks look at it)
        p["offsets"] = _cuda(inside)
        if inside[0] < inside[3]:
            _check_forward(p, "silu", want["out"], want["pre_out"], dtype, str(bounds))
            _check_backward(p, "silu", pre, dout, {n: want[n] for n in ("dX", "dW", "dbias", "dmul")}, dtype, str(bounds))
        else:
            assert all(bool((want[n] == FILL).all()) for n in ("out", "pre_out", "dX", "dmul"))
        for e, lo, hi in ref.spans(T, p["offsets"]):
            if lo == hi:
                assert not bool(want["dW"][e].any()) and not bool(want["dbias"][e].any())


@pytest.mark.parametrize("dtype,T,d_in,d_out", SIZES)
def test_bounds_that_fall(gpu_device, dtype, T, d_in, d_out):
    """No promise of values: the call ends, writes inside alone, and rows in no span keep what they held."""
    far = 2 ** 31 - 1
    for bounds in ((0, T // 2, T // 4, T), (0, T + 100, T + 100, 0), (-7, T // 3, 5000000, T // 2), (T // 2, T // 3, T // 4, T // 5), (far, -far, far, -far), (T, 0, T, 0),
                   (T // 2, 0, T // 4, 0)):
        p = _make(T, d_in, d_out, dtype, E=3)
        pre, dout = _saved(p, dtype)
        got = _run(p, pre, dout, 3, _cuda(bounds))
        inside = torch.zeros(T, dtype=torch.bool, device="cuda")
        for e in range(3):
            lo = min(max(bounds[e], 0), T)
            inside[lo:max(lo, min(bounds[e + 1], T))] = True
        for name in ("out", "pre_out", "dX", "dmul"):
            assert bool((got[name][~inside] == FILL).all()), f"{name}, {bounds}"
