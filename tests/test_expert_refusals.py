"""Host-only: what dass_expert_* and dass_linear* refuse, before anything is launched (no GPU call is made here)."""
import ctypes

import pytest
import torch

import paper_2405_01943_amd as dass
from paper_2405_01943_amd import binding

A, ODD = 0x10000, 0x10004          # aligned and not, never dereferenced
B, C, D = 0x200000, 0x400000, 0x600000


@pytest.fixture(scope="module")
def lib():
    return dass.load_library()


def _name(lib, status):
    if status:
        assert lib.dass_last_error_string() != b""
    return lib.dass_status_string(status).decode().replace("DASS_ERR_", "")


def test_sort_rejections(lib):
    def call(ids=A, width=4, T=64, k=2, E=8, off=A, order=A, place=A, ws=None, wsb=0):
        return _name(lib, lib.dass_expert_sort(ids, width, T, k, E, off, order, place, ws, wsb, None))
    for name in ("ids", "off", "order", "place"):
        assert call(**{name: None}) == "NULL"
        assert call(**{name: 0x10002}) == "ALIGN"
    assert call(ids=ODD, width=8) == "ALIGN"
    assert call(width=2) == "ARG"
    assert call(T=0) == call(k=0) == call(k=65) == call(E=0) == call(E=1025) == call(T=2 ** 30, k=2) == "SHAPE"
    assert call(T=1 << 20) == call(T=1 << 20, ws=A, wsb=64) == "WORKSPACE"
    assert call(T=1 << 20, ws=ODD, wsb=1 << 30) == "ALIGN"
    need = lib.dass_expert_sort_workspace_bytes
    assert need(64, 2, 8) == 0 and need(0, 2, 8) == 0 and need(2 ** 40, 64, 8) == 0 and need(1 << 20, 2, 8) > 0


def test_row_rejections(lib):
    def gather(X=A, T=8, ldx=64, d=64, dt=1, place=A, k=2, out=A, ldo=64):
        return _name(lib, lib.dass_expert_gather(X, T, ldx, d, dt, place, k, out, ldo, None))

    def combine(X=A, T=8, ldx=64, d=64, dt=1, place=A, k=2, out=A, ldo=64, w=A, r=A, ldr=64):
        return _name(lib, lib.dass_expert_combine(X, ldx, place, T, k, w, r, ldr, d, dt, out, ldo, None))

    def grad(X=A, T=8, ldx=64, d=64, dt=1, place=A, k=2, out=A, ldo=64, w=A, dw=A, Y=A, ldy=64):
        return _name(lib, lib.dass_expert_combine_backward(X, ldx, Y, ldy, place, T, k, w, d, dt, out, ldo, dw, None))

    for call in (gather, combine, grad):
        assert call(X=None) == call(place=None) == call(out=None) == "NULL"
        assert call(dt=2) == "DTYPE"
        assert call(T=0) == call(k=0) == call(k=65) == call(d=0) == call(d=60) == call(ldx=56) == call(ldo=56) == call(ldx=2 ** 50) == "SHAPE"
        assert call(T=2 ** 30, k=2) == "SHAPE"
        assert call(X=ODD) == call(out=ODD) == call(ldx=68) == call(ldo=68) == call(place=0x10002) == "ALIGN"
    assert gather(T=1 << 24, d=1 << 20, ldx=1 << 20, ldo=1 << 20) == "SHAPE"      # more chunks than a launch has threads
    assert combine(r=ODD) == combine(ldr=68) == combine(w=0x10002) == "ALIGN" and combine(ldr=56) == "SHAPE"
    assert grad(w=None) == grad(dw=None) == grad(Y=None) == "NULL" and grad(dw=0x10002) == "ALIGN" and grad(ldy=56) == "SHAPE"


def test_rows_over_their_inputs(lib):
    """An output that begins where an input does would be read after it is written."""
    assert _name(lib, lib.dass_expert_gather(A, 8, 64, 64, 1, B, 2, A, 64, None)) == "ARG"
    assert _name(lib, lib.dass_expert_combine(A, 64, B, 8, 2, C, None, 0, 64, 1, A, 64, None)) == "ARG"
    assert _name(lib, lib.dass_expert_combine(A, 64, B, 8, 2, C, D, 72, 64, 1, D, 64, None)) == "ARG"     # the residual's own stride alone
    for dout, Y, dY, w, dw in ((A, B, A, C, D), (A, B, B, C, D), (A, B, 0x800000, C, C)):
        assert _name(lib, lib.dass_expert_combine_backward(dout, 64, Y, 64, D, 8, 2, w, 64, 1, dY, 64, dw, None)) == "ARG"


def _linear(lib, **change):
    t = dict(X=A, T=8, ldx=64, W=A, ldw=64, expert_stride=0, d_in=64, d_out=64, offsets=None, n_experts=1, bias=None, mul=None, ldm=0,
             residual=None, ldr=0, pre_out=None, ldp=0, out=B, ldo=64, dt=1, act=4)
    t.update(change)
    return _name(lib, lib.dass_linear(ctypes.byref(binding.LinearTask(**t)), None, 0, None))


def test_linear_rejections(lib):
    assert _name(lib, lib.dass_linear(None, None, 0, None)) == "NULL"
    for p, ld in (("X", "ldx"), ("W", "ldw"), ("out", "ldo")):
        assert _linear(lib, **{p: None}) == "NULL"
    for p, ld in (("X", "ldx"), ("W", "ldw"), ("out", "ldo"), ("mul", "ldm"), ("residual", "ldr"), ("pre_out", "ldp")):
        assert _linear(lib, **{p: ODD, ld: 64}) == "ALIGN"
        assert _linear(lib, **{p: A, ld: 68}) == "ALIGN"
        assert _linear(lib, **{p: A, ld: 56}) == "SHAPE"
    assert _linear(lib, bias=ODD) == _linear(lib, offsets=0x10002) == "ALIGN"
    assert _linear(lib, dt=2) == _linear(lib, act=5) == _linear(lib, act=-1) == "DTYPE"
    for name in ("T", "d_in", "d_out", "n_experts"):
        assert _linear(lib, **{name: 0}) == "SHAPE"
    assert _linear(lib, d_in=2 ** 25, ldx=2 ** 25, ldw=2 ** 25) == _linear(lib, ldx=2 ** 40) == _linear(lib, offsets=A, n_experts=2, expert_stride=2 ** 60) == "SHAPE"
    assert _linear(lib, T=2 ** 31) == _linear(lib, d_in=60) == _linear(lib, d_out=60) == "SHAPE"
    assert _linear(lib, n_experts=2) == _linear(lib, offsets=A, n_experts=1025) == "SHAPE"
    assert _linear(lib, offsets=A, n_experts=2, expert_stride=63 * 64) == "SHAPE"
    assert _linear(lib, offsets=A, n_experts=2, expert_stride=64 * 64 + 4) == "ALIGN"
    # outputs over operands; mul and residual alone may be out, with its stride
    assert _linear(lib, out=A) == _linear(lib, pre_out=B, ldp=64) == _linear(lib, pre_out=A, ldp=64) == "ARG"
    assert _linear(lib, pre_out=C, ldp=64, mul=C, ldm=64) == "ARG"
    assert _linear(lib, residual=B, ldr=72) == _linear(lib, mul=B, ldm=72) == "ARG"
    # few rows of many columns: k is split, and its shares need room
    assert lib.dass_linear_workspace_bytes(64, 4096, 512, 1, 1) > 0
    wide = dict(T=64, d_in=4096, ldx=4096, ldw=4096, d_out=512, ldo=512)
    assert _linear(lib, **wide) == "WORKSPACE"
    assert lib.dass_linear_workspace_bytes(0, 64, 64, 1, 1) == lib.dass_linear_workspace_bytes(8, 64, 64, 9, 1) == 0


def test_linear_limits(lib):
    """What is beyond the stated sizes is refused by size alone, before any part of the work."""
    for dt, e in ((1, 2), (0, 4)):
        near, far = (1 << 23) // e - 16, (1 << 23) // e          # elements: rows less than 8 MiB apart, and 8 MiB
        assert _linear(lib, dt=dt, ldx=far) == _linear(lib, dt=dt, ldw=far) == "SHAPE"
        assert _linear(lib, dt=dt, ldx=near, ldw=near, out=ODD) == _linear(lib, dt=dt, ldo=1 << 36, out=ODD) == "ALIGN"
        for ld in ("ldg", "ldx", "ldw"):
            assert _grad(lib, dt=dt, **{ld: far}) == "SHAPE" and _grad(lib, dt=dt, **{ld: near}, dX=ODD) == "ALIGN"
        assert _linear(lib, dt=dt, T=2 ** 30 + 1) == _linear(lib, dt=dt, d_out=2 ** 20 + 8, ldo=2 ** 21) == "SHAPE"
        assert _linear(lib, dt=dt, d_in=2 ** 20 + 8, ldx=2 ** 21 - 16, ldw=2 ** 21 - 16) == "SHAPE"
    assert lib.dass_linear_workspace_bytes(2 ** 30 + 1, 64, 64, 1, 1) == 0


def _grad(lib, ws=A, wsb=1 << 30, **change):
    t = dict(dout=A, T=8, ldg=64, X=A, ldx=64, W=A, ldw=64, expert_stride=0, d_in=64, d_out=64, offsets=None, n_experts=1, pre=A, ldp=64,
             mul=None, ldm=0, dX=B, lddx=64, dW=C, lddw=64, dw_stride=0, dbias=None, dmul=None, lddm=0, dt=1, act=0)
    t.update(change)
    return _name(lib, lib.dass_linear_backward(ctypes.byref(binding.LinearGradTask(**t)), ws, wsb, None))


def test_linear_backward_rejections(lib):
    assert _name(lib, lib.dass_linear_backward(None, A, 1 << 30, None)) == "NULL"
    assert _grad(lib, dX=None, dW=None) == "NULL"                                     # nothing asked for
    assert _grad(lib, dout=None) == _grad(lib, X=None) == _grad(lib, W=None) == _grad(lib, pre=None) == "NULL"
    assert _grad(lib, dmul=A, lddm=64) == "NULL"                                      # dmul without mul
    assert _grad(lib, act=4, pre=None, mul=A, ldm=64, dmul=A, lddm=64) == "NULL"      # and without pre
    for p, ld in (("dout", "ldg"), ("X", "ldx"), ("W", "ldw"), ("pre", "ldp"), ("dX", "lddx"), ("dW", "lddw")):
        assert _grad(lib, **{p: ODD}) == _grad(lib, **{ld: 68}) == "ALIGN"
        assert _grad(lib, **{ld: 56}) == "SHAPE"
    assert _grad(lib, mul=A, ldm=64, dmul=ODD, lddm=64) == _grad(lib, dbias=ODD) == "ALIGN"
    assert _grad(lib, dt=2) == _grad(lib, act=5) == "DTYPE"
    assert _grad(lib, offsets=A, n_experts=2, expert_stride=64 * 64, dw_stride=8) == "SHAPE"
    assert _grad(lib, ws=None) == _grad(lib, wsb=64) == "WORKSPACE" and _grad(lib, ws=ODD) == "ALIGN"
    for out in ("dX", "dW", "dbias"):
        assert _grad(lib, **{out: A}) == "ARG"
    assert _grad(lib, dX=C) == _grad(lib, mul=D, ldm=64, dmul=D, lddm=64) == _grad(lib, mul=D, ldm=64, dmul=B, lddm=64) == "ARG"
    need = lib.dass_linear_backward_workspace_bytes
    assert need(0, 64, 64, 1, 1) == 0 and need(8, 64, 64, 7, 1) == 0 and need(8, 64, 64, 1, 2000) == 0
    assert need(1000, 64, 688, 1, 4) >= 1000 * 688 * 2 + 4 * 688


def test_binding_rejections():
    """Wrong shapes, types and strides, and tensors that are not on the GPU, are refused by the binding."""
    X, W, out = torch.zeros(4, 64), torch.zeros(32, 64), torch.zeros(4, 32)
    off, ids = torch.zeros(3, dtype=torch.int32), torch.zeros((4, 2), dtype=torch.int32)
    order, place = torch.zeros(8, dtype=torch.int32), torch.zeros((4, 2), dtype=torch.int32)
    with pytest.raises(ValueError, match="on the GPU"):
        dass.linear(X, W, out)
    with pytest.raises(ValueError, match="on the GPU"):
        dass.linear_backward(out, X, W, dX=torch.zeros(4, 64))
    with pytest.raises(ValueError, match="on the GPU"):
        dass.expert_sort(ids, 2, off, order, place)
    with pytest.raises(ValueError, match="on the GPU"):
        dass.expert_gather(X, place, torch.zeros(8, 64))
    with pytest.raises(ValueError, match="on the GPU"):
        dass.expert_combine(torch.zeros(8, 64), place, X)
    with pytest.raises(ValueError, match="on the GPU"):
        dass.expert_combine_backward(X, torch.zeros(8, 64), place, torch.zeros(4, 2), torch.zeros(8, 64), torch.zeros(4, 2))
    with pytest.raises(KeyError):
        dass.linear(X, W, out, act="tanh")
    for bad in (dict(W=torch.zeros(32, 60)), dict(out=torch.zeros(4, 40)), dict(mul=torch.zeros(5, 32)), dict(residual=torch.zeros(4, 32).bfloat16())):
        with pytest.raises((TypeError, ValueError)):
            dass.linear(**{"X": X, "W": W, "out": out, **bad})
    for bad in (dict(W=torch.zeros(32, 64).bfloat16()), dict(X=X.t()), dict(bias=torch.zeros(31)), dict(bias=torch.zeros(64)[::2]),
                dict(offsets=off), dict(offsets=off.long(), W=torch.zeros(2, 32, 64)), dict(offsets=off, W=torch.zeros(3, 32, 64)),
                dict(offsets=off, W=torch.zeros(2, 32, 64), bias=torch.zeros(32))):
        with pytest.raises((TypeError, ValueError)):
            dass.linear(**{"X": X, "W": W, "out": out, **bad})
    with pytest.raises(ValueError):
        dass.linear_backward(out, X, W, dW=torch.zeros(32, 60))
    for bad in (dict(experts=ids.float()), dict(offsets=off[:2]), dict(order=order[:7]), dict(place=place.long()), dict(experts=ids[:, :1])):
        with pytest.raises(TypeError):
            dass.expert_sort(**{"experts": ids, "n_experts": 2, "offsets": off, "order": order, "place": place, **bad})
    with pytest.raises(ValueError):
        dass.expert_gather(X, place, torch.zeros(7, 64))
    with pytest.raises(TypeError):
        dass.expert_combine(torch.zeros(8, 64), place, X, weights=torch.zeros(4, 2).bfloat16())
