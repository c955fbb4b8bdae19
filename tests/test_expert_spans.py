"""Host-only: rows and strides that are allowed each by itself, but not together (no GPU call is made here).

Every call has a misaligned operand as well, which is looked at after the rows: what passes as far as that is refused as ALIGN."""
import pytest
import torch  # noqa: F401  (the library is linked against the runtime that torch loads)

import paper_2405_01943_amd as dass

from test_expert_refusals import A, B, C, ODD, _grad, _linear, _name

FAR = 1 << 36          # the longest stride


@pytest.fixture(scope="module")
def lib():
    return dass.load_library()


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("p,ld", [("out", "ldo"), ("mul", "ldm"), ("residual", "ldr"), ("pre_out", "ldp")])
def test_linear_rows_times_stride(lib, p, ld, dt):
    at = {"out": B}.get(p, C)
    assert _linear(lib, dt=dt, T=1 << 10, **{p: at, ld: FAR}, bias=ODD) == "ALIGN"                  # 2^46 elements
    assert _linear(lib, dt=dt, T=(1 << 10) + 1, **{p: at, ld: FAR}, bias=ODD) == "SHAPE"
    assert _linear(lib, dt=dt, T=1 << 30, **{p: at, ld: FAR}, bias=ODD) == "SHAPE"                  # 2^66
    assert _linear(lib, dt=dt, T=1 << 30, **{p: at, ld: 1 << 16}, bias=ODD) == "ALIGN"


def test_linear_operands_rows_times_stride(lib):
    long = (1 << 22) - 16                                                                              # rows of X just below 8 MiB apart
    assert _linear(lib, T=1 << 30, ldx=long, bias=ODD) == "SHAPE" and _linear(lib, T=1 << 24, ldx=long, bias=ODD) == "ALIGN"


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("p,ld", [("pre", "ldp"), ("mul", "ldm"), ("dX", "lddx"), ("dmul", "lddm"), ("dW", "lddw")])
def test_linear_backward_rows_times_stride(lib, p, ld, dt):
    rows = "d_out" if p == "dW" else "T"
    wide = dict(ldg=1 << 16, ldp=1 << 16, ldm=1 << 16, lddm=1 << 16) if p == "dW" else {}
    with_mul = dict(wide, dt=dt, mul=0x600000, dmul=0x800000, dbias=ODD)
    with_mul.setdefault("ldm", 64)
    with_mul.setdefault("lddm", 64)
    with_mul[ld] = FAR
    assert _grad(lib, **{**with_mul, rows: 1 << 10}) == "ALIGN"
    assert _grad(lib, **{**with_mul, rows: (1 << 10) + 8}) == "SHAPE"


def test_rows_times_stride(lib):
    far = dict(T=1 << 24, k=2)

    def gather(T=8, k=2, ldx=64, ldo=64):
        return _name(lib, lib.dass_expert_gather(A, T, ldx, 64, 1, 0x10002, k, B, ldo, None))

    def combine(T=8, k=2, ldx=64, ldo=64, ldr=64):
        return _name(lib, lib.dass_expert_combine(A, ldx, 0x10002, T, k, None, C, ldr, 64, 1, B, ldo, None))

    def grad(T=8, k=2, ldx=64, ldo=64, ldy=64):
        return _name(lib, lib.dass_expert_combine_backward(A, ldx, C, ldy, 0x10002, T, k, A, 64, 1, B, ldo, A, None))

    for call, strides in ((gather, ("ldx", "ldo")), (combine, ("ldx", "ldo", "ldr")), (grad, ("ldx", "ldo", "ldy"))):
        assert call(**far) == "ALIGN"
        for ld in strides:
            assert call(**far, **{ld: FAR}) == "SHAPE" and call(T=512, k=2, **{ld: FAR}) == "ALIGN"
    # pairs, not tokens, are the rows of the sorted side
    assert gather(T=1 << 10, k=1, ldo=FAR) == "ALIGN" and gather(T=1 << 10, k=2, ldo=FAR) == "SHAPE" and gather(T=1 << 10, k=2, ldx=FAR) == "ALIGN"
