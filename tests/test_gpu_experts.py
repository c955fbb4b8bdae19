"""GPU parity: tokens sorted by expert and back, and the gradients, against float64.

Tolerances: sorts and copies are exact.  A weighted sum of k rows and a residual has k + 1 f32 roundings (at most
v = 2^-24 of the partial sums, themselves at most A = the sum of the terms' magnitudes): (k + 2) v A, and u (half a step of the
stored type) of the value for the one rounding.  dY is one f32 product and one rounding: u + v.  dweights adds d f32
products, in parts: sqrt(d) v A as a random walk, times 4.
"""
import pytest
import torch

import paper_2405_01943_amd as dass

import linear_reference as ref
from gpu_helpers import padded

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
V = 2.0 ** -24


def _ids(T, k, E, seed=0, pad=0, dtype=torch.int32):
    g = torch.Generator().manual_seed(seed + 13 * T + 5 * k + E)
    logits = torch.randn((T, E), generator=g) + torch.randn((E,), generator=g)
    ids = torch.topk(logits, k, dim=1).indices if k <= E else torch.randint(0, E, (T, k), generator=g)
    if pad:
        ids[T - pad:] = -1
    return ids.to(dtype).cuda()


def _sort(ids, E):
    T, k = ids.shape
    offsets = torch.full((E + 1,), -7, dtype=torch.int32, device="cuda")
    order = torch.full((T * k,), -7, dtype=torch.int32, device="cuda")
    place = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    dass.expert_sort(ids, E, offsets, order, place)
    torch.cuda.synchronize()
    return offsets, order, place


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("T,k,E,pad", [(1, 1, 1, 0), (1, 2, 8, 0), (1, 8, 8, 1), (3, 2, 8, 1), (63, 1, 5, 0), (64, 1, 64, 0), (65, 3, 7, 9),
                                       (333, 4, 16, 20), (1000, 2, 1024, 0), (2048, 2, 8, 203), (4096, 2, 8, 0), (4097, 2, 65, 3)])
def test_sort(gpu_device, T, k, E, pad, dtype):
    ids = _ids(T, k, E, pad=pad, dtype=dtype)
    for got, want, name in zip(_sort(ids, E), ref.sort(ids, E), ("offsets", "order", "place")):
        assert torch.equal(got.cpu(), want), name


@pytest.mark.parametrize("T,k,E", [(5000, 2, 8), (70000, 1, 300), (32768, 8, 64), (262144, 8, 128), (9000, 1, 1024)])
def test_sort_of_many_pairs(gpu_device, T, k, E):
    """Several blocks: a stable sort of the ids gives the same order (the loop of the reference takes minutes here)."""
    ids = _ids(T, k, E, pad=T // 9)
    offsets, order, place = _sort(ids, E)
    key = ids.reshape(-1).long()
    key = torch.where(key < 0, E, key)
    pair = torch.sort(key, stable=True).indices
    n = int((key < E).sum())
    assert torch.equal(order[:n].long(), pair[:n]) and torch.all(order[n:] == -1)
    assert torch.equal(offsets.long(), torch.searchsorted(key[pair].contiguous(), torch.arange(E + 1, device="cuda")))
    back = torch.full_like(key, -1)
    back[pair[:n]] = torch.arange(n, device="cuda")
    assert torch.equal(place.reshape(-1).long(), back)


def test_sort_of_strange_ids(gpu_device):
    """Ids outside the range on either side go nowhere, an expert twice is two rows, and all tokens may go nowhere."""
    ids = torch.tensor([[3, 3], [-1, 4], [2 ** 31 - 1, -2 ** 31], [0, 0], [4, 1]], dtype=torch.int32)
    for t in (ids.cuda(), ids.long().cuda(), (ids.long() * 2 ** 31).cuda(), torch.full((5, 2), -1, dtype=torch.int32).cuda()):
        for got, want in zip(_sort(t, 4), ref.sort(t, 4)):
            assert torch.equal(got.cpu(), want)


ROWS = [(1, 1, 1, 8, 0), (1, 2, 8, 4096, 0), (3, 2, 8, 136, 1), (65, 8, 9, 520, 7), (333, 4, 16, 72, 20), (700, 3, 64, 2056, 0), (5, 2, 4, 64, 5)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,E,d,pad", ROWS)
def test_rows_to_experts_and_back(gpu_device, T, k, E, d, pad, dtype):
    ids = _ids(T, k, E, pad=pad)
    offsets, order, place = _sort(ids, E)
    g = torch.Generator().manual_seed(T + d)
    dt = DT[dtype]
    X, R, dout = (padded(torch.randn((T, d), generator=g).to(dt).cuda(), 8) for _ in range(3))
    Y = padded(torch.randn((T * k, d), generator=g).to(dt).cuda(), 16)
    w = torch.rand((T, k), generator=g).cuda()
    n, u = int(offsets[-1]), torch.finfo(dt).eps / 2
    token = order[:n].long() // k

    rows = padded(torch.full((T * k, d), 3.0, dtype=dt, device="cuda"), 8)
    dass.expert_gather(X, place, rows)
    assert torch.equal(rows[:n], X[token]) and torch.all(rows[n:] == 3.0) and torch.all(rows._base[:, d:] == 7.0)

    # the experts' outputs of pairs that go nowhere may hold anything
    Y[n:] = float("nan")
    at = place.clamp(min=0).long()
    Yp = torch.where((place >= 0)[..., None], Y[at].double(), 0.0)          # [T, k, d]
    for weights, residual in ((None, None), (w, None), (w, R), (None, R)):
        out = padded(torch.full((T, d), 3.0, dtype=dt, device="cuda"), 8)
        dass.expert_combine(Y, place, out, weights=weights, residual=residual)
        terms = Yp * (weights.double()[..., None] if weights is not None else 1)
        want, A = terms.sum(1), terms.abs().sum(1)
        if residual is not None:
            want, A = want + residual.double(), A + residual.double().abs()
        assert torch.all((out.double() - want).abs() <= u * want.abs() + (k + 2) * V * A)
        assert torch.all(out._base[:, d:] == 7.0)
        if residual is not None:
            same = residual.clone()
            dass.expert_combine(Y, place, same, weights=weights, residual=same)
            assert torch.equal(same, out)

    dY = padded(torch.full((T * k, d), 3.0, dtype=dt, device="cuda"), 8)
    dw = torch.full((T, k), 3.0, device="cuda")
    dass.expert_combine_backward(dout, Y, place, w, dY, dw)
    torch.cuda.synchronize()
    want = dout[token].double() * w.reshape(-1)[order[:n].long()].double()[:, None]
    assert torch.all((dY[:n].double() - want).abs() <= (u + V) * want.abs())
    assert torch.all(dY[n:] == 3.0) and torch.all(dY._base[:, d:] == 7.0)
    terms = Yp * dout.double()[:, None]
    assert torch.all((dw.double() - terms.sum(2)).abs() <= 4 * d ** 0.5 * V * terms.abs().sum(2))
    assert torch.all(dw[place < 0] == 0.0)


def test_places_outside_are_nowhere(gpu_device):
    """A place beyond the rows, as a mistake would leave it, is neither read nor written."""
    X = torch.randn((4, 64), device="cuda")
    place = torch.tensor([[0, 8], [2 ** 30, -5], [1, 2], [-1, 3]], dtype=torch.int32, device="cuda")
    rows = torch.zeros((8, 64), device="cuda")
    dass.expert_gather(X, place, rows)
    assert torch.equal(rows[:4], X[[0, 2, 2, 3]]) and torch.all(rows[4:] == 0)
    out, dw, dY = torch.empty((4, 64), device="cuda"), torch.empty((4, 2), device="cuda"), torch.zeros((8, 64), device="cuda")
    dass.expert_combine(rows, place, out)
    assert torch.equal(out, torch.stack([X[0], torch.zeros(64, device="cuda"), X[2] + X[2], X[3]]))
    dass.expert_combine_backward(X, rows, place, torch.ones((4, 2), device="cuda"), dY, dw)
    assert torch.equal(dw != 0, (place >= 0) & (place < 8)) and torch.equal(dY, rows)


def test_gather_and_combine_gradients_against_differences(gpu_device):
    """The combined sum is linear in X, Y and the weights, so differences of any size are exact: moving each operand by
    a direction changes <out, dout> by the gradient's product with it."""
    T, k, E, d = 29, 3, 5, 48
    ids = _ids(T, k, E, pad=4)
    _, order, place = _sort(ids, E)
    g = torch.Generator().manual_seed(2)
    rnd = lambda *s: torch.randn(s, generator=g).cuda()
    X, Y, w, dout, dX, dY, dw = rnd(T, d), rnd(T * k, d), rnd(T, k), rnd(T, d), rnd(T, d), rnd(T * k, d), rnd(T, k)

    def combined(y, weights):
        keep = (place >= 0)[..., None]
        return (torch.where(keep, y[place.clamp(min=0).long()], 0.0) * weights[..., None]).sum(1)

    gY, gw, gX = torch.zeros_like(Y), torch.zeros_like(w), torch.empty_like(X)
    dass.expert_combine_backward(dout, Y, place, w, gY, gw)
    rows = rnd(T * k, d)                                    # a gradient that arrives at the gathered rows
    dass.expert_combine(rows, place, gX)
    D = lambda t: t.double()
    moved = float((D(dout) * (combined(D(Y) + D(dY), D(w)) - combined(D(Y), D(w)))).sum())
    assert abs(float((D(gY) * D(dY)).sum()) - moved) <= 1e-6 * float((D(gY) * D(dY)).abs().sum())
    moved = float((D(dout) * (combined(D(Y), D(w) + D(dw)) - combined(D(Y), D(w)))).sum())
    assert abs(float((D(gw) * D(dw)).sum()) - moved) <= 1e-6 * float((D(gw) * D(dw)).abs().sum())
    n = int((order >= 0).sum())
    moved = float((D(rows[:n]) * D(dX)[order[:n].long() // k]).sum())
    assert abs(float((D(gX) * D(dX)).sum()) - moved) <= 1e-6 * float((D(gX) * D(dX)).abs().sum())
