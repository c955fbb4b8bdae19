"""GPU: a block of GLU experts as a program uses it, on the library's entry points throughout: sorted, gathered, calibrated
and pruned expert by expert, run, and trained for a step; eager, on a side stream and captured into a graph."""
import numpy as np
import pytest
import torch

import oracle
import paper_2405_01943_amd as dass

import linear_reference as ref
from gpu_helpers import bits_equal, to_np32

pytestmark = pytest.mark.gpu

T, K, E, D, D_INT, ACT = 300, 2, 4, 128, 192, "silu"


class Block:
    """Inputs, weights and every buffer of one block."""

    def __init__(self, seed=0, dtype=torch.bfloat16):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s, std=1.0: (torch.randn(s, generator=g) * std).to(dtype).cuda()
        new = lambda *s: torch.zeros(s, dtype=dtype, device="cuda")
        self.X, self.dout = rnd(T, D), rnd(T, D, std=0.1)
        self.Wg, self.Wu, self.Wd = rnd(E, D_INT, D, std=0.09), rnd(E, D_INT, D, std=0.09), rnd(E, D, D_INT, std=0.07)
        self.bias = rnd(E, D, std=0.5)
        top, ids = torch.topk(torch.randn((T, E), generator=g), K, dim=1)
        self.ids, self.w = ids.to(torch.int32).cuda(), torch.softmax(top, 1).cuda()
        self.ids[T - 23:] = -1                                             # a padded batch
        ints = dict(dtype=torch.int32, device="cuda")
        self.offsets, self.order, self.place = torch.zeros(E + 1, **ints), torch.zeros(T * K, **ints), torch.zeros((T, K), **ints)
        R = T * K
        self.rows, self.U, self.pre, self.Y, self.Z, self.out = new(R, D), new(R, D_INT), new(R, D_INT), new(R, D_INT), new(R, D), new(T, D)
        self.dZ, self.dY, self.dU, self.dr1, self.dr2, self.dX = new(R, D), new(R, D_INT), new(R, D_INT), new(R, D), new(R, D), new(T, D)
        self.dw = torch.zeros((T, K), device="cuda")
        self.dWg, self.dWu, self.dWd, self.db = new(E, D_INT, D), new(E, D_INT, D), new(E, D, D_INT), new(E, D)
        need = max(dass.linear_backward_workspace_bytes(R, a, b, dtype, E) for a, b in ((D, D_INT), (D_INT, D)))
        self.ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
        self.ws_sort = torch.zeros(max(16, dass.expert_sort_workspace_bytes(T, K, E)), dtype=torch.uint8, device="cuda")

    def forward(self):
        dass.expert_sort(self.ids, E, self.offsets, self.order, self.place, workspace=self.ws_sort)
        dass.expert_gather(self.X, self.place, self.rows)
        dass.linear(self.rows, self.Wu, self.U, offsets=self.offsets)
        dass.linear(self.rows, self.Wg, self.Y, act=ACT, mul=self.U, pre_out=self.pre, offsets=self.offsets)
        dass.linear(self.Y, self.Wd, self.Z, bias=self.bias, offsets=self.offsets)
        dass.expert_combine(self.Z, self.place, self.out, weights=self.w, residual=self.X)

    def backward(self):
        dass.expert_combine_backward(self.dout, self.Z, self.place, self.w, self.dZ, self.dw)
        dass.linear_backward(self.dZ, self.Y, self.Wd, dX=self.dY, dW=self.dWd, dbias=self.db, offsets=self.offsets, workspace=self.ws)
        dass.linear_backward(self.dY, self.rows, self.Wg, act=ACT, pre=self.pre, mul=self.U, dX=self.dr1, dW=self.dWg, dmul=self.dU,
                             offsets=self.offsets, workspace=self.ws)
        # the gradient that arrives by the gate product is added as the residual of the up product's
        dass.linear_backward(self.dU, self.rows, self.Wu, dX=self.dr2, dW=self.dWu, offsets=self.offsets, workspace=self.ws)
        dass.expert_combine(self.dr1, self.place, self.dX, residual=self.dout)
        dass.expert_combine(self.dr2, self.place, self.dX, residual=self.dX)

    def outputs(self):
        return [getattr(self, n) for n in ("offsets", "order", "place", "out", "dX", "dWg", "dWu", "dWd", "db", "dw")]

    def wipe(self):
        for t in self.outputs() + [self.rows, self.U, self.pre, self.Y, self.Z, self.dZ, self.dY, self.dU, self.dr1, self.dr2]:
            t.zero_()
        self.ws.fill_(0xEE)


def _bits(t):
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


def _autograd(b):
    """The block in float64 with torch's own differentiation."""
    leaves = {n: getattr(b, n).double().requires_grad_() for n in ("X", "Wg", "Wu", "Wd", "bias", "w")}
    out = leaves["X"]
    for j in range(K):
        for e in range(E):
            t = torch.nonzero(b.ids[:, j] == e)[:, 0]
            x = leaves["X"][t]
            y = ref.act(x @ leaves["Wg"][e].t().contiguous(), ACT) * (x @ leaves["Wu"][e].t().contiguous())
            z = y @ leaves["Wd"][e].t().contiguous() + leaves["bias"][e]
            out = out.index_add(0, t, leaves["w"][t, j, None] * z)
    out.backward(b.dout.double())
    return out.detach(), {n: t.grad for n, t in leaves.items()}


def test_block_forward_and_gradients(gpu_device):
    """bf16 throughout.  Between its operators the block rounds four times on the way forward and four on the way back (2^-9 in
    the root mean square each, independent): the root mean square error of each output is below sqrt(8) 2^-9 = 0.0055
    of the output's own for sums of terms of either sign, asked to stay below 2^-6 = 0.0156."""
    b = Block()
    b.forward()
    b.backward()
    torch.cuda.synchronize()
    out, grads = _autograd(b)
    for name, got, want in [("out", b.out, out), ("dX", b.dX, grads["X"]), ("dWg", b.dWg, grads["Wg"]), ("dWu", b.dWu, grads["Wu"]),
                            ("dWd", b.dWd, grads["Wd"]), ("db", b.db, grads["bias"]), ("dw", b.dw, grads["w"])]:
        err = float(torch.linalg.vector_norm(got.double() - want) / torch.linalg.vector_norm(want))
        assert err <= 2.0 ** -6, f"{name}: {err:.4f}"


def test_block_on_a_side_stream(gpu_device):
    b, c = Block(1), Block(1)
    b.forward()
    b.backward()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c.forward()
        c.backward()
    side.synchronize()
    for x, y in zip(b.outputs(), c.outputs()):
        assert torch.equal(_bits(x), _bits(y))


def test_block_replayed_from_a_graph(gpu_device):
    """Two captured blocks of their own buffers, replayed in turn with eager work between, against the eager bits; then the
    same graph on another routing (the captured calls read ids and offsets when they run)."""
    blocks = [Block(2), Block(3)]
    side = torch.cuda.Stream()
    eager, graphs = [], []
    for b in blocks:
        with torch.cuda.stream(side):
            b.forward()
            b.backward()
        side.synchronize()
        eager.append([t.clone() for t in b.outputs()])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.forward()
            b.backward()
        graphs.append(graph)
    for _ in range(3):
        for b in blocks:
            b.wipe()
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for b, want in zip(blocks, eager):
            for x, y in zip(b.outputs(), want):
                assert torch.equal(_bits(x), _bits(y))
    b, fresh = blocks[0], Block(2)
    for t in (b, fresh):
        t.ids.copy_(torch.flip(t.ids, (0,)))
        t.wipe()
    torch.cuda.synchronize()
    graphs[0].replay()
    torch.cuda.synchronize()
    fresh.forward()
    fresh.backward()
    torch.cuda.synchronize()
    for x, y in zip(b.outputs(), fresh.outputs()):
        assert torch.equal(_bits(x), _bits(y))


def test_experts_calibrated_and_pruned(gpu_device):
    """Each expert's rows go to dass_calib_norms as they lie, the masks of all experts in one batched call, and the pruned block
    runs: norms and masks are the oracle's for the expert's tokens."""
    b = Block(4)
    dass.expert_sort(b.ids, E, b.offsets, b.order, b.place, workspace=b.ws_sort)
    dass.expert_gather(b.X, b.place, b.rows)
    lo = b.offsets.tolist()
    norms = torch.zeros((E, D_INT), device="cuda")
    sumsq = torch.zeros((E, D_INT), device="cuda")
    dense = [w.clone() for w in (b.Wg, b.Wu, b.Wd)]
    tasks = []
    for e in range(E):
        dass.calib_norms(b.rows[lo[e]:lo[e + 1]], b.Wg[e], b.Wu[e], ACT, sumsq[e], norms_out=norms[e])
        tasks += [(b.Wg[e], norms[e], "rows", "rows", 0.5), (b.Wu[e], norms[e], "rows", "rows", 0.5), (b.Wd[e], norms[e], "cols", "cols", 1.0)]
    dass.score_mask_nm_batched(tasks, 2, 4)
    b.forward()
    torch.cuda.synchronize()
    for e in range(E):
        mine = (b.ids == e).any(1)
        want = oracle.norms(oracle.sumsq(to_np32(b.X[mine]), to_np32(dense[0][e]), to_np32(dense[1][e]), ACT))
        assert float(np.max(np.abs(norms[e].cpu().numpy() - want) / want)) <= 2e-3
        n32 = norms[e].cpu().numpy()
        for w, d, axis, alpha in ((b.Wg, dense[0], "rows", 0.5), (b.Wu, dense[1], "rows", 0.5), (b.Wd, dense[2], "cols", 1.0)):
            assert bits_equal(w[e], oracle.mask_nm(to_np32(d[e]), n32, axis, axis, alpha, 2, 4)[0])
    out, _ = _autograd(b)
    err = float(torch.linalg.vector_norm(b.out.double() - out) / torch.linalg.vector_norm(out))
    assert err <= 2.0 ** -6
