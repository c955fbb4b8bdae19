"""GPU: every entry point of the experts' rows and linear layers on a stream that is given, not the current one."""
import types

import pytest
import torch

import paper_2405_01943_amd as dass
from paper_2405_01943_amd import binding

pytestmark = pytest.mark.gpu

# few pairs and many (the sort's workspace); outputs with shares of k in a workspace and without
SIZES = [(300, 2, 4, 128, 192), (6000, 2, 8, 64, 72), (64, 1, 1, 4096, 512)]


class Calls:
    """Buffers of one block, and its calls on a stream (None: the current one), each workspace left to the binding or not."""

    def __init__(self, T, k, E, d, n):
        g = torch.Generator().manual_seed(T + n)
        rnd = lambda *s, std=1.0: (torch.randn(s, generator=g) * std).bfloat16().cuda()
        new = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")
        i32 = torch.int32
        self.k, self.E, R = k, E, T * k
        self.source = {"X": rnd(T, d), "ids": torch.randint(0, E, (T, k), generator=g, dtype=i32).cuda(), "w": torch.rand((T, k), generator=g).cuda()}
        self.X, self.ids, self.w = new(T, d), new(T, k, dt=i32), new(T, k, dt=torch.float32)
        self.W, self.V = rnd(E, n, d, std=d ** -0.5), rnd(E, d, n, std=n ** -0.5)
        self.offsets, self.order, self.place = new(E + 1, dt=i32), new(R, dt=i32), new(T, k, dt=i32)
        self.rows, self.pre, self.y, self.z, self.out = new(R, d), new(R, n), new(R, n), new(R, d), new(T, d)
        self.dz, self.dw, self.dy, self.dr, self.dX = new(R, d), new(T, k, dt=torch.float32), new(R, n), new(R, d), new(T, d)
        self.dW, self.dV, self.db = torch.zeros_like(self.W), torch.zeros_like(self.V), new(E, d)

    def fill(self):
        """The inputs, as the last step of a long piece of work on the current stream."""
        a = torch.ones((4096, 4096), device="cuda")
        for _ in range(20):
            a = (a @ a) * (1 / 4096)
        one = a[0, 0]            # exactly 1
        self.X.copy_(self.source["X"] * one)
        self.w.copy_(self.source["w"] * one)
        self.ids.copy_(self.source["ids"] * one.to(torch.int32))

    def run(self, stream):
        on = dict(stream=stream)
        dass.expert_sort(self.ids, self.E, self.offsets, self.order, self.place, **on)
        dass.expert_gather(self.X, self.place, self.rows, **on)
        dass.linear(self.rows, self.W, self.y, act="silu", pre_out=self.pre, offsets=self.offsets, **on)
        dass.linear(self.y, self.V, self.z, offsets=self.offsets, **on)
        dass.expert_combine(self.z, self.place, self.out, weights=self.w, residual=self.X, **on)
        dass.expert_combine_backward(self.out, self.z, self.place, self.w, self.dz, self.dw, **on)
        dass.linear_backward(self.dz, self.y, self.V, dX=self.dy, dW=self.dV, dbias=self.db, offsets=self.offsets, **on)
        dass.linear_backward(self.dy, self.rows, self.W, act="silu", pre=self.pre, dX=self.dr, dW=self.dW, offsets=self.offsets, **on)
        dass.expert_combine(self.dr, self.place, self.dX, **on)

    def results(self):
        return {n: getattr(self, n) for n in ("offsets", "order", "place", "rows", "pre", "y", "z", "out", "dz", "dw", "dy", "dV", "db", "dr", "dW", "dX")}


@pytest.mark.parametrize("T,k,E,d,n", SIZES)
def test_calls_go_to_the_given_stream(gpu_device, T, k, E, d, n):
    """The inputs are there only when the given stream's work before the calls is done: on another stream they would be read
    too early.  Beside it the current stream keeps taking and filling memory of the workspaces' sizes."""
    want, got = Calls(T, k, E, d, n), Calls(T, k, E, d, n)
    want.fill()
    want.run(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got.fill()
    got.run(side)
    for size in (1 << 12, 1 << 16, 1 << 18, 1 << 20, 1 << 22) * 4:
        torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    side.synchronize()
    for (name, a), b in zip(want.results().items(), got.results().values()):
        assert torch.equal(a, b), name
    torch.cuda.synchronize()


def test_a_stream_of_another_gpu_is_refused(gpu_device, monkeypatch):
    """The tensors' GPU, the stream's and the current one have to be one: workspaces and launches go by each of them."""
    c = Calls(300, 2, 4, 128, 192)
    other = types.SimpleNamespace(device_index=1, cuda_stream=0)
    with pytest.raises(ValueError, match="stream is of GPU 1"):
        dass.expert_gather(c.X, c.place, c.rows, stream=other)
    with pytest.raises(ValueError, match="stream is of GPU 1"):
        dass.linear(c.rows, c.W, c.y, offsets=c.offsets, stream=other)
    mine = torch.cuda.Stream()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current"):
        dass.expert_gather(c.X, c.place, c.rows)
    for call in (lambda: dass.expert_gather(c.X, c.place, c.rows, stream=mine), lambda: dass.expert_sort(c.ids, 4, c.offsets, c.order, c.place, stream=mine),
                 lambda: dass.linear(c.rows, c.W, c.y, offsets=c.offsets, stream=mine),
                 lambda: dass.linear_backward(c.y, c.rows, c.W, dX=c.dr, offsets=c.offsets, stream=mine)):
        with pytest.raises(ValueError, match="current"):
            call()


def test_a_workspace_of_the_current_stream_is_not_switched_to(gpu_device, monkeypatch):
    """The current stream given by name: its blocks come without entering it again; another stream's do not."""
    device = torch.device("cuda", torch.cuda.current_device())
    current, side = torch.cuda.current_stream(), torch.cuda.Stream()
    entered = []
    switch = torch.cuda.stream
    monkeypatch.setattr(torch.cuda, "stream", lambda s: entered.append(s) or switch(s))
    at = binding._scratch(5 << 20, device).data_ptr()
    assert binding._scratch(5 << 20, device, current).data_ptr() == at and not entered
    assert binding._scratch(5 << 20, device, side).data_ptr() != at and entered == [side]
    with switch(side):
        assert binding._scratch(5 << 20, device, side).data_ptr() != at and entered == [side]
        assert binding._scratch(5 << 20, device, current).data_ptr() == at and entered == [side, current]
