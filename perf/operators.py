"""Work of a mixture of GLU experts and of its linear layers, as cases that can be timed and compared.

Three steps of such a block, each forwards and backwards: the rows of the tokens are brought into the order of
their experts and the experts' outputs back, weighted (``route``, ``route_grad``); and rows are multiplied
by a weight matrix, one for all rows or that of their expert, with bias, activation, the other branch of a
GLU and a residual in the same pass (``linear``, ``linear_grad``).

With ``own`` the framework's entry points do the work; without it elementary torch operations in f32,
rounded once at the end.  ``exact`` has the same values in f64, by other steps.
"""
import math

import torch

own = False             # True: run() calls the framework

DEVICE = "cuda:0"
MAX_FLOPS = 2.0 * 8192 * 4096 * 14336   # the largest listed product; drawn ones stay below it
MAX_ROUTED = 32768 * 8 * 2048           # elements of the largest listed routing
_ELEM = {"f32": 4, "bf16": 2}
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_ACTS = ("none", "silu", "gelu_tanh", "gelu_erf", "relu")


def listed():
    return [
        # one token of a text being written: two of eight experts (launches and latency)
        {"name": "route_token", "op": "route", "dtype": "bf16", "T": 1, "k": 2, "E": 8, "d": 4096, "pad": 0, "residual": True},
        # one sequence of the calibration set, the last tokens padded (ordinary)
        {"name": "route_seq", "op": "route", "dtype": "bf16", "T": 2048, "k": 2, "E": 8, "d": 4096, "pad": 203, "residual": True},
        # a batch of 16 sequences over many small experts (the largest routing)
        {"name": "route_batch", "op": "route", "dtype": "bf16", "T": 32768, "k": 8, "E": 64, "d": 2048, "pad": 0, "residual": False},
        # the training step of one sequence
        {"name": "route_grad_seq", "op": "route_grad", "dtype": "bf16", "T": 2048, "k": 2, "E": 8, "d": 4096, "pad": 203},
        # a small f32 model in training, odd token count and row length
        {"name": "route_grad_small_f32", "op": "route_grad", "dtype": "f32", "T": 333, "k": 4, "E": 16, "d": 520, "pad": 20},
        # one token through a dense layer: bound by the weights
        {"name": "linear_token", "op": "linear", "dtype": "bf16", "rows": 1, "E": 0, "d_in": 4096, "d_out": 11008,
         "act": "silu", "bias": True, "mul": False, "residual": False, "pre": False, "drop": 0},
        # one sequence through the down projection of a dense block, added to the residual stream (ordinary)
        {"name": "linear_seq", "op": "linear", "dtype": "bf16", "rows": 2048, "E": 0, "d_in": 11008, "d_out": 4096,
         "act": "none", "bias": True, "mul": False, "residual": True, "pre": False, "drop": 0},
        # the tiny f32 configuration
        {"name": "linear_tiny_f32", "op": "linear", "dtype": "f32", "rows": 512, "E": 0, "d_in": 256, "d_out": 688,
         "act": "gelu_erf", "bias": True, "mul": False, "residual": False, "pre": True, "drop": 0},
        # eight texts being written, a token each, two of eight experts a token: the gate product of a GLU
        {"name": "experts_tokens", "op": "linear", "dtype": "bf16", "rows": 16, "E": 8, "d_in": 4096, "d_out": 14336,
         "act": "silu", "bias": False, "mul": True, "residual": False, "pre": False, "drop": 0},
        # two sequences, two experts a token, in training: the gate product of a GLU, its inputs kept (the largest product)
        {"name": "experts_seq", "op": "linear", "dtype": "bf16", "rows": 8192, "E": 8, "d_in": 4096, "d_out": 14336,
         "act": "silu", "bias": False, "mul": True, "residual": False, "pre": True, "drop": 0},
        # the gradients of a gate product, ragged experts, padded rows at the end
        {"name": "experts_grad", "op": "linear_grad", "dtype": "bf16", "rows": 6001, "E": 8, "d_in": 4096, "d_out": 11008,
         "act": "silu", "bias": False, "mul": True, "drop": 59},
        # the gradients of a small dense f32 layer
        {"name": "linear_grad_small_f32", "op": "linear_grad", "dtype": "f32", "rows": 301, "E": 0, "d_in": 256, "d_out": 688,
         "act": "gelu_tanh", "bias": True, "mul": False, "drop": 0},
    ]


def _spread(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread over its logarithm."""
    v = int(round(lo * (hi / lo) ** rng.random()))
    return min(hi // step * step, max(-(-lo // step) * step, v // step * step))


def draw(rng):
    op = rng.choice(("route", "route_grad", "linear", "linear", "linear_grad", "linear_grad"))
    f32 = rng.random() < 0.3
    case = {"op": op, "dtype": "f32" if f32 else "bf16"}
    step = 4 if f32 else 8
    if op.startswith("route"):
        case["E"] = _spread(rng, 2, 128)
        case["k"] = rng.randint(1, min(8, case["E"]))
        case["d"] = _spread(rng, 128, 8192, step)
        case["T"] = _spread(rng, 1, min(65536, MAX_ROUTED // ((2 if f32 else 1) * case["d"] * case["k"])))
        case["pad"] = int(case["T"] * rng.choice((0, 0, 0.1, 0.5)))
        if op == "route":
            case["residual"] = rng.random() < 0.5
        return case
    case["E"] = 0 if rng.random() < 0.5 else _spread(rng, 2, 32)
    many = max(1, case["E"])
    case["d_in"] = _spread(rng, 128, 1024 if f32 else 14336, step)
    case["d_out"] = _spread(rng, 128, 1024 if f32 else 14336, step)
    if many * case["d_in"] * case["d_out"] > 8 * 4096 * 14336:
        case["d_in"] = max(128, 8 * 4096 * 14336 // (many * case["d_out"]) // step * step)
    flops = (2.0 if op == "linear" else 4.0) * case["d_in"] * case["d_out"]
    most = min(4096 if f32 else 16384, max(1, int(MAX_FLOPS / flops)))
    case["rows"] = _spread(rng, 1, most)
    case["act"] = rng.choice(_ACTS)
    case["bias"], case["mul"] = rng.random() < 0.5, rng.random() < 0.4
    case["drop"] = int(case["rows"] * rng.choice((0, 0, 0.1))) if case["E"] else 0
    if op == "linear":
        case["residual"], case["pre"] = rng.random() < 0.5, rng.random() < 0.4
    return case


def _counts(case):
    """Rows of each expert, most popular first: shares that fall with the square root of the rank."""
    share = [(1 + e) ** -0.5 for e in range(case["E"])]
    kept, total = case["rows"] - case["drop"], sum(share)
    n = [int(kept * s / total) for s in share]
    for e in range(kept - sum(n)):
        n[e % case["E"]] += 1
    return n


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    dt = _TORCH[case["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device=DEVICE) * std).to(dt)

    s = {"case": dict(case)}
    if case["op"].startswith("route"):
        T, k, E, d = (case[x] for x in ("T", "k", "E", "d"))
        # the router's choice: some experts are asked for more often; padded tokens go to none
        logits = torch.randn((T, E), generator=gen, device=DEVICE) + torch.randn((E,), generator=gen, device=DEVICE)
        top, ids = torch.topk(logits, k, dim=1)
        s["weights"] = torch.softmax(top, dim=1).contiguous()
        s["ids"] = ids.to(torch.int32)
        if case["pad"]:
            s["ids"][T - case["pad"]:] = -1
        s["Y"] = normal(T * k, d)
        ints = dict(dtype=torch.int32, device=DEVICE)
        s["offsets"] = torch.zeros(E + 1, **ints)
        s["order"], s["place"] = torch.zeros(T * k, **ints), torch.zeros((T, k), **ints)
        s["out"] = torch.zeros((T, d), dtype=dt, device=DEVICE)
        s["rows_out"] = torch.zeros((T * k, d), dtype=dt, device=DEVICE)   # rows behind the last one stay as they are
        if case["op"] == "route":
            s["X"] = normal(T, d)
            s["residual"] = normal(T, d) if case["residual"] else None
            if own:
                import paper_2405_01943_amd as dass
                s["workspace"] = torch.empty(max(16, dass.expert_sort_workspace_bytes(T, k, E)), dtype=torch.uint8, device=DEVICE)
        else:
            s["offsets"], s["order"], s["place"] = _sorted_plain(s["ids"], E)
            s["dout"] = normal(T, d, std=0.01)
            s["dX_rows"] = normal(T * k, d, std=0.01)
            s["dweights"] = torch.zeros((T, k), device=DEVICE)
        return s

    R, E, d_in, d_out = (case[x] for x in ("rows", "E", "d_in", "d_out"))
    shape = (E, d_out, d_in) if E else (d_out, d_in)
    s["X"] = normal(R, d_in)
    s["W"] = torch.empty(shape, dtype=dt, device=DEVICE)
    for w in (s["W"] if E else [s["W"]]):
        w.copy_(normal(d_out, d_in, std=0.02))
    s["bias"] = normal(*shape[:-1], std=0.5) if case["bias"] else None
    s["mul"] = normal(R, d_out, std=1.3) if case["mul"] else None
    s["offsets"] = None
    if E:
        n = torch.tensor(_counts(case))[torch.randperm(E, generator=gen, device=DEVICE).cpu()]
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32).to(DEVICE)
        s["bounds"] = [int(v) for v in s["offsets"].cpu()]

    def zeros(*shape):
        return torch.zeros(shape, dtype=dt, device=DEVICE)

    if case["op"] == "linear":
        s["residual"] = normal(R, d_out) if case["residual"] else None
        s["out"] = zeros(R, d_out)
        s["pre"] = zeros(R, d_out) if case["pre"] else None
    else:
        s["pre"] = normal(R, d_out, std=0.02 * math.sqrt(d_in)) if case["act"] != "none" or case["mul"] else None
        s["dout"] = normal(R, d_out, std=0.01)
        s["dX"], s["dW"] = zeros(R, d_in), zeros(*shape)
        s["dbias"] = zeros(*shape[:-1]) if case["bias"] else None
        s["dmul"] = zeros(R, d_out) if case["mul"] else None
        if own:
            import paper_2405_01943_amd as dass
            need = dass.linear_backward_workspace_bytes(R, d_in, d_out, dt, max(1, E))
            s["workspace"] = torch.empty(max(16, need), dtype=torch.uint8, device=DEVICE)
    return s


# ------------------------------------------------------------------ plain forms --
def _sorted_plain(ids, E):
    flat = ids.reshape(-1).to(torch.int64)
    n = flat.numel()
    key = torch.where((flat >= 0) & (flat < E), flat, E)
    pair = torch.argsort(key, stable=True)
    counts = (key[:, None] == torch.arange(E, device=key.device)).sum(0)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
    order = torch.where(key[pair] < E, pair, -1).to(torch.int32)
    place = torch.empty(n, dtype=torch.int64, device=key.device)
    place[pair] = torch.arange(n, device=key.device)
    place = torch.where(key < E, place, -1).to(torch.int32)
    return offsets, order, place.reshape(ids.shape)


def _gathered(X, order, k):
    keep = (order >= 0)[:, None]
    return torch.where(keep, X[order.clamp(min=0).to(torch.int64) // k], torch.zeros((), dtype=X.dtype, device=X.device))


def _combined(Y, place, weights, residual):
    T, k = place.shape
    total = residual.float() if residual is not None else torch.zeros((T, Y.shape[1]), device=Y.device)
    for j in range(k):
        rows = Y[place[:, j].clamp(min=0).to(torch.int64)].float()
        if weights is not None:
            rows = rows * weights[:, j, None]
        total = total + torch.where((place[:, j] >= 0)[:, None], rows, 0.0)
    return total.to(Y.dtype)


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _act(x, act):
    if act == "none":
        return x
    if act == "silu":
        return x * _sigmoid(x)
    if act == "gelu_tanh":
        return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))
    if act == "gelu_erf":
        return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))
    return torch.where(x > 0, x, torch.zeros_like(x))


def _act_slope(x, act):
    if act == "none":
        return torch.ones_like(x)
    if act == "silu":
        s = _sigmoid(x)
        return s * (1.0 + x * (1.0 - s))
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (x + 0.044715 * x * x * x))
        return 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * x * x)
    if act == "gelu_erf":
        return 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))
    return (x > 0).to(x.dtype)


def _segments(s):
    if not s["case"]["E"]:
        return [(0, s["case"]["rows"], s["W"], s["bias"], 0)]
    b = s["bounds"]
    return [(b[e], b[e + 1], s["W"][e], None if s["bias"] is None else s["bias"][e], e) for e in range(s["case"]["E"])]


def _linear_plain(s):
    case, dt = s["case"], _TORCH[s["case"]["dtype"]]
    out = torch.zeros((case["rows"], case["d_out"]), dtype=dt, device=DEVICE)
    pre = torch.zeros_like(out) if case["pre"] else None
    for lo, hi, W, bias, _ in _segments(s):
        if lo == hi:
            continue
        p = s["X"][lo:hi].float() @ W.float().t()
        if bias is not None:
            p = p + bias.float()
        if pre is not None:
            pre[lo:hi] = p.to(dt)
        p = _act(p, case["act"])
        if s["mul"] is not None:
            p = p * s["mul"][lo:hi].float()
        if s["residual"] is not None:
            p = p + s["residual"][lo:hi].float()
        out[lo:hi] = p.to(dt)
    return [out] + ([pre] if pre is not None else [])


def _linear_grad_plain(s):
    case, dt = s["case"], _TORCH[s["case"]["dtype"]]
    dX, dW = torch.zeros_like(s["dX"]), torch.zeros_like(s["dW"])
    dbias = torch.zeros_like(s["dbias"]) if case["bias"] else None
    dmul = torch.zeros_like(s["dmul"]) if case["mul"] else None
    for lo, hi, W, _, e in _segments(s):
        if lo == hi:
            continue
        g = s["dout"][lo:hi].float()
        x = s["pre"][lo:hi].float() if s["pre"] is not None else None
        if case["mul"]:
            dmul[lo:hi] = (g * _act(x, case["act"])).to(dt)
            g = g * s["mul"][lo:hi].float()
        if case["act"] != "none":
            g = g * _act_slope(x, case["act"])
        dX[lo:hi] = (g @ W.float()).to(dt)
        (dW[e] if case["E"] else dW).copy_((g.t() @ s["X"][lo:hi].float()).to(dt))
        if dbias is not None:
            (dbias[e] if case["E"] else dbias).copy_(g.sum(0).to(dt))
    return [dX, dW] + [t for t in (dbias, dmul) if t is not None]


# ------------------------------------------------------------------------- a pass --
def run(s):
    case = s["case"]
    if not own:
        if case["op"] == "linear":
            return _linear_plain(s)
        if case["op"] == "linear_grad":
            return _linear_grad_plain(s)
        if case["op"] == "route":
            offsets, order, place = _sorted_plain(s["ids"], case["E"])
            return [offsets, order, place, _gathered(s["X"], order, case["k"]),
                    _combined(s["Y"], place, s["weights"], s["residual"])]
        # the weighted sum's gradient, then that of the gather
        k, place, order = case["k"], s["place"], s["order"]
        dY = _gathered(s["dout"], order, k).float()
        dY = (dY * s["weights"].reshape(-1)[order.clamp(min=0).to(torch.int64), None]).to(s["Y"].dtype)
        dweights = torch.empty_like(s["weights"])
        for j in range(k):
            dots = (s["dout"].float() * s["Y"][place[:, j].clamp(min=0).to(torch.int64)].float()).sum(1)
            dweights[:, j] = torch.where(place[:, j] >= 0, dots, 0.0)
        return [dY, dweights, _combined(s["dX_rows"], place, None, None)]

    import paper_2405_01943_amd as dass
    if case["op"] == "linear":
        dass.linear(s["X"], s["W"], s["out"], act=case["act"], bias=s["bias"], mul=s["mul"], residual=s["residual"],
                    pre_out=s["pre"], offsets=s["offsets"])
        return [s["out"]] + ([s["pre"]] if s["pre"] is not None else [])
    if case["op"] == "linear_grad":
        dass.linear_backward(s["dout"], s["X"], s["W"], act=case["act"], pre=s["pre"], mul=s["mul"], dX=s["dX"], dW=s["dW"],
                             dbias=s["dbias"], dmul=s["dmul"], offsets=s["offsets"], workspace=s["workspace"])
        return [s["dX"], s["dW"]] + [t for t in (s["dbias"], s["dmul"]) if t is not None]
    if case["op"] == "route":
        dass.expert_sort(s["ids"], case["E"], s["offsets"], s["order"], s["place"], workspace=s["workspace"])
        dass.expert_gather(s["X"], s["place"], s["rows_out"])
        dass.expert_combine(s["Y"], s["place"], s["out"], weights=s["weights"], residual=s["residual"])
        return [s["offsets"], s["order"], s["place"], s["rows_out"], s["out"]]
    dass.expert_combine_backward(s["dout"], s["Y"], s["place"], s["weights"], s["rows_out"], s["dweights"])
    dass.expert_combine(s["dX_rows"], s["place"], s["out"])
    return [s["rows_out"], s["dweights"], s["out"]]


def work(case):
    e = _ELEM[case["dtype"]]
    if case["op"].startswith("route"):
        T, k, d = case["T"], case["k"], case["d"]
        kept = T - case["pad"]
        n = kept * k
        ints, weights = 4 * (3 * T * k + case["E"] + 1), 4 * T * k
        if case["op"] == "route":   # ids, tokens, expert outputs, residual in; the order, rows and sums out
            return {"bytes": ints + weights + e * d * (kept + 2 * n + T + (T if case["residual"] else 0)), "flops": 2 * n * d}
        return {"bytes": 4 * T * k + 2 * weights + e * d * (kept + 3 * n + T), "flops": 4 * n * d}
    R, d_in, d_out = case["rows"] - case["drop"], case["d_in"], case["d_out"]
    used = sum(n > 0 for n in _counts(case)) if case["E"] else 1
    weights, bias = used * d_in * d_out, used * d_out if case["bias"] else 0
    if case["op"] == "linear":
        wide = 1 + case["mul"] + case["residual"] + case["pre"]
        return {"bytes": e * (R * d_in + weights + bias + wide * R * d_out), "flops": 2 * R * d_in * d_out}
    wide = 1 + (case["act"] != "none" or case["mul"]) + 2 * case["mul"]
    return {"bytes": e * (2 * R * d_in + weights + max(1, case["E"]) * d_in * d_out + bias + wide * R * d_out),
            "flops": 4 * R * d_in * d_out}


# ------------------------------------------------------------------ the same in f64 --
def _act64(x, act):
    """The activation and its slope."""
    if act == "silu":
        s = torch.special.expit(x)
        return x * s, s + x * s * torch.special.expit(-x)
    if act == "gelu_tanh":
        a = 2.0 * math.sqrt(2.0 / math.pi)
        s, c = torch.special.expit(a * (x + 0.044715 * x ** 3)), torch.special.expit(-a * (x + 0.044715 * x ** 3))
        return x * s, s + x * s * c * a * (1.0 + 0.134145 * x ** 2)
    if act == "gelu_erf":
        cdf = torch.special.ndtr(x)
        return x * cdf, cdf + x * torch.exp(-x * x / 2.0) / math.sqrt(2.0 * math.pi)
    if act == "relu":
        return x.clamp(min=0.0), torch.heaviside(x, torch.zeros((), dtype=x.dtype, device=x.device))
    return x, torch.ones_like(x)


def exact(case, seed):
    s = prepare(case, seed)
    f64 = dict(dtype=torch.float64, device=DEVICE)
    if case["op"].startswith("route"):
        T, k, E, d = (case[x] for x in ("T", "k", "E", "d"))
        # a pair's row: rows of smaller experts, and earlier pairs of its own
        flat = s["ids"].reshape(-1).to(torch.int64)
        place = torch.full_like(flat, -1)
        offsets = [0]
        for e in range(E):
            mine = flat == e
            place = torch.where(mine, offsets[-1] + torch.cumsum(mine, 0) - 1, place)
            offsets.append(offsets[-1] + int(mine.sum()))
        pairs = torch.nonzero(place >= 0)[:, 0]
        order = torch.full_like(place, -1)
        order[place[pairs]] = pairs
        n = pairs.numel()
        token, of = order[:n] // k, place.reshape(T, k)
        if case["op"] == "route":
            rows = torch.zeros((T * k, d), dtype=s["X"].dtype, device=DEVICE)
            rows[:n] = s["X"].index_select(0, token)
            total = torch.zeros((T, d), **f64) if s["residual"] is None else s["residual"].double()
            for j in range(k):
                t = torch.nonzero(of[:, j] >= 0)[:, 0]
                total[t] += s["weights"][t, j, None].double() * s["Y"][of[t, j]].double()
            ints = [torch.tensor(offsets, dtype=torch.int32, device=DEVICE), order.to(torch.int32), of.to(torch.int32)]
            return ints + [rows, total]
        dY, dweights, total = torch.zeros((T * k, d), **f64), torch.zeros(T * k, **f64), torch.zeros((T, d), **f64)
        step = max(1, (1 << 26) // d)
        for lo in range(0, n, step):
            p = order[lo:min(n, lo + step)]
            g = s["dout"][p // k].double()
            dY[lo:lo + p.numel()] = g * s["weights"].reshape(-1)[p, None].double()
            dweights[p] = torch.linalg.vecdot(g, s["Y"][lo:lo + p.numel()].double())
        for j in range(k):
            t = torch.nonzero(of[:, j] >= 0)[:, 0]
            total[t] += s["dX_rows"][of[t, j]].double()
        return [dY, dweights.reshape(T, k), total]

    R, E, act = case["rows"], case["E"], case["act"]
    bounds = s["bounds"] if E else [0, R]
    stack = s["W"] if E else s["W"][None]

    def wide(name, lo, hi):
        return s[name][lo:hi].double()

    if case["op"] == "linear":
        out = torch.zeros((R, case["d_out"]), **f64)
        pre = torch.zeros((R, case["d_out"]), **f64) if case["pre"] else None
        for e in range(len(stack)):
            lo, hi = bounds[e], bounds[e + 1]
            p = torch.matmul(stack[e].double(), wide("X", lo, hi).t().contiguous()).t()
            if case["bias"]:
                p = p + s["bias"].reshape(len(stack), -1)[e].double()
            if pre is not None:
                pre[lo:hi] = p
            y = _act64(p, act)[0]
            y = y * wide("mul", lo, hi) if case["mul"] else y
            out[lo:hi] = y + wide("residual", lo, hi) if case["residual"] else y
        return [out] + ([pre] if pre is not None else [])
    dX, dW = torch.zeros((R, case["d_in"]), **f64), torch.zeros(stack.shape, **f64)
    dbias = torch.zeros((len(stack), case["d_out"]), **f64)
    dmul = torch.zeros((R, case["d_out"]), **f64) if case["mul"] else None
    for e in range(len(stack)):
        lo, hi = bounds[e], bounds[e + 1]
        g = wide("dout", lo, hi)
        if s["pre"] is not None:
            y, slope = _act64(wide("pre", lo, hi), act)
            if dmul is not None:
                dmul[lo:hi] = y * g
                slope = slope * wide("mul", lo, hi)
            g = slope * g
        dX[lo:hi] = torch.matmul(stack[e].double().t().contiguous(), g.t().contiguous()).t()
        dW[e] = torch.matmul(wide("X", lo, hi).t().contiguous(), g).t()
        dbias[e] = torch.matmul(torch.ones((1, hi - lo), **f64), g)[0]
    outs = [dX, dW.reshape(s["dW"].shape)] + ([dbias.reshape(s["dbias"].shape)] if case["bias"] else [])
    return outs + ([dmul] if dmul is not None else [])
