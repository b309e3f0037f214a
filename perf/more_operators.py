"""Workloads of the operators of one layer at eight bits: quantisation to 8-bit integers with a scale for each token or
channel, the products of such matrices (forward for batches and for single frames, backward for both gradients), and the gated
layer y = act(x Wg^T) * (x Wv^T) (forward, and backward down to both gradients).

``listed()`` names the cases, ``draw()`` makes more of the same ranges, ``prepare()`` makes what a program has in hand before the
call, ``run()`` is one call (the plain torch form, or with ``own`` the library's), ``exact()`` the definition in 64 bits, ``work()``
the bytes and operations a call cannot do without.

The 8-bit format: every row (a token, or an output channel of a weight matrix) has one FP32 scale
    s = max(largest magnitude of the row / 127, 2^-126),  codes q = nearest integer to x * r, ties to even, with r = 1 / s,
s and r rounded to FP32, the product x * r not rounded before it is made an integer.  A code stands for q * s.  Layout: row r of
the codes is 16 * ceil(cols / 16) bytes, zeros behind the last column.

The gated layer keeps its two matrices as one of 2 F rows, the gate's first; what the forward pass leaves for the backward pass
is pre = (x Wg^T | x Wv^T), frames x 2 F.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}


# ------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # the encoder's output of one frame (d = 512), sent and read back in eight bits: latency
        {"name": "round trip, one frame", "op": "round_trip", "rows": 1, "cols": 512, "type": "f16", "both": False},
        # a feed-forward matrix (4d x d, d = 2048) decompressed by the store, quantised along both of its axes
        # as a training step needs it
        {"name": "round trip, weight matrix both ways", "op": "round_trip", "rows": 8192, "cols": 2048, "type": "f32", "both": True},
        # streaming recognition: one frame through the first feed-forward matrix at d = 2048
        {"name": "linear, one frame", "op": "linear", "m": 1, "n": 8192, "k": 2048, "type": "bf16"},
        # a short utterance through layers of odd widths (pruned or ragged models)
        {"name": "linear, ragged", "op": "linear", "m": 77, "n": 777, "k": 1000, "type": "f16"},
        # the second feed-forward matrix at d = 2048 for a large batch
        {"name": "linear, d 2048", "op": "linear", "m": 16384, "n": 2048, "k": 8192, "type": "bf16"},
        # backward through the feed-forward matrix at d = 512, a batch whose frames do not fill the tiles
        {"name": "linear backward, d 512", "op": "linear_backward", "m": 1999, "n": 2048, "k": 512, "type": "f32"},
        # backward through the feed-forward matrix at d = 2048
        {"name": "linear backward, d 2048", "op": "linear_backward", "m": 8192, "n": 8192, "k": 2048, "type": "bf16"},
        # streaming recognition: one frame through a gated feed-forward layer at d = 512
        {"name": "gated, one frame", "op": "gated", "m": 1, "f": 2048, "k": 512, "type": "f16", "act": "silu", "keep": False},
        # training: the pointwise convolution and gated linear unit of a convolution module of odd width, a ragged batch
        {"name": "gated, ragged", "op": "gated", "m": 1501, "f": 513, "k": 1000, "type": "f32", "act": "sigmoid", "keep": True},
        # training: a gated feed-forward layer at d = 2048, a large batch
        {"name": "gated, d 2048", "op": "gated", "m": 8192, "f": 8192, "k": 2048, "type": "bf16", "act": "silu", "keep": True},
        # the gradients of gate and value alone, for a program that goes on in FP32
        {"name": "gated backward, ragged", "op": "gated_backward", "m": 1501, "f": 513, "k": 1000, "type": "f32", "act": "gelu"},
        # the whole backward pass of the gated layer at d = 2048
        {"name": "gated backward, d 2048", "op": "gated_step_backward", "m": 8192, "f": 8192, "k": 2048, "type": "bf16", "act": "silu"},
    ]


def _log_int(rng, lo, hi):
    v = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))
    v = min(max(v, lo), hi)
    pick = rng.random()
    if pick < 0.4 and v >= 64:          # widths and batches are round numbers about as often as not
        v -= v % 32
    elif pick < 0.6 and v % 2 == 0 and v > lo:
        v -= 1
    return v


def draw(rng):
    op = rng.choice(["round_trip", "linear", "linear", "linear_backward", "gated", "gated", "gated_backward", "gated_step_backward"])
    kind = rng.choice(["f32", "f16", "bf16"])
    if op == "round_trip":
        rows, cols = _log_int(rng, 1, 16384), _log_int(rng, 1, 8192)
        rows = max(1, min(rows, 8192 * 2048 // cols))
        return {"op": op, "rows": rows, "cols": cols, "type": kind, "both": rng.random() < 0.5}
    if op in ("linear", "linear_backward"):
        n, k = _log_int(rng, 64, 8192), _log_int(rng, 64, 8192)
        m = _log_int(rng, 1, 16384) if op == "linear" else _log_int(rng, 32, 8192)
        most = 16384 * 2048 * 8192 if op == "linear" else 8192 * 8192 * 2048
        m = max(1, min(m, most // (n * k)))
        return {"op": op, "m": m, "n": n, "k": k, "type": kind}
    if op == "gated_step_backward":     # the codes of FP32 gradients follow the last bit of the activation: not comparable
        kind = rng.choice(["f16", "bf16"])
    f, k = _log_int(rng, 32, 8192), _log_int(rng, 64, 8192)
    m = _log_int(rng, 1, 8192) if op == "gated" else _log_int(rng, 32, 8192)
    m = max(1, min(m, 8192 * 8192 * 2048 // (f * k), 8192 * 8192 * 2 // _BYTES[kind] // f))
    case = {"op": op, "m": m, "f": f, "k": k, "type": kind, "act": rng.choice(["sigmoid", "silu", "gelu"])}
    if op == "gated":
        case["keep"] = rng.random() < 0.5
    return case


def work(case):
    b = _BYTES[case["type"]]
    if case["op"] == "round_trip":
        n = case["rows"] * case["cols"]
        both = 2 if case["both"] else 1
        return {"bytes": n * b * (1 + both), "flops": 0}
    m, k = case["m"], case["k"]
    if case["op"] == "linear":
        n = case["n"]
        return {"bytes": m * k * b + _stored(n, k) + m * n * b, "flops": 2 * m * n * k}
    if case["op"] == "linear_backward":
        n = case["n"]
        return {"bytes": m * n * b + _stored(k, n) + _stored(k, m) + m * k * b + n * k * 4, "flops": 4 * m * n * k}
    f = case["f"]
    if case["op"] == "gated":
        return {"bytes": m * k * b + _stored(2 * f, k) + m * f * b * (3 if case["keep"] else 1), "flops": 4 * m * f * k}
    if case["op"] == "gated_backward":
        return {"bytes": m * f * b * 5, "flops": 12 * m * f}
    return {"bytes": m * f * b * 3 + _stored(k, 2 * f) + _stored(k, m) + m * k * b + 2 * f * k * b, "flops": 8 * m * f * k}


def _stored(rows, cols):
    return rows * (cols + 4)        # codes and scales of a quantised matrix


# ------------------------------------------------------------------------------------------- inputs

def _gen(seed, tag):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 16 + tag)


def _normal(seed, tag, rows, cols):
    return torch.randn(rows, cols, generator=_gen(seed, tag), device="cuda")


def _activations(seed, tag, rows, cols, dtype):
    """Unit-variance features, a few channels larger, and the zero frames that pad a batch's utterances."""
    x = _normal(seed, tag, rows, cols)
    x[:, ::61] *= 8.0
    if rows >= 16:
        x[rows - rows // 16:] = 0.0
    return x.to(dtype)


def _gradients(seed, tag, rows, cols, dtype):
    """Loss-scaled gradients: magnitudes that differ from frame to frame, zero for padding."""
    x = _normal(seed, tag, rows, cols)
    x *= torch.exp2(torch.randint(-6, 3, (rows, 1), generator=_gen(seed, tag + 1), device="cuda").float())
    if rows >= 16:
        x[rows - rows // 16:] = 0.0
    return x.to(dtype)


def _weights(seed, tag, rows, cols):
    """Weight matrix of unit gain with outliers, one value in a hundred eight times as large."""
    x = _normal(seed, tag, rows, cols)
    big = torch.rand(rows, cols, generator=_gen(seed, tag + 1), device="cuda") < 0.01
    return x * torch.where(big, 8.0, 1.0) * (0.5 / math.sqrt(cols))


def _inputs(case, seed):
    t = _TYPES[case["type"]]
    op = case["op"]
    if op == "round_trip":
        r, c = case["rows"], case["cols"]
        return {"x": _weights(seed, 0, r, c).to(t) if case["both"] else _activations(seed, 0, r, c, t)}
    m, k = case["m"], case["k"]
    if op == "linear":
        return {"x": _activations(seed, 0, m, k, t), "w": _stored_of(_weights(seed, 1, case["n"], k))}
    if op == "linear_backward":
        # the weights along their other axis, and the layer's input along the frames, as the forward pass left them
        return {"dy": _gradients(seed, 0, m, case["n"], t), "wt": _stored_of(_weights(seed, 2, k, case["n"])),
                "xt": _stored_of(_activations(seed, 4, m, k, t).float().t().contiguous())}
    f = case["f"]
    if op == "gated":
        return {"x": _activations(seed, 0, m, k, t), "w": _stored_of(_weights(seed, 1, 2 * f, k))}
    d = {"dy": _gradients(seed, 0, m, f, t), "pre": _activations(seed, 6, m, 2 * f, t)}
    if op == "gated_step_backward":
        d["wt"] = _stored_of(_weights(seed, 2, k, 2 * f))
        d["xt"] = _stored_of(_activations(seed, 4, m, k, t).float().t().contiguous())
    return d


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        s.update(_buffers(case))
    return s


# ------------------------------------------------------------------------------------------- plain form

def _encode(x):
    """FP32 rows x cols -> (codes as FP32 whole numbers, FP32 scales)."""
    amax = x.abs().amax(1, keepdim=True)
    finite = torch.isfinite(amax)
    # (divided by a tensor: torch divides by a number by multiplying by its reciprocal, which rounds twice)
    s = torch.where(finite, (amax / torch.full_like(amax, 127.0)).clamp(min=2.0 ** -126), float("nan"))
    # the integer next to the product itself: 64 bits hold it whole
    q = (x.double() * (1.0 / s).double()).round()
    return torch.where(finite, q, 0.0).float(), s


def _stored_of(x):
    """The stored layout: (codes, scales)."""
    q, s = _encode(x)
    return torch.nn.functional.pad(q.to(torch.int8), (0, -x.shape[1] % 16)).contiguous(), s[:, 0].contiguous()


def _values(stored, cols):
    return stored[0][:, :cols].float() * stored[1][:, None]


def _rounded(x):
    """FP32 values of x after quantisation along the rows."""
    q, s = _encode(x)
    return q * s


def _act(name, a):
    if name == "gelu":
        return a * 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5)))
    g = 1.0 / (1.0 + torch.exp(-a))
    return a * g if name == "silu" else g


def _slope(name, a):
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5))) + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))
    g = 1.0 / (1.0 + torch.exp(-a))
    return g * (1.0 + a * (1.0 - g)) if name == "silu" else g * (1.0 - g)


def _plain(s):
    case = s["case"]
    t = _TYPES[case["type"]]
    op = case["op"]
    if op == "round_trip":
        x = s["x"].float()
        if not case["both"]:
            return _rounded(x).to(t)
        return _rounded(x).to(t), _rounded(x.t().contiguous()).to(t)
    m, k = case["m"], case["k"]
    if op == "linear":
        return (_rounded(s["x"].float()) @ _values(s["w"], k).t()).to(t)
    if op == "linear_backward":
        dy = s["dy"].float()
        dx = (_rounded(dy) @ _values(s["wt"], case["n"]).t()).to(t)
        return dx, _rounded(dy.t().contiguous()) @ _values(s["xt"], m).t()
    f = case["f"]
    if op == "gated":
        pre = _rounded(s["x"].float()) @ _values(s["w"], k).t()
        y = (_act(case["act"], pre[:, :f]) * pre[:, f:]).to(t)
        return (y, pre.to(t)) if case["keep"] else y
    # before a quantisation in 64 bits: codes follow the last bit of what they are made of
    wide = torch.float64 if op == "gated_step_backward" else torch.float32
    dy, a, b = s["dy"].to(wide), s["pre"][:, :f].to(wide), s["pre"][:, f:].to(wide)
    dpre = torch.cat((dy * b * _slope(case["act"], a), dy * _act(case["act"], a)), 1).to(t)
    if op == "gated_backward":
        return dpre
    dpre = dpre.float()
    dx = (_rounded(dpre) @ _values(s["wt"], 2 * f).t()).to(t)
    return dx, (_rounded(dpre.t().contiguous()) @ _values(s["xt"], m).t()).to(t)


# ------------------------------------------------------------------------------------------- the library's calls

def _code(case):
    import paper_2205_03494_b200 as omc
    return {"f32": omc.F32, "f16": omc.F16, "bf16": omc.BF16}[case["type"]]


def _gate(case):
    import paper_2205_03494_b200 as omc
    return {"sigmoid": omc.GATE_SIGMOID, "silu": omc.GATE_SILU, "gelu": omc.GATE_GELU}[case["act"]]


def _room(rows, cols):
    """Codes and scales of a quantised rows x cols matrix."""
    import paper_2205_03494_b200 as omc
    codes, scales = omc.byte_sizes(rows, cols)
    return torch.empty(codes, dtype=torch.uint8, device="cuda"), torch.empty(scales, dtype=torch.uint8, device="cuda")


def _buffers(case):
    """Outputs and workspaces, which a user's program keeps from call to call."""
    import paper_2205_03494_b200 as omc
    t, op = _TYPES[case["type"]], case["op"]
    new = lambda *shape, dtype=t: torch.empty(*shape, dtype=dtype, device="cuda")
    space = lambda n: new(n, dtype=torch.uint8)
    d = {"status": torch.zeros(4, dtype=torch.int32, device="cuda")}
    if op == "round_trip":
        r, c = case["rows"], case["cols"]
        d["q"], d["y"] = _room(r, c), new(r, c)
        d["workspace"] = space(omc.byte_quantise_workspace_bytes(r, c))
        if case["both"]:
            d["qt"], d["yt"] = _room(c, r), new(c, r)
        return d
    m, k = case["m"], case["k"]
    if op == "linear":
        d["y"], d["workspace"] = new(m, case["n"]), space(sum(omc.byte_sizes(m, k)))
    elif op == "linear_backward":
        n = case["n"]
        d["q"], d["qt"], d["workspace"] = _room(m, n), _room(n, m), space(omc.byte_quantise_workspace_bytes(m, n))
        d["dx"], d["dw"] = new(m, k), new(n, k, dtype=torch.float32)
    elif op == "gated":
        f = case["f"]
        d["y"], d["workspace"] = new(m, f), space(sum(omc.byte_sizes(m, k)))
        if case["keep"]:
            d["kept"] = new(m, 2 * f)
    elif op == "gated_backward":
        d["dpre"] = new(m, 2 * case["f"])
    else:
        f = case["f"]
        d["q"], d["qt"], d["workspace"] = _room(m, 2 * f), _room(2 * f, m), space(omc.gated_backward_workspace_bytes(m, f))
        d["dx"], d["dw"] = new(m, k), new(2 * f, k)
    return d


def _own(s):
    import paper_2205_03494_b200 as omc
    case = s["case"]
    op, ty = case["op"], _code(case)
    st = torch.cuda.current_stream().cuda_stream
    if op == "round_trip":
        r, c, q = case["rows"], case["cols"], s["q"]
        qt = s.get("qt")
        omc.byte_quantise(s["x"].data_ptr(), ty, r, c, c, q[0].data_ptr(), q[1].data_ptr(), qt[0].data_ptr() if qt else 0,
                        qt[1].data_ptr() if qt else 0, s["workspace"].data_ptr(), stream=st)
        omc.byte_dequantise(q[0].data_ptr(), q[1].data_ptr(), r, c, s["y"].data_ptr(), ty, c, stream=st)
        if not qt:
            return s["y"]
        omc.byte_dequantise(qt[0].data_ptr(), qt[1].data_ptr(), c, r, s["yt"].data_ptr(), ty, r, stream=st)
        return s["y"], s["yt"]
    m, k = case["m"], case["k"]
    if op == "linear":
        n = case["n"]
        omc.byte_linear(s["x"].data_ptr(), ty, m, k, k, s["w"][0].data_ptr(), s["w"][1].data_ptr(), n, s["y"].data_ptr(), ty, n,
                      s["workspace"].data_ptr(), s["status"].data_ptr(), stream=st)
        return s["y"]
    if op == "linear_backward":
        n, q, qt = case["n"], s["q"], s["qt"]
        omc.byte_quantise(s["dy"].data_ptr(), ty, m, n, n, q[0].data_ptr(), q[1].data_ptr(), qt[0].data_ptr(), qt[1].data_ptr(),
                        s["workspace"].data_ptr(), stream=st)
        omc.byte_matmul(q[0].data_ptr(), q[1].data_ptr(), m, s["wt"][0].data_ptr(), s["wt"][1].data_ptr(), k, n, s["dx"].data_ptr(), ty, k,
                      s["status"].data_ptr(), stream=st)
        omc.byte_matmul(qt[0].data_ptr(), qt[1].data_ptr(), n, s["xt"][0].data_ptr(), s["xt"][1].data_ptr(), k, m, s["dw"].data_ptr(), omc.F32, k,
                      s["status"].data_ptr(), stream=st)
        return s["dx"], s["dw"]
    f, act = case["f"], _gate(case)
    if op == "gated":
        kept = s.get("kept")
        omc.byte_gated_linear(s["x"].data_ptr(), ty, m, k, k, s["w"][0].data_ptr(), s["w"][1].data_ptr(), f, act, s["y"].data_ptr(), ty, f,
                            0 if kept is None else kept.data_ptr(), 2 * f, s["workspace"].data_ptr(), s["status"].data_ptr(), stream=st)
        return s["y"] if kept is None else (s["y"], kept)
    if op == "gated_backward":
        omc.gated_backward(s["dy"].data_ptr(), f, s["pre"].data_ptr(), 2 * f, ty, m, f, act, s["dpre"].data_ptr(), 2 * f, stream=st)
        return s["dpre"]
    q, qt = s["q"], s["qt"]
    omc.gated_backward(s["dy"].data_ptr(), f, s["pre"].data_ptr(), 2 * f, ty, m, f, act, 0, 0, q[0].data_ptr(), q[1].data_ptr(),
                       qt[0].data_ptr(), qt[1].data_ptr(), s["workspace"].data_ptr(), stream=st)
    omc.byte_matmul(q[0].data_ptr(), q[1].data_ptr(), m, s["wt"][0].data_ptr(), s["wt"][1].data_ptr(), k, 2 * f, s["dx"].data_ptr(), ty, k,
                  s["status"].data_ptr(), stream=st)
    omc.byte_matmul(qt[0].data_ptr(), qt[1].data_ptr(), 2 * f, s["xt"][0].data_ptr(), s["xt"][1].data_ptr(), k, m, s["dw"].data_ptr(), ty, k,
                  s["status"].data_ptr(), stream=st)
    return s["dx"], s["dw"]


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------- the definition in 64 bits

def _quantised64(x):
    """Values of the 8-bit format nearest to x (FP64, one scale a row).  Scale and reciprocal are FP32 numbers."""
    top = torch.maximum(x.max(1).values, -x.min(1).values)
    scale = torch.clamp(top / torch.full_like(top, 127.0), min=2.0 ** -126).float().double()
    inverse = (1 / scale).float().double()
    u = x * inverse[:, None]
    low = torch.floor(u)
    up = (u - low > 0.5) | ((u - low == 0.5) & (torch.remainder(low, 2) == 1))
    return (low + up) * scale[:, None]


def _stored64(stored, cols):
    """FP64 values of a stored matrix."""
    return torch.einsum("rc,r->rc", stored[0][:, :cols].double(), stored[1].double())


def _sigmoid64(a):
    return 0.5 * (1 + torch.tanh(a / 2))


def _normal64(a):
    return 0.5 * torch.erfc(-a / math.sqrt(2))


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "round_trip":
        x = s["x"].double()
        return (_quantised64(x), _quantised64(x.t().contiguous())) if case["both"] else _quantised64(x)
    m, k = case["m"], case["k"]
    if op == "linear":
        return _quantised64(s["x"].double()) @ _stored64(s["w"], k).t()
    if op == "linear_backward":
        dy = s["dy"].double()
        return (_quantised64(dy) @ _stored64(s["wt"], case["n"]).t(), _quantised64(dy.t().contiguous()) @ _stored64(s["xt"], m).t())
    f, act = case["f"], case["act"]
    gate = {"sigmoid": _sigmoid64, "silu": lambda a: a * _sigmoid64(a), "gelu": lambda a: a * _normal64(a)}[act]
    if op == "gated":
        pre = _quantised64(s["x"].double()) @ _stored64(s["w"], k).t()
        y = gate(pre[:, :f]) * pre[:, f:]
        return (y, pre) if case["keep"] else y
    # derivatives of the gate
    slope = {"sigmoid": lambda a: _sigmoid64(a) * _sigmoid64(-a),
             "silu": lambda a: _sigmoid64(a) + a * _sigmoid64(a) * _sigmoid64(-a),
             "gelu": lambda a: _normal64(a) + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)}[act]
    a, b = torch.split(s["pre"].double(), f, 1)
    dy = s["dy"].double()
    dpre = torch.empty(m, 2 * f, dtype=torch.float64, device="cuda")
    dpre[:, :f] = slope(a) * b * dy
    dpre[:, f:] = gate(a) * dy
    if op == "gated_backward":
        return dpre
    # the gradient that the layer quantises is a matrix of the activations' type
    dpre = dpre.to(_TYPES[case["type"]]).double()
    return _quantised64(dpre) @ _stored64(s["wt"], 2 * f).t(), _quantised64(dpre.t().contiguous()) @ _stored64(s["xt"], m).t()
