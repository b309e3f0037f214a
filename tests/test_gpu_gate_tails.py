"""The gated layer where its activations are small: results relative to themselves, far into the tails, against the formulas in 64 bits.

Errors in units u = 2^-23, relative; the hardware's exponential of 2 is off by 2 of its last places and its reciprocal by 1 (at most u each).
  e = e^-|a| or e^(-a^2 / 2), as the square of its root: 2 twice, the square's half, and half for what the exponent's rounding left out: 5.  Where the result has 16
      bits that is not done: the exponent's half and its constant's 0.11 make |a| 0.61 instead, a^2 / 2 those and the square's half, a^2 0.56.
  P: the tail Q e has a polynomial Q off by 0.6 where it is exact, and by 4.4 with its roundings and those of t; e's and a product's half.  Above 0
      P = 1 - tail, the tail being the smaller one, and half a unit more: e's + 5.4.
  r = 1 / (1 + e): e's error enters with e / (1 + e) <= 1 / (1 + e); the sum's half and the reciprocal's 1: e's + 1.5.
  The larger one of s and 1 - s is r; the smaller one e r: e's error with 1 / (1 + e), the other two, and a product's half: e's + 2.
  y = act(a) b, act = a P or a s: two products, half a unit each (of the sigmoid one).
Absolute: where e^-|a| is no normal number it is off by a subnormal step of FP32 or two, and s with it; where the result has 16 bits it is then 0."""
import numpy as np
import pytest
import torch

import i8_reference as i8
import paper_2205_03494_b200 as omc
from test_gpu_i8 import stored
from test_gpu_mx import TYPES, UNIT, host, stream

pytestmark = pytest.mark.gpu
U = 2.0 ** -23
LEAST = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}      # the smallest subnormal
ACTS = {"sigmoid": omc.GATE_SIGMOID, "silu": omc.GATE_SILU, "gelu": omc.GATE_GELU}


def e_units(name, a, ty):
    if ty == "f32":
        return 5.0
    return 4.5 + (0.56 * a * a if name == "gelu" else 0.61 * np.abs(a))


def least_of(ty):
    """Absolute error of s and 1 - s."""
    return 3 * LEAST["f32"] if ty == "f32" else 2.0 ** -126


def act_units(name, a, ty):
    """Relative error of act(a), in u."""
    return e_units(name, a, ty) + {"gelu": 5.4 + 0.5, "sigmoid": 2.0, "silu": 2.0 + 0.5}[name]


def gated(M, low, high, name, ty, value=1.0):
    """M frames whose gates run from low to high, all with about the same value: y, and the FP32 gates and values."""
    code, dtype = TYPES[ty]
    F, K = 500, 16
    x, w = np.zeros((M, K), np.float32), np.zeros((2 * F, K), np.float32)
    x[:, 0], x[:, 1] = 1.0, 0.5
    w[:F, 0], w[F:, 1] = np.linspace(low, high, F), np.linspace(value, 2 * value, F)
    x[:, 0] += np.linspace(0, 0.5, M)
    xc, xs, xq, xsc = stored(x)
    wc, ws, wq, wsc = stored(w)
    pre = i8.product(xq, xsc, wq, wsc).astype(np.float64)
    status, y = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty(M, F, dtype=dtype, device="cuda")
    omc.byte_gated(xc.data_ptr(), xs.data_ptr(), M, wc.data_ptr(), ws.data_ptr(), F, K, ACTS[name], y.data_ptr(), code, F, 0, 0, status.data_ptr(), stream=stream())
    got = host(y)
    assert int(status[0]) == 0
    return got, pre[:, :F], pre[:, F:]


def check_relative(got, want, units, ty, least):
    """Relative: `units` u and half a step of the type; absolute: `least`, and a subnormal step of the type.  What rounds past the type's largest value is infinite."""
    past = float(torch.finfo(TYPES[ty][1]).max) * (1 + UNIT[ty])
    got, want = np.where(np.isinf(got), np.copysign(past, got), got), np.clip(want, -past, past)
    bound = np.abs(want) * (1.01 * units * U + 1.01 * UNIT[ty]) + least + LEAST[ty]
    err = np.abs(got - want)
    assert not np.isnan(got).any()
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("M", [3, 40, 2000])          # each of the products' kernels
def test_gelu_tails_forward(M, ty):
    for low, high in ((-8.0, 4.0), (-1.0, 1.0)):
        y, a, b = gated(M, low, high, "gelu", ty, 1024.0)
        assert a.min() < low + 0.1 and (np.abs(b) > 500).all()
        check_relative(y, i8.act("gelu", a) * b, act_units("gelu", a, ty) + 0.5, ty, 0.0)


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("name", ["sigmoid", "silu"])
@pytest.mark.parametrize("M", [3, 40, 2000])
def test_sigmoid_tails_forward(M, name, ty):
    for low, high in ((-100.0, 10.0), (-16.0, 16.0)):
        y, a, b = gated(M, low, high, name, ty, 1024.0 if ty == "f16" else 2.0 ** 70)
        check_relative(y, i8.act(name, a) * b, act_units(name, a, ty) + 0.5, ty, least_of(ty) * np.maximum(np.abs(a), 1) * np.abs(b))


def backward(dy, pre, name, ty):
    code, dtype = TYPES[ty]
    rows, F = dy.shape
    d, p = (torch.from_numpy(v).to(dtype).cuda() for v in (dy, pre))
    out = torch.empty(rows, 2 * F, dtype=dtype, device="cuda")
    omc.gated_backward(d.data_ptr(), F, p.data_ptr(), 2 * F, code, rows, F, ACTS[name], out.data_ptr(), 2 * F, stream=stream())
    return host(out), host(d), host(p)[:, :F], host(p)[:, F:]


def problem(F, low, high, scale):
    """Gates from low to high, values and gradients of one order of magnitude."""
    rng = np.random.default_rng(F)
    rows = 40
    dy, b = (rng.uniform(1, 2, (rows, F)) * rng.choice([-1.0, 1.0], (rows, F)) for _ in range(2))
    return dy * scale, np.concatenate([np.linspace(low, high, rows * F).reshape(rows, F), b], 1)


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("F", [512, 333])
def test_gelu_tails_backward(F, ty):
    """dy act(a) as the forward pass; dy b act'(a) with act' = P + a phi: P's units of P; of a phi e's, the constant's half and a product's; half of the sum;
    and two products' halves."""
    got, dy, a, b = backward(*problem(F, -8.0, 4.0, 1024.0), "gelu", ty)
    check_relative(got[:, F:], dy * i8.act("gelu", a), act_units("gelu", a, ty) + 0.5, ty, 0.0)
    tail = np.abs(a) * np.exp(-0.5 * a * a) / np.sqrt(2 * np.pi)
    slope = i8.slope("gelu", a)
    units = e_units("gelu", a, ty)
    own = i8.cdf(a) * (units + 5.4) + tail * (units + 1) + np.abs(slope) * 1.5
    check_relative(got[:, :F], dy * b * slope, 0.0, ty, np.abs(dy * b) * own * 1.01 * U)


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("F", [512, 333])
def test_sigmoid_tails_backward(F, ty):
    """act' = s t, t = 1 - s: e's units and 2 of one, 1.5 of the other (into which e's enter with e / (1 + e), into the first with 1 / (1 + e)), the product's half, and two
    products more."""
    for low, high in ((-100.0, 100.0), (-6.0, 18.0)):
        got, dy, a, b = backward(*problem(F, low, high, 1024.0 if ty == "f16" else 2.0 ** 40), "sigmoid", ty)
        least = least_of(ty) * np.abs(dy) * np.maximum(np.abs(b), 1)
        check_relative(got[:, :F], dy * b * i8.slope("sigmoid", a), e_units("sigmoid", a, ty) + 3.5 + 1.5, ty, least)
        check_relative(got[:, F:], dy * i8.act("sigmoid", a), act_units("sigmoid", a, ty) + 0.5, ty, least)


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("F", [512, 333])
def test_silu_tails_backward(F, ty):
    """act' = s (1 + a t): t's units (e's and 2) of s |a| t; of the whole s's, the sum's half, the product's half, and two products more.  Where the result has 16 bits as
    (a s) t + s: of s |a| t both factors' units, of s its own; of the whole the sum's half, and two products."""
    for low, high in ((-100.0, 100.0), (-16.0, 30.0)):
        got, dy, a, b = backward(*problem(F, low, high, 1024.0 if ty == "f16" else 2.0 ** 40), "silu", ty)
        least = least_of(ty) * np.abs(dy) * np.maximum(np.abs(b), 1) * np.maximum(np.abs(a), 1)
        want = dy * b * i8.slope("silu", a)
        units = e_units("silu", a, ty) + 2
        s, t = i8.sigmoid(a), i8.sigmoid(-a)
        own = s * np.abs(a) * t * units if ty == "f32" else s * np.abs(a) * t * (2 * units + 0.5) + s * units
        check_relative(got[:, :F], want, units + 2 if ty == "f32" else 1.5, ty, least + np.abs(dy * b) * own * 1.01 * U)
        check_relative(got[:, F:], dy * i8.act("silu", a), act_units("silu", a, ty) + 0.5, ty, least)


def half_step(x, dtype):
    """Half the distance of the neighbours of FP64 values in a 16-bit type, normal numbers."""
    _, e = np.frexp(x)
    return np.ldexp(float(torch.finfo(dtype).eps) / 4, e)


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_open_gates_next_to_ties(name, ty):
    """Where act(a) / a and act'(a) are next to 1 the gradients are g a and g b times almost 1, which lie on ties of the result for many 16-bit g, a and b, and next to them
    a little further down.  The result is the nearer one wherever the formula's value is further from the middle than: of a 1 - t and of the slope the last rounding, a quarter
    of a u and half of one, of a P or a s another half, of the last product another; and next to nothing of the tails (2.7e-3 of themselves below, off by 8 u + 0.7 a u, or
    GELU's at a = 4, 2.1e-3, 22 u)."""
    _, dtype = TYPES[ty]
    low, high = (8.0, 24.0) if name == "silu" else (4.0, 7.0)
    a = np.unique(torch.linspace(low, high, 600).to(dtype).double().numpy())
    g = np.unique(torch.linspace(1.0, 2.0, 300).to(dtype).double().numpy())[:-1]
    for b in (1.0, 1.0078125, 1.2578125, 1.5234375, 1.9921875):
        pre = np.concatenate([np.broadcast_to(a, (len(g), len(a))), np.full((len(g), len(a)), b)], 1)
        got, dy, av, bv = backward(np.broadcast_to(g[:, None], (len(g), len(a))).copy(), pre, name, ty)
        for part, want in ((got[:, :len(a)], dy * bv * i8.slope(name, av)), (got[:, len(a):], dy * i8.act(name, av))):
            assert (np.abs(part - want) <= half_step(want, dtype) + np.abs(want) * (1.25 + 0.1) * U).all(), float(((np.abs(part - want) - half_step(want, dtype)) / np.abs(want)).max() / U)


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("name", list(ACTS))
def test_gates_far_out_and_infinite(name, ty):
    """Gates from 200 up to the type's largest, of both signs: the activation and its slope are their limits.  An infinite gate or value makes its own two gradients what
    the formula gives for it (Inf or NaN, or a limit), and nothing else."""
    code, dtype = TYPES[ty]
    rows, F = 24, 48
    rng = np.random.default_rng(3)
    top = float(torch.finfo(dtype).max)
    far = np.concatenate([[200.0, 1000.0, 30000.0, top], np.geomspace(200.0, top, F - 4)])
    a = np.where(np.arange(rows)[:, None] % 2, -far, far)
    dy, b = (rng.choice([0.5, 0.25, -0.5], (rows, F)) for _ in range(2))
    got, g, av, bv = backward(dy, np.concatenate([a, b], 1), name, ty)
    near = lambda got, want: (np.abs(got - want) <= np.abs(want) * 1.01 * UNIT[ty]).all()
    if name == "sigmoid":
        assert (got[:, :F] == 0).all() and near(got[:, F:], np.where(av > 0, g, 0.0))
    else:
        assert near(got[:, :F], np.where(av > 0, g * bv, 0.0)) and near(got[:, F:], np.where(av > 0, g * av, 0.0))
    pre = np.concatenate([rng.standard_normal((rows, F)), b], 1)
    want, *_ = backward(dy, pre, name, ty)
    pre[3, 7], pre[4, 8], pre[10, F + 5], pre[11, F + 6] = np.inf, -np.inf, np.inf, -np.inf
    got, g, av, bv = backward(dy, pre, name, ty)
    own = np.zeros((rows, 2 * F), bool)
    for r, c in ((3, 7), (4, 8), (10, 5), (11, 6)):
        own[r, [c, c + F]] = True
    assert np.array_equal(got[~own], want[~own])
    # (value: da is infinite, db as it was.  Gate: the sigmoid's limits; a or a P times 0 is NaN, or its limit)
    assert np.isinf(got[[10, 11], [5, 6]]).all() and np.array_equal(got[[10, 11], [F + 5, F + 6]], want[[10, 11], [F + 5, F + 6]])
    if name == "sigmoid":
        assert (got[[3, 4], [7, 8]] == 0).all() and got[3, F + 7] == dy[3, 7] and got[4, F + 8] == 0
    else:
        assert np.isinf(got[3, F + 7]) and all(np.isnan(v) or v == 0 for v in (got[4, 8], got[4, F + 8])) and (np.isnan(got[3, 7]) or got[3, 7] == g[3, 7] * bv[3, 7])
