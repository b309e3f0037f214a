"""The gated layer where its activations are small: results relative to themselves, far into the tails, against the formulas in 64 bits.

Errors in units u = 2^-23, relative; the hardware's exponential of 2 is off by 2 of its last places and its reciprocal by 1 (at most u each).
  e = e^(-a^2 / 2): 2 and a last sum's half, the exponent being held in two numbers.
  P: the tail Q e has a polynomial Q off by 0.6 where it is exact, and by 4.4 with its roundings and those of t; e's 2.5 and a product's half: 7.5.  Above 0
      P = 1 - tail, the tail being the smaller one, and half a unit more: 8.
  y = a P b: two products, half a unit each."""
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


def act_units(name, a):
    """Relative error of act(a), in u."""
    return 8 + 0.5 + 0 * a


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
    """Relative: `units` u and half a step of the type; absolute: `least`, and a subnormal step of the type."""
    bound = np.abs(want) * (1.01 * units * U + 1.01 * UNIT[ty]) + least + LEAST[ty]
    err = np.abs(got - want)
    assert np.isfinite(got).all()
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("M", [3, 40, 2000])          # each of the products' kernels
def test_gelu_tails_forward(M, ty):
    for low, high in ((-8.0, 4.0), (-1.0, 1.0)):
        y, a, b = gated(M, low, high, "gelu", ty, 1024.0)
        assert a.min() < low + 0.1 and (np.abs(b) > 500).all()
        check_relative(y, i8.act("gelu", a) * b, act_units("gelu", a) + 0.5, ty, 0.0)


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
    """dy act(a) as the forward pass; dy b act'(a) with act' = P + a phi: P's 8 of P; of a phi e's 2.5, the constant's half and a product's; half of the sum;
    and two products' halves."""
    got, dy, a, b = backward(*problem(F, -8.0, 4.0, 1024.0), "gelu", ty)
    check_relative(got[:, F:], dy * i8.act("gelu", a), act_units("gelu", a) + 0.5, ty, 0.0)
    tail = np.abs(a) * np.exp(-0.5 * a * a) / np.sqrt(2 * np.pi)
    slope = i8.slope("gelu", a)
    own = i8.cdf(a) * 8 + tail * 3.5 + np.abs(slope) * 1.5
    check_relative(got[:, :F], dy * b * slope, 0.0, ty, np.abs(dy * b) * own * 1.01 * U)
