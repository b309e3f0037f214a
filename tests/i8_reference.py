"""The 8-bit integer format and the gated layer from their definitions, in 64 bits."""
import math

import numpy as np
import torch

LEAST = np.float32(2.0 ** -126)
ACTS = {"sigmoid": 0, "silu": 1, "gelu": 2}


def encode(x):
    """x (FP64 values of a 32- or 16-bit type) -> codes (int8, rows x cols), scales (float32, rows)."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(1)
    finite = np.isfinite(top)
    # (a quotient of FP32 numbers taken in FP64 and rounded to FP32 is the FP32 quotient)
    s = np.maximum((np.where(finite, top, 1.0) / 127.0).astype(np.float32), LEAST)
    r = (1.0 / s.astype(np.float64)).astype(np.float32)
    with np.errstate(invalid="ignore"):
        q = np.rint(np.where(finite[:, None], x, 0.0) * r.astype(np.float64)[:, None])       # 24 x 24 bits: the product is exact
    assert np.abs(q).max() <= 127
    return q.astype(np.int8), np.where(finite, s, np.float32("nan"))


def pack(codes):
    """The stored layout, flat."""
    rows, cols = codes.shape
    out = np.zeros((rows, -(-cols // 16) * 16), np.int8)
    out[:, :cols] = codes
    return out.reshape(-1)


def values(codes, scales):
    return codes.astype(np.float32) * scales[:, None]


def product(xc, xs, wc, ws):
    """FP32 values of the product: (sum * sx) * sw, each step rounded; the first one as if FP32 had no largest value."""
    total = (xc.astype(np.float64) @ wc.astype(np.float64).T).astype(np.int64)       # whole numbers below 2^53: exact
    assert np.abs(total).max() < 2 ** 31
    with np.errstate(over="ignore", invalid="ignore"):
        sx = xs.astype(np.float64)
        big = sx >= 2.0 ** 64
        f, g = np.where(big, sx * 2.0 ** -64, sx).astype(np.float32), np.where(big, np.float32(2.0 ** 64), np.float32(1.0))
        return total.astype(np.float32) * f[:, None] * ws[None, :] * g[:, None].astype(np.float32)


def sigmoid(a):
    e = np.exp(-np.abs(a))
    return np.where(a >= 0, 1.0, e) / (1.0 + e)


def cdf(a):
    return 0.5 * torch.erfc(torch.from_numpy(-np.asarray(a) / math.sqrt(2.0))).numpy()


def act(name, a):
    return {"sigmoid": sigmoid, "silu": lambda v: v * sigmoid(v), "gelu": lambda v: v * cdf(v)}[name](a)


def slope(name, a):
    density = np.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
    return {"sigmoid": lambda v: sigmoid(v) * sigmoid(-v), "silu": lambda v: sigmoid(v) * (1 + v * sigmoid(-v)),
            "gelu": lambda v: cdf(v) + v * density}[name](a)


# Errors of the kernels' activations, from the error bounds of CUDA's functions: __expf(x) is off by 2 + 1.173 |x| units (2^-23 relative),
# __fdividef by 2, erff by 2; every other operation by half a unit.

def sigmoid_error(a):
    """Relative error of s = 1 / (1 + e^-a): e's, weakened by e / (1 + e) <= 1, the addition's and the quotient's.  Where 1 + e passes 2^126
    the quotient is 0 instead of a number below 2^-126 (that is added separately, as an absolute error)."""
    return (2 + 1.173 * np.abs(a) + 0.5 + 2) * 2.0 ** -23


def cdf_error(a):
    """Absolute error of P = (1 + erf(a / sqrt 2)) / 2: erf's 2 units of at most 1, its argument's two half units (of the factor and of the
    product) times max |x erf'(x)| < 0.49, both halved, and the last sum's half unit."""
    return (0.5 * (2 + 0.49) + 0.5) * 2.0 ** -23 * np.ones_like(a)


def act_error(name, a):
    """Absolute error of act(a), the last product's half unit included."""
    if name == "gelu":
        return np.abs(a) * cdf_error(a) + np.abs(act(name, a)) * 2.0 ** -24
    s = sigmoid(a)
    own = s * sigmoid_error(a) + 2.0 ** -126
    return own if name == "sigmoid" else np.abs(a) * own + np.abs(a) * s * 2.0 ** -24


def slope_error(name, a):
    """Absolute error of act'(a).  GELU: P's, and of a 0.3989 e^(-a^2 / 2) the exponential's (its argument is off by two half units of a^2 / 2), the factor's,
    two products' and the sum's.  Others: with s off by es and t = 1 - s by s es + half a unit of t, s t by their sum; 1 + a t by a times t's error and
    half a unit of itself, s (1 + a t) by that times s, es of itself and half a unit."""
    if name == "gelu":
        tail = np.abs(a) * np.exp(-0.5 * a * a) * 0.39894228
        return cdf_error(a) + tail * (2 + 1.173 * 0.5 * a * a + 0.5 * a * a + 2) * 2.0 ** -23 + np.abs(slope(name, a)) * 2.0 ** -24
    s, t = sigmoid(a), sigmoid(-a)
    es = sigmoid_error(a) + 2.0 ** -126
    et = s * es + t * 2.0 ** -24
    if name == "sigmoid":
        return s * t * (es + 2.0 ** -24) + s * et
    inner = 1 + a * t
    return s * (np.abs(a) * et + np.abs(inner) * 2.0 ** -24) + s * np.abs(inner) * (es + 2.0 ** -24) + 2.0 ** -126 * (1 + np.abs(a))
