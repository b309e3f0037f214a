"""Pins of the 4-bit microscaled format's definition (mx_reference.py), and the plain form of perf/operators.py against it.
No GPU needed."""
import os
import sys

import numpy as np
import torch

import mx_reference as mx

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "perf"))


def test_values_and_ties():
    # scale 1 (largest magnitude 4): every value of the format, the ties between them, what saturates
    x = np.zeros((1, 32))
    x[0, :15] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 4.0, -0.25, -0.75, -2.5, -3.5, 0.26, 0.74, 3.49, -0.0]
    codes, scales = mx.encode(x)
    assert scales.tolist() == [[127]]
    assert mx.decode(codes, scales, 32)[0, :15].tolist() == [0, 1, 1, 2, 2, 4, 4, -0.0, -1, -2, -4, 0.5, 0.5, 3, -0.0]
    assert codes[0, 14] == 8                                   # -0 keeps its sign
    x[0, 0] = 7.9                                              # below 8: the scale stays, the value saturates
    assert mx.quantised(x)[0, 0] == 6.0
    x[0, 0] = 8.0
    assert mx.encode(x)[1].tolist() == [[128]] and mx.quantised(x)[0, 0] == 8.0


def test_blocks_of_their_own():
    x = np.ones((2, 70))
    x[0, 31], x[0, 32], x[1, 69] = np.inf, 2.0 ** 100, np.nan
    codes, scales = mx.encode(x)
    assert scales.tolist() == [[255, 225, 125], [125, 125, 255]]
    v = mx.decode(codes, scales, 70)
    assert np.isnan(v[0, :32]).all() and v[0, 32] == 2.0 ** 100 and (v[0, 33:64] == 0).all() and (v[1, :64] == 1).all()
    assert mx.encode(np.full((1, 3), 2.0 ** -140))[1].tolist() == [[0]]      # the scale is at least 2^-127
    assert mx.encode(np.zeros((1, 3)))[1].tolist() == [[0]]


def test_stored_places():
    offs = mx.scale_offsets(300, 1000)
    assert offs.shape == (300, 32) and len(np.unique(offs)) == offs.size and offs.max() < 3 * 4 * 1024
    assert offs[0].tolist()[:9] == [0, 1, 2, 3, 512, 513, 514, 515, 1024]
    assert [int(offs[r, 0]) for r in (1, 31, 32, 64, 127, 128)] == [16, 496, 4, 8, 508, 4096]
    packed, _ = mx.pack(np.arange(32, dtype=np.uint8)[None] % 16, np.array([[127]], np.uint8), 32)
    assert packed[:4].tolist() == [0x10, 0x32, 0x54, 0x76]


def test_plain_form_of_the_measured_cases():
    import operators as op
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((130, 300)) * 2.0 ** rng.integers(-30, 30, (130, 1))).astype(np.float32)
    x[3], x[4, 5], x[6], x[7, 299] = 0, np.nan, np.finfo(np.float32).tiny / 4, np.inf
    codes, scales = op._encode(torch.from_numpy(x))
    want_codes, want_scales = mx.encode(x)
    assert np.array_equal(codes.numpy(), want_codes) and np.array_equal(scales.numpy(), want_scales)
    stored = op._pack(codes, scales)
    want = mx.pack(want_codes, want_scales, 300)
    assert all(np.array_equal(a.numpy(), b) for a, b in zip(stored, want))
    assert np.array_equal(op._unpack(stored, 130, 300).numpy().astype(np.float64), mx.decode(want_codes, want_scales, 300), equal_nan=True)
