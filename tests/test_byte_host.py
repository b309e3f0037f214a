"""What the 8-bit and gated operators refuse, their sizes, and what their Python entry points take.  Checked before anything touches a device: no GPU
needed."""
import numpy as np
import pytest

import paper_2205_03494_b200 as omc
from test_layer_host import A, INVALID, MISALIGNED, NULL, refused


def test_sizes():
    assert omc.byte_sizes(1, 1) == (16, 16)
    assert omc.byte_sizes(5, 16) == (80, 32)
    assert omc.byte_sizes(129, 257) == (129 * 272, 528)
    for rows, cols in ((0, 5), (5, 0), (1 << 31, 1), (1, 1 << 31)):
        refused(INVALID, omc.byte_sizes, rows, cols)
        refused(INVALID, omc.byte_quantise_workspace_bytes, rows, cols)
        refused(INVALID, omc.gated_backward_workspace_bytes, rows, cols)
    refused(INVALID, omc.gated_backward_workspace_bytes, 4, 1 << 30)
    assert omc.lib().omc_byte_sizes(4, 4, None, None) == 0
    assert omc.lib().omc_byte_quantise_workspace(4, 4, None) == NULL and omc.lib().omc_gated_backward_workspace(4, 4, None) == NULL
    assert omc.byte_quantise_workspace_bytes(10 ** 6, 2048) % 16 == 0


def test_quantise_refusals():
    ok = dict(x=A, type_=omc.F16, rows=4, cols=64, ld=64, codes=A, scales=A, codes_t=A, scales_t=A, workspace=A)
    for name in ("x", "codes", "scales", "codes_t", "scales_t", "workspace"):
        refused(NULL, omc.byte_quantise, **{**ok, name: 0})
    refused(NULL, omc.byte_quantise, **{**ok, "codes": 0, "scales": 0, "codes_t": 0, "scales_t": 0})
    for bad in (dict(type_=3), dict(type_=-1), dict(rows=0), dict(cols=0), dict(ld=63), dict(rows=1 << 31)):
        refused(INVALID, omc.byte_quantise, **{**ok, **bad})
    for bad in (dict(x=A + 1), dict(codes=A + 8), dict(scales=A + 2), dict(codes_t=A + 8), dict(scales_t=A + 1), dict(workspace=A + 8)):
        refused(MISALIGNED, omc.byte_quantise, **{**ok, **bad})
    ok = dict(codes=A, scales=A, rows=4, cols=64, out=A, type_=omc.F32, ld=64)
    for name in ("codes", "scales", "out"):
        refused(NULL, omc.byte_dequantise, **{**ok, name: 0})
        refused(MISALIGNED, omc.byte_dequantise, **{**ok, name: A + 2})
    for bad in (dict(type_=9), dict(rows=0), dict(cols=0), dict(ld=60)):
        refused(INVALID, omc.byte_dequantise, **{**ok, **bad})


def test_product_refusals():
    ok = dict(x_codes=A, x_scales=A, M=4, w_codes=A, w_scales=A, N=8, K=64, y=A, type_=omc.F32, ldy=8, status=A)
    gated = {**{k: v for k, v in ok.items() if k != "N"}, "F": 8, "activation": omc.GATE_SILU, "pre": A, "ld_pre": 16}
    for fn, args, width in ((omc.byte_matmul, ok, "N"), (omc.byte_gated, gated, "F")):
        for name in ("x_codes", "x_scales", "w_codes", "w_scales", "y", "status"):
            refused(NULL, fn, **{**args, name: 0})
            refused(MISALIGNED, fn, **{**args, name: A + 2})
        for bad in ({"M": 0}, {width: 0}, {"K": 0}, {"K": 1 << 17}, {"ldy": 7}, {"type_": 7}, {"M": 128 * 65535 + 1}):
            refused(INVALID, fn, **{**args, **bad})
    ok = dict(x=A, type_=omc.BF16, M=4, K=64, ldx=64, w_codes=A, w_scales=A, N=8, y=A, y_type=omc.F32, ldy=8, workspace=A, status=A)
    gated_linear = {**{k: v for k, v in ok.items() if k != "N"}, "F": 8, "activation": omc.GATE_SILU, "pre": A, "ld_pre": 16}
    for fn, args, width in ((omc.byte_linear, ok, "N"), (omc.byte_gated_linear, gated_linear, "F")):
        for name in ("x", "w_codes", "w_scales", "y", "workspace", "status"):
            refused(NULL, fn, **{**args, name: 0})
            refused(MISALIGNED, fn, **{**args, name: A + 1})
        for bad in ({"M": 0}, {width: 0}, {"K": 0}, {"K": 1 << 17, "ldx": 1 << 17}, {"ldx": 63}, {"ldy": 7}, {"type_": 7}, {"y_type": -2}):
            refused(INVALID, fn, **{**args, **bad})
    for fn, args in ((omc.byte_gated, gated), (omc.byte_gated_linear, gated_linear)):
        for bad in ({"activation": 3}, {"activation": -1}, {"ld_pre": 15}, {"F": 1 << 30, "ldy": 1 << 30, "ld_pre": 1 << 31}):
            refused(INVALID, fn, **{**args, **bad})
        refused(MISALIGNED, fn, **{**args, "pre": A + 2})
    for polls, what in ((0, 1), ((1 << 16) + 1, 1), (5, 0), (5, 3)):
        refused(INVALID, omc.byte_inject_wait_timeout, polls, what)


def test_gated_backward_refusals():
    far = dict(dy=1 << 20, pre=2 << 20, dpre=3 << 20)
    ok = dict(**far, ld_dy=8, ld_pre=16, type_=omc.F32, rows=4, F=8, activation=omc.GATE_GELU, ld_dpre=16, codes=A, scales=A, codes_t=A, scales_t=A, workspace=A)
    for name in ("dy", "pre", "codes", "scales", "codes_t", "scales_t", "workspace"):
        refused(NULL, omc.gated_backward, **{**ok, name: 0})
    refused(NULL, omc.gated_backward, **{**ok, "dpre": 0, "codes": 0, "scales": 0, "codes_t": 0, "scales_t": 0})
    for name in ("dy", "pre", "dpre", "codes", "scales", "codes_t", "scales_t", "workspace"):
        refused(MISALIGNED, omc.gated_backward, **{**ok, name: ok[name] + 2})
    for bad in (dict(type_=4), dict(rows=0), dict(F=0), dict(F=1 << 30), dict(activation=3), dict(ld_dy=7), dict(ld_pre=15), dict(ld_dpre=15),
                dict(dpre=far["dy"]), dict(dpre=far["pre"]), dict(dpre=far["pre"] + 4 * (3 * 16 + 15)), dict(dpre=far["dy"] - 4 * (3 * 16 + 15))):
        refused(INVALID, omc.gated_backward, **{**ok, **bad})


class Whole:
    def __init__(self, v):
        self.v = v

    def __index__(self):
        return self.v


def calls(n):
    """Every call with n() around its integers, the first address missing."""
    z, a = n(0), n(A)
    return [
        (omc.byte_quantise, (z, n(1), n(4), n(64), n(64), a, a, z, z, z, z)),
        (omc.byte_dequantise, (z, a, n(4), n(64), a, n(1), n(64), z)),
        (omc.byte_matmul, (z, a, n(4), a, a, n(8), n(64), a, n(0), n(8), a, z)),
        (omc.byte_linear, (z, n(1), n(4), n(64), n(64), a, a, n(8), a, n(0), n(8), a, a, z)),
        (omc.byte_gated, (z, a, n(4), a, a, n(8), n(64), n(1), a, n(0), n(8), a, n(16), a, z)),
        (omc.byte_gated_linear, (z, n(1), n(4), n(64), n(64), a, a, n(8), n(1), a, n(0), n(8), a, n(16), a, a, z)),
        (omc.gated_backward, (z, n(8), a, n(16), n(1), n(4), n(8), n(1), a, n(16), a, a, a, a, a, z)),
    ]


@pytest.mark.parametrize("n", [int, np.int64, np.uint64, np.int32, Whole], ids=lambda n: n.__name__)
def test_integers_of_every_kind(n):
    assert omc.byte_sizes(n(4), n(64)) == (256, 16)
    for fn, args in calls(n):
        refused(NULL, fn, *args)


def test_what_is_no_address_or_no_integer():
    for fn, args in calls(int):
        refused(NULL, fn, None, *args[1:])
        for at in range(len(args)):
            for bad, error in ((4.0, TypeError), ("4", TypeError), (1 << 64, OverflowError), (Whole(-(1 << 70)), OverflowError)):
                with pytest.raises(error):
                    fn(*args[:at], bad, *args[at + 1:])
