"""What the layer operators refuse, and their sizes.  Checked before anything touches a device: no GPU needed."""
import ctypes as C

import pytest

import paper_2205_03494_b200 as omc

A = 1 << 20          # an address that looks aligned; nothing below may reach the point of using it
INVALID, NULL, MISALIGNED = -1, -3, -4


def refused(expected, fn, *args, **kw):
    with pytest.raises(omc.OmcError) as e:
        fn(*args, **kw)
    assert e.value.status == expected


def test_sizes():
    assert omc.mx_sizes(1, 1) == (16, 1024)
    assert omc.mx_sizes(128, 256) == (128 * 128, 1024)
    assert omc.mx_sizes(129, 257) == (129 * 144, 4 * 1024)
    for rows, cols in ((0, 5), (5, 0), (1 << 31, 1), (1, 1 << 31), ((1 << 31) - 1, (1 << 31) - 1)):
        refused(INVALID, omc.mx_sizes, rows, cols)
    assert omc.lib().omc_mx_sizes(4, 4, None, None) == 0
    assert omc.layer_norm_workspace_bytes(0, 8) >= 64
    assert omc.layer_norm_workspace_bytes(10 ** 6, 2048) % 16 == 0
    refused(INVALID, omc.layer_norm_workspace_bytes, 4, 0)
    assert omc.lib().omc_layer_norm_workspace(4, 4, None) == NULL


def test_quantise_refusals():
    ok = dict(type_=omc.F16, rows=4, cols=64, ld=64, codes=A, scales=A)
    refused(NULL, omc.mx_quantise, 0, **ok)
    for bad in (dict(type_=3), dict(type_=-1), dict(rows=0), dict(cols=0), dict(ld=63), dict(rows=1 << 31)):
        refused(INVALID, omc.mx_quantise, A, **{**ok, **bad})
    for bad in (dict(codes=0), dict(scales=0), dict(codes=0, scales=0), dict(codes_t=A), dict(scales_t=A)):
        refused(NULL, omc.mx_quantise, A, **{**ok, **bad})
    for bad in (dict(codes=A + 8), dict(scales=A + 4), dict(codes_t=A, scales_t=A + 1), dict(codes_t=A + 8, scales_t=A)):
        refused(MISALIGNED, omc.mx_quantise, A, **{**ok, **bad})
    refused(MISALIGNED, omc.mx_quantise, A + 1, **ok)
    refused(NULL, omc.mx_dequantise, A, 0, 4, 64, A, omc.F32, 64)
    refused(INVALID, omc.mx_dequantise, A, A, 4, 64, A, omc.F32, 60)
    refused(INVALID, omc.mx_dequantise, A, A, 4, 64, A, 9, 64)
    refused(MISALIGNED, omc.mx_dequantise, A, A, 4, 64, A + 2, omc.F32, 64)


def test_product_refusals():
    ok = dict(x_codes=A, x_scales=A, M=4, w_codes=A, w_scales=A, N=8, K=64, y=A, type_=omc.F32, ldy=8, status=A)
    for name in ("x_codes", "x_scales", "w_codes", "w_scales", "y", "status"):
        refused(NULL, omc.mx_matmul, **{**ok, name: 0})
        refused(MISALIGNED, omc.mx_matmul, **{**ok, name: A + 2})
    for bad in (dict(M=0), dict(N=0), dict(K=0), dict(ldy=7), dict(type_=7), dict(M=128 * 65535 + 1)):
        refused(INVALID, omc.mx_matmul, **{**ok, **bad})
    ok = dict(x=A, type_=omc.BF16, M=4, K=64, ldx=64, w_codes=A, w_scales=A, N=8, y=A, y_type=omc.F32, ldy=8, workspace=A, status=A)
    for name in ("x", "w_codes", "w_scales", "y", "workspace", "status"):
        refused(NULL, omc.mx_linear, **{**ok, name: 0})
        refused(MISALIGNED, omc.mx_linear, **{**ok, name: A + 1})
    for bad in (dict(M=0), dict(N=0), dict(K=0), dict(ldx=63), dict(ldy=7), dict(type_=7), dict(y_type=-2)):
        refused(INVALID, omc.mx_linear, **{**ok, **bad})


def test_norm_refusals():
    ok = dict(x=A, type_=omc.F16, rows=4, cols=64, ld=64, gamma=A, beta=A, eps=1e-5, y=A, ldy=64, mean=A, rstd=A)
    for name in ("x", "gamma", "beta", "y"):
        refused(NULL, omc.layer_norm, **{**ok, name: 0})
        refused(MISALIGNED, omc.layer_norm, **{**ok, name: A + 1})
    refused(MISALIGNED, omc.layer_norm, **{**ok, "gamma": A + 4})
    refused(MISALIGNED, omc.layer_norm, **{**ok, "mean": A + 2})
    for bad in (dict(cols=0), dict(ld=63), dict(ldy=63), dict(eps=-1.0), dict(eps=float("nan")), dict(type_=5), dict(rows=1 << 31)):
        refused(INVALID, omc.layer_norm, **{**ok, **bad})
    omc.layer_norm(**{**ok, "rows": 0, "x": 0, "y": 0})          # nothing to do
    ok = dict(dy=A, ld_dy=64, x=A, ld_x=64, type_=omc.F16, rows=4, cols=64, gamma=A, mean=A, rstd=A, dx=A, ld_dx=64, dgamma=A, dbeta=A,
              workspace=A)
    for name in ("dy", "x", "gamma", "mean", "rstd", "dx", "dgamma", "dbeta", "workspace"):
        refused(NULL, omc.layer_norm_backward, **{**ok, name: 0})
        refused(MISALIGNED, omc.layer_norm_backward, **{**ok, name: A + 1})
    for bad in (dict(cols=0), dict(ld_x=63), dict(ld_dy=63), dict(ld_dx=63), dict(type_=5)):
        refused(INVALID, omc.layer_norm_backward, **{**ok, **bad})
