"""Layer norm of matrices that begin off the 16-byte boundaries, a few values wide and wider: forward and backward against
the formulas in 64 bits, with the bounds of test_gpu_norm.py.  What lies before, between and behind the rows is NaN, so that a
value taken from there shows."""
import numpy as np
import pytest
import torch

import paper_2205_03494_b200 as omc
from harness import Guarded
from test_gpu_norm import EPS, TYPES, U, UNIT, depth, host, stream, vector

pytestmark = pytest.mark.gpu


def placed(values, dtype, ld, offset):
    """values `offset` elements behind a 16-byte boundary, NaN around them; (buffer, address, the rounded values)."""
    rows, cols = values.shape
    buf = torch.full((16 + rows * ld + 16,), float("nan"), dtype=dtype, device="cuda")
    view = buf[8 + offset:8 + offset + rows * ld].view(rows, ld)[:, :cols]      # (8 values: 16 or 32 bytes)
    view.copy_(torch.from_numpy(values))
    return buf, view.data_ptr(), host(view)


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(40, 1), (40, 2), (33, 3), (65, 5), (41, 7), (9, 33), (50, 100), (12, 300), (7, 1001), (5, 2050), (3, 8191)])
def test_offset_matrices(rows, cols, ty):
    code, dtype = TYPES[ty]
    rng = np.random.default_rng(rows + cols)
    gamma, g = vector(rng, cols, 1.0, 0.2)
    beta, b = vector(rng, cols, 0.0, 0.3)
    D = depth(cols)
    half = UNIT[ty] * 1.01
    tiny = 2.0 ** -25 if ty == "f16" else 0
    for offset in range(1, 4 if ty == "f32" else 8):
        ld = cols + offset % 2
        xb, xp, x = placed(rng.standard_normal((rows, cols)) + 0.5, dtype, ld, offset)
        y = Guarded(8 + rows * ld, dtype, "cuda", fill=-7.0)
        mg, rg = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        out = y.t[offset:offset + rows * ld].view(rows, ld)
        omc.layer_norm(xp, code, rows, cols, ld, gamma.data_ptr(), beta.data_ptr(), EPS, out.data_ptr(), ld, mg.data_ptr(), rg.data_ptr(),
                       stream=stream())
        torch.cuda.synchronize()
        assert y.intact() and bool((y.t[:offset] == -7.0).all()) and bool((out[:, cols:] == -7.0).all())
        mean = x.mean(1, keepdims=True)
        var = ((x - mean) ** 2).mean(1, keepdims=True)
        rstd = 1 / np.sqrt(var + EPS)
        em = D * U * np.abs(x).mean(1, keepdims=True) + U * np.abs(mean)
        rel = 1.01 * (0.5 * (em ** 2 + (D + 3) * U * (var + em ** 2) + U * (var + EPS)) / (var + EPS) + 3 * U)
        assert (np.abs(host(mg)[:, None] - mean) <= em).all() and (np.abs(host(rg)[:, None] - rstd) <= rel * rstd).all()
        want = (x - mean) * rstd * g + b
        bound = np.abs(g) * rstd * (em + np.abs(x - mean) * (rel + 3 * U)) + 2 * U * (np.abs(want) + np.abs(b)) + half * np.abs(want) + tiny
        assert (np.abs(host(out[:, :cols]) - want) <= bound).all()

        db, dp, dy = placed(rng.standard_normal((rows, cols)), dtype, ld, (offset + 2) % (4 if ty == "f32" else 8))
        dxg = Guarded(8 + rows * ld, dtype, "cuda", fill=-7.0)
        dx = dxg.t[offset:offset + rows * ld].view(rows, ld)
        dg, dbeta = Guarded(cols, torch.float32, "cuda", fill=-7.0), Guarded(cols, torch.float32, "cuda", fill=-7.0)
        ws = Guarded(omc.layer_norm_workspace_bytes(rows, cols), torch.uint8, "cuda", fill=0xFF)
        m, r = torch.from_numpy(mean[:, 0]).float().cuda(), torch.from_numpy(rstd[:, 0]).float().cuda()
        omc.layer_norm_backward(dp, ld, xp, ld, code, rows, cols, gamma.data_ptr(), m.data_ptr(), r.data_ptr(), dx.data_ptr(), ld,
                                dg.t.data_ptr(), dbeta.t.data_ptr(), ws.t.data_ptr(), stream=stream())
        torch.cuda.synchronize()
        assert dxg.intact() and dg.intact() and dbeta.intact() and ws.intact()
        assert bool((dxg.t[:offset] == -7.0).all()) and bool((dx[:, cols:] == -7.0).all())
        mh, rh = host(m)[:, None], host(r)[:, None]
        xhat, gr = (x - mh) * rh, dy * g
        m1, m2 = gr.mean(1, keepdims=True), (gr * xhat).mean(1, keepdims=True)
        want = rh * (gr - m1 - xhat * m2)
        e1 = (D + 2) * U * np.abs(gr).mean(1, keepdims=True)
        e2 = (D + 6) * U * np.abs(gr * xhat).mean(1, keepdims=True)
        bound = rh * (4 * U * (np.abs(gr) + np.abs(m1) + np.abs(xhat * m2)) + e1 + np.abs(xhat) * e2 + 3 * U * np.abs(xhat * m2)) * 1.01 \
            + half * np.abs(want) + tiny
        assert (np.abs(host(dx[:, :cols]) - want) <= bound).all()
        deep = (148 + rows / 16 + 96 + 4) * U
        assert (np.abs(host(dg.t[:cols]) - (dy * xhat).sum(0)) <= deep * np.abs(dy * xhat).sum(0) + 1e-30).all()
        assert (np.abs(host(dbeta.t[:cols]) - dy.sum(0)) <= deep * np.abs(dy).sum(0) + 1e-30).all()
