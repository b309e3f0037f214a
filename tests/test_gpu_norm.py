"""omc_layer_norm and its backward pass against the formulas in 64 bits.

Bounds, with u = 2^-24: a sum of n terms is formed by at most D = 96 + n / 256 additions one after the other on
the way of any term (registers, shuffles, warps), so it is off by at most D u sum |terms|.
  mean   D u mean|x| + u |mean|
  var    the squared deviations from a mean that is off by em sum to n (var + em^2) before rounding; their rounding (D + 3) u
  rstd   half of var's relative error, and 3 u for the root and the division
  y      |gamma| rstd (em + |x - mean| (rel(rstd) + 3 u)) + 2 u (|y| + |beta|), and the rounding to the type
  dx     rstd (4 u (|g| + |m1| + |xhat m2|) + e1 + |xhat| e2 + 3 u |xhat m2|), e1 = (D + 2) u mean|g|, e2 = (D + 6) u mean|g xhat|
  dgamma, dbeta   (148 + rows / 16 + 96) u sum |terms| and 4 u per term
with the type's half unit u_T |y| (FP16: plus half its smallest subnormal) for each rounded result."""
import numpy as np
import pytest
import torch

import paper_2205_03494_b200 as omc
from harness import Guarded

pytestmark = pytest.mark.gpu

TYPES = {"f32": (omc.F32, torch.float32), "f16": (omc.F16, torch.float16), "bf16": (omc.BF16, torch.bfloat16)}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
U = 2.0 ** -24
EPS = 1e-5
SHAPES = [(1, 512), (1, 1), (5, 7), (300, 32), (37, 96), (129, 512), (64, 1000), (33, 1023), (700, 1024), (20, 2048), (19, 2056),
          (9, 4096), (7, 5001), (6, 8192), (3, 8200), (2, 20000), (3000, 256), (2000, 40)]


def stream():
    return torch.cuda.current_stream().cuda_stream


def host(t):
    return t.double().cpu().numpy()


def make(rng, rows, cols, dtype, ld, shift=0.5):
    """A device matrix (NaN between its rows) and its values; some rows constant or zero."""
    x = rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-3, 3, (rows, 1)) + shift
    if rows > 2:
        x[rows // 2] = 0.0
        x[rows - 1] = 1.25
    buf = torch.full((rows, ld), float("nan"), dtype=dtype, device="cuda")
    buf[:, :cols] = torch.from_numpy(x)
    return buf, host(buf[:, :cols])


def vector(rng, cols, mean, std):
    v = torch.from_numpy(mean + std * rng.standard_normal(cols)).float().cuda()
    return v, host(v)


def depth(cols):
    return 96 + cols / 256


def leading(cols, ty):
    step = 4 if ty == "f32" else 8
    up = (cols + step - 1) // step * step
    return sorted({cols, up, up + step, cols + 1})


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward(rows, cols, ty):
    code, dtype = TYPES[ty]
    rng = np.random.default_rng(rows + 31 * cols)
    gamma, g = vector(rng, cols, 1.0, 0.2)
    beta, b = vector(rng, cols, 0.0, 0.3)
    for ld in leading(cols, ty):
        buf, x = make(rng, rows, cols, dtype, ld)
        yg = Guarded(rows * ld, dtype, "cuda", fill=-7.0)
        mg, rg = Guarded(rows, torch.float32, "cuda", fill=-7.0), Guarded(rows, torch.float32, "cuda", fill=-7.0)
        omc.layer_norm(buf.data_ptr(), code, rows, cols, ld, gamma.data_ptr(), beta.data_ptr(), EPS, yg.t.data_ptr(), ld,
                       mg.t.data_ptr(), rg.t.data_ptr(), stream=stream())
        torch.cuda.synchronize()
        assert yg.intact() and mg.intact() and rg.intact()
        out = yg.t[:rows * ld].view(rows, ld)
        assert bool((out[:, cols:] == -7.0).all())
        mean, D = x.mean(1), depth(cols)
        var = ((x - mean[:, None]) ** 2).mean(1)
        rstd = 1 / np.sqrt(var + EPS)
        em = D * U * np.abs(x).mean(1) + U * np.abs(mean)
        rel = 0.5 * (em ** 2 + (D + 3) * U * (var + em ** 2) + U * (var + EPS)) / (var + EPS) + 3 * U
        assert (np.abs(host(mg.t[:rows]) - mean) <= em).all()
        assert (np.abs(host(rg.t[:rows]) - rstd) <= rel * rstd * 1.01).all()
        xhat = (x - mean[:, None]) * rstd[:, None]
        want = xhat * g + b
        bound = np.abs(g) * rstd[:, None] * (em[:, None] + np.abs(x - mean[:, None]) * (rel[:, None] * 1.01 + 3 * U)) \
            + 2 * U * (np.abs(want) + np.abs(b)) + UNIT[ty] * np.abs(want) * 1.01 + (2.0 ** -25 if ty == "f16" else 0)
        err = np.abs(host(out[:, :cols]) - want)
        assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_backward(rows, cols, ty):
    code, dtype = TYPES[ty]
    rng = np.random.default_rng(rows + 17 * cols)
    gamma, g = vector(rng, cols, 1.0, 0.2)
    nbytes = omc.layer_norm_workspace_bytes(rows, cols)
    for ld in leading(cols, ty):
        xb, x = make(rng, rows, cols, dtype, ld)
        db, dy = make(rng, rows, cols, dtype, ld, shift=0.1)
        mean = torch.from_numpy(x.mean(1)).float().cuda()
        rstd = torch.from_numpy(1 / np.sqrt(x.var(1) + EPS)).float().cuda()
        m, r = host(mean)[:, None], host(rstd)[:, None]
        dg = Guarded(rows * ld, dtype, "cuda", fill=-7.0)
        gg, bg = Guarded(cols, torch.float32, "cuda", fill=-7.0), Guarded(cols, torch.float32, "cuda", fill=-7.0)
        ws = Guarded(nbytes, torch.uint8, "cuda", fill=0xFF)
        omc.layer_norm_backward(db.data_ptr(), ld, xb.data_ptr(), ld, code, rows, cols, gamma.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                dg.t.data_ptr(), ld, gg.t.data_ptr(), bg.t.data_ptr(), ws.t.data_ptr(), stream=stream())
        torch.cuda.synchronize()
        assert dg.intact() and gg.intact() and bg.intact() and ws.intact()
        out = dg.t[:rows * ld].view(rows, ld)
        assert bool((out[:, cols:] == -7.0).all())
        D = depth(cols)
        xhat, gr = (x - m) * r, dy * g
        m1, m2 = gr.mean(1, keepdims=True), (gr * xhat).mean(1, keepdims=True)
        want = r * (gr - m1 - xhat * m2)
        e1 = (D + 2) * U * np.abs(gr).mean(1, keepdims=True)
        e2 = (D + 6) * U * np.abs(gr * xhat).mean(1, keepdims=True)
        bound = r * (4 * U * (np.abs(gr) + np.abs(m1) + np.abs(xhat * m2)) + e1 + np.abs(xhat) * e2 + 3 * U * np.abs(xhat * m2)) * 1.01 \
            + UNIT[ty] * np.abs(want) * 1.01 + (2.0 ** -25 if ty == "f16" else 0)
        err = np.abs(host(out[:, :cols]) - want)
        assert (err <= bound).all(), float((err / bound).max())
        deep = (148 + rows / 16 + 96 + 4) * U
        assert (np.abs(host(gg.t[:cols]) - (dy * xhat).sum(0)) <= deep * np.abs(dy * xhat).sum(0) + 1e-30).all()
        assert (np.abs(host(bg.t[:cols]) - dy.sum(0)) <= deep * np.abs(dy).sum(0) + 1e-30).all()


MORE = [(1000, 64), (999, 100), (513, 128), (1201, 66), (3, 17), (77, 130), (41, 258), (200, 1002), (31, 2050), (5, 8190), (1, 33), (6, 65)]


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("rows,cols", MORE)
def test_narrow_rows_and_rows_on_four_bytes(rows, cols, ty):
    """Several rows to a warp, the last of them missing; rows that begin on multiples of 4 bytes but not of 16."""
    test_forward(rows, cols, ty)
    test_backward(rows, cols, ty)


def test_backward_against_differences():
    """Central differences of the forward formula in 64 bits (step 1e-4: error about 1e-8 of the third derivative)."""
    rng = np.random.default_rng(3)
    rows, cols, h = 5, 48, 1e-4
    xt = torch.from_numpy(rng.standard_normal((rows, cols))).float().cuda()
    wt = torch.from_numpy(rng.standard_normal((rows, cols))).float().cuda()
    gamma, g = vector(rng, cols, 1.0, 0.2)
    beta, b = vector(rng, cols, 0.0, 0.2)
    x, w = host(xt), host(wt)

    def loss(x, g, b):
        mu = x.mean(1, keepdims=True)
        return float((w * ((x - mu) / np.sqrt(((x - mu) ** 2).mean(1, keepdims=True) + EPS) * g + b)).sum())
    y, mean, rstd, dx = (torch.empty(s, device="cuda") for s in ((rows, cols), rows, rows, (rows, cols)))
    dgamma, dbeta = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(omc.layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    omc.layer_norm(xt.data_ptr(), omc.F32, rows, cols, cols, gamma.data_ptr(), beta.data_ptr(), EPS, y.data_ptr(), cols, mean.data_ptr(),
                   rstd.data_ptr(), stream=stream())
    omc.layer_norm_backward(wt.data_ptr(), cols, xt.data_ptr(), cols, omc.F32, rows, cols, gamma.data_ptr(), mean.data_ptr(),
                            rstd.data_ptr(), dx.data_ptr(), cols, dgamma.data_ptr(), dbeta.data_ptr(), ws.data_ptr(), stream=stream())
    got_x, got_g, got_b = host(dx), host(dgamma), host(dbeta)
    for _ in range(30):
        r, c = rng.integers(rows), rng.integers(cols)
        e = np.zeros((rows, cols))
        e[r, c] = h
        assert abs((loss(x + e, g, b) - loss(x - e, g, b)) / (2 * h) - got_x[r, c]) < 2e-6
        e = np.zeros(cols)
        e[c] = h
        assert abs((loss(x, g + e, b) - loss(x, g - e, b)) / (2 * h) - got_g[c]) < 1e-5
        assert abs((loss(x, g, b + e) - loss(x, g, b - e)) / (2 * h) - got_b[c]) < 1e-5


@pytest.mark.parametrize("cols", [33, 100, 300, 1000, 1023, 2048, 5000, 9000])
def test_rows_of_equal_values_give_the_bias(cols):
    """Padding frames: the deviations are zero, whatever the sum rounds to.  A first mean that is off by D u |x| leaves
    D u |x| u after its correction, times 1 / sqrt(eps) = 316 and a gain below 2: under 1e-9 for |x| < 2, so that y is the bias
    to half a unit of the last place."""
    x = torch.tensor([0.3, -1.7, 0.1, 1.2345], device="cuda")[:, None].expand(4, cols).contiguous()
    gamma, beta = torch.rand(cols, device="cuda") + 0.5, torch.rand(cols, device="cuda") + 0.5
    y, mean = torch.empty_like(x), torch.empty(4, device="cuda")
    omc.layer_norm(x.data_ptr(), omc.F32, 4, cols, cols, gamma.data_ptr(), beta.data_ptr(), EPS, y.data_ptr(), cols, mean.data_ptr(), 0,
                   stream=stream())
    assert np.abs(host(y) - host(beta)).max() < 2e-7
    assert (np.abs(host(mean) - host(x[:, 0])) <= 2.0 ** -23 * np.abs(host(x[:, 0]))).all()


@pytest.mark.parametrize("cols", [512, 1000, 2048, 9000])
def test_large_mean_does_not_cancel(cols):
    """Mean 1000, deviation 1: the variance is taken around the mean, not as a difference of large squares."""
    rng = np.random.default_rng(cols)
    x = torch.from_numpy(1000 + rng.standard_normal((40, cols))).float().cuda()
    gamma, beta = torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda")
    y, rstd = torch.empty_like(x), torch.empty(40, device="cuda")
    omc.layer_norm(x.data_ptr(), omc.F32, 40, cols, cols, gamma.data_ptr(), beta.data_ptr(), 0.0, y.data_ptr(), cols, 0, rstd.data_ptr(),
                   stream=stream())
    v = host(x)
    want = 1 / v.std(1)
    # the mean may be off by (depth + 1) 2^-24 x 1000, below 0.01: its square adds 1e-4 of the variance at most
    assert (np.abs(host(rstd) / want - 1) < 1e-4).all()
    assert (np.abs(host(y) - (v - v.mean(1, keepdims=True)) * want[:, None]) < 0.012).all()


@pytest.mark.parametrize("rows,cols", [(40, 512), (30, 2048), (9, 1001), (5, 9000), (7, 50), (6, 100)])
def test_non_finite_rows_stay_in_their_rows(rows, cols):
    """Inf and NaN make their own row NaN; in the backward pass also the column sums, which run over all rows."""
    rng = np.random.default_rng(2)
    x = torch.from_numpy(rng.standard_normal((rows, cols))).to(torch.bfloat16).cuda()
    x[1, 3], x[4, cols - 1] = float("inf"), float("nan")
    gamma, beta = torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    omc.layer_norm(x.data_ptr(), omc.BF16, rows, cols, cols, gamma.data_ptr(), beta.data_ptr(), EPS, y.data_ptr(), cols, mean.data_ptr(),
                   rstd.data_ptr(), stream=stream())
    dy, dx = torch.ones_like(x), torch.empty_like(x)
    dg, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(omc.layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    omc.layer_norm_backward(dy.data_ptr(), cols, x.data_ptr(), cols, omc.BF16, rows, cols, gamma.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                            dx.data_ptr(), cols, dg.data_ptr(), db.data_ptr(), ws.data_ptr(), stream=stream())
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[1] = bad[4] = True
    assert bool(torch.isnan(y[bad]).all()) and bool(torch.isfinite(y[~bad]).all())
    assert bool(torch.isnan(dx[bad]).all()) and bool(torch.isfinite(dx[~bad]).all())
    assert bool(torch.isnan(dg).all()) and bool((db == rows).all())


@pytest.mark.parametrize("rows,cols", [(1000, 512), (300, 1023), (500, 2048), (40, 9000)])
def test_in_place_no_moments_no_rows_same_bits(rows, cols):
    rng = np.random.default_rng(4)
    x = torch.from_numpy(rng.standard_normal((rows, cols))).half().cuda()
    dy = torch.from_numpy(rng.standard_normal((rows, cols))).half().cuda()
    gamma, beta = torch.rand(cols, device="cuda"), torch.rand(cols, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    args = (gamma.data_ptr(), beta.data_ptr(), EPS)
    omc.layer_norm(x.data_ptr(), omc.F16, rows, cols, cols, *args, y.data_ptr(), cols, mean.data_ptr(), rstd.data_ptr(), stream=stream())
    z = x.clone()
    omc.layer_norm(z.data_ptr(), omc.F16, rows, cols, cols, *args, z.data_ptr(), cols, stream=stream())
    assert torch.equal(y, z)
    ws = torch.empty(omc.layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    results = []
    for i in range(3):
        dyi, dg, db = dy.clone(), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        dx = dyi if i else torch.empty_like(dy)
        torch.cuda.synchronize()
        omc.layer_norm_backward(dyi.data_ptr(), cols, x.data_ptr(), cols, omc.F16, rows, cols, gamma.data_ptr(), mean.data_ptr(),
                                rstd.data_ptr(), dx.data_ptr(), cols, dg.data_ptr(), db.data_ptr(), ws.data_ptr(),
                                stream=side.cuda_stream if i == 2 else stream())
        torch.cuda.synchronize()
        results.append((dx, dg, db))
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))
    dg, db = results[0][1], results[0][2]
    omc.layer_norm_backward(0, cols, 0, cols, omc.F16, 0, cols, gamma.data_ptr(), 0, 0, 0, cols, dg.data_ptr(), db.data_ptr(), ws.data_ptr(),
                            stream=stream())
    assert not dg.any() and not db.any()
