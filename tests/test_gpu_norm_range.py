"""omc_layer_norm on rows whose arithmetic leaves the finite numbers: mean, rstd and result are what IEEE-754 gives for
the formulas.

A row that holds an Inf or a NaN: mean = sum / cols (Inf of one sign stays Inf, both signs or a NaN give NaN); the deviation
of an Inf from an infinite mean is NaN, so the variance, rstd and the whole result are NaN.
A finite FP32 row whose squared deviations pass FP32's largest value: the variance is Inf, rstd 0 and the result the bias.
One whose sum does: the mean is Inf, rstd 0, the result -Inf * 0 = NaN."""
import numpy as np
import pytest
import torch

import paper_2205_03494_b200 as omc

pytestmark = pytest.mark.gpu

TYPES = {"f32": (omc.F32, torch.float32), "f16": (omc.F16, torch.float16), "bf16": (omc.BF16, torch.bfloat16)}
# every width class of the kernels (several rows to a warp, a warp, several warps, 32 values a thread, rows that stay in memory),
# rows on and off the 16-byte boundaries
COLS = [2, 7, 50, 64, 100, 128, 200, 256, 300, 512, 1001, 2048, 5001, 8192, 9000]


def forward(x, code, gamma, beta, eps):
    rows, cols = x.shape
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    omc.layer_norm(x.data_ptr(), code, rows, cols, cols, gamma.data_ptr(), beta.data_ptr(), eps, y.data_ptr(), cols, mean.data_ptr(),
                   rstd.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
    return y.double().cpu().numpy(), mean.double().cpu().numpy(), rstd.double().cpu().numpy()


@pytest.mark.parametrize("eps", [1e-5, 0.0])
@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("cols", COLS)
def test_moments_of_rows_with_inf_and_nan(cols, ty, eps):
    code, dtype = TYPES[ty]
    rng = np.random.default_rng(cols)
    x = torch.from_numpy(rng.standard_normal((12, cols))).to(dtype).cuda()
    inf = float("inf")
    x[1, cols // 2] = float("nan")
    x[3, 0] = inf
    x[4, cols - 1] = -inf
    x[6, 0], x[6, cols - 1] = inf, -inf
    x[7] = inf
    x[9, cols - 1], x[9, 0] = float("nan"), inf
    gamma, beta = torch.rand(cols, device="cuda") + 0.5, torch.rand(cols, device="cuda")
    y, mean, rstd = forward(x, code, gamma, beta, eps)
    bad = [1, 3, 4, 6, 7, 9]
    good = [r for r in range(12) if r not in bad]
    assert np.array_equal(mean[bad], [np.nan, np.inf, -np.inf, np.nan, np.inf, np.nan], equal_nan=True)
    assert np.isnan(rstd[bad]).all() and np.isnan(y[bad]).all()
    assert np.isfinite(mean[good]).all() and np.isfinite(rstd[good]).all() and np.isfinite(y[good]).all()


@pytest.mark.parametrize("cols", COLS)
def test_finite_rows_whose_moments_overflow(cols):
    """Deviations of 1e28 to 1e33: the squares overflow, the sums do not.  The mean's bound is that of the other tests."""
    rng = np.random.default_rng(cols + 1)
    v = rng.standard_normal((8, cols))
    v[:, 0], v[:, 1] = 2.0, -1.0               # deviations above 1 whatever the draw
    scale = np.array([1.0, 1e28, 1e30, 1e33, 1e28, 1e28, 1e15, 1.0])
    shift = np.array([0.0, 0.0, 0.0, 0.0, 3e28, -1e30, 0.0, 0.0])
    x = torch.from_numpy(v * scale[:, None] + shift[:, None]).float().cuda()
    x[7] = 3e38                                # the sum of two overflows
    gamma, beta = torch.rand(cols, device="cuda") + 0.5, torch.rand(cols, device="cuda")
    y, mean, rstd = forward(x, omc.F32, gamma, beta, 1e-5)
    h = x.double().cpu().numpy()
    over = slice(1, 6)
    assert (rstd[over] == 0).all() and np.array_equal(y[over], np.broadcast_to(beta.double().cpu().numpy(), (5, cols)))
    bound = (96 + cols / 256) * 2.0 ** -24 * np.abs(h[:7]).mean(1) + 2.0 ** -24 * np.abs(h[:7].mean(1))
    assert (np.abs(mean[:7] - h[:7].mean(1)) <= bound).all()
    assert mean[7] == np.inf and rstd[7] == 0 and np.isnan(y[7]).all()
    for r in (0, 6):
        assert abs(rstd[r] * np.sqrt(h[r].var() + 1e-5) - 1) < 1e-4 and np.isfinite(y[r]).all()
