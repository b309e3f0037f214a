"""Results of the 8-bit products in rows that start anywhere: at every place within 16 bytes, with rows of every remainder, the bits are those of a result whose rows
start on 16-byte boundaries, and nothing between the rows or around them is written."""
import numpy as np
import pytest
import torch

import paper_2205_03494_b200 as omc
from harness import Guarded
from test_gpu_i8 import TYPES, stored
from test_gpu_mx import stream

pytestmark = pytest.mark.gpu

# few rows, a divided K, tiles on an SM, tiles on pairs of SMs, one of several tiles
SHAPES = [(3, 70, 100), (20, 333, 1100), (300, 601, 200), (260, 37, 130), (2100, 2309, 300)]


@pytest.mark.parametrize("gated", [False, True], ids=["matmul", "gated"])
@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_rows_that_start_anywhere(M, N, K, ty, gated):
    code, dtype = TYPES[ty][:2]
    rng = np.random.default_rng(M + N + K)
    xc, xs, _, _ = stored(rng.standard_normal((M, K)).astype(np.float32))
    wc, ws, _, _ = stored((rng.standard_normal((2 * N if gated else N, K)) * 0.1).astype(np.float32))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def product(y, ld, pre, ld_pre):
        if gated:
            omc.byte_gated(xc.data_ptr(), xs.data_ptr(), M, wc.data_ptr(), ws.data_ptr(), N, K, omc.GATE_SILU, y.data_ptr(), code, ld, pre.data_ptr(), ld_pre,
                           status.data_ptr(), stream=stream())
        else:
            omc.byte_matmul(xc.data_ptr(), xs.data_ptr(), M, wc.data_ptr(), ws.data_ptr(), N, K, y.data_ptr(), code, ld, status.data_ptr(), stream=stream())
        torch.cuda.synchronize()
        assert int(status[0]) == 0

    def placed(offset, rows, ld):
        g = Guarded(offset + rows * ld, dtype, "cuda", fill=-7.0)
        return g, g.t[offset:offset + rows * ld].view(rows, ld)

    even, even_pre = (N + 7) // 8 * 8, (2 * N + 7) // 8 * 8
    _, y0 = placed(0, M, even)
    _, p0 = placed(0, M, even_pre)
    product(y0, even, p0, even_pre)
    want, want_pre = y0[:, :N].clone(), p0[:, :2 * N].clone()
    assert bool((y0[:, N:] == -7.0).all())
    for offset in range(8):
        for ld in ([N + offset, N + 9 - offset] if M < 2000 else [N + offset]):
            gy, y = placed(offset, M, ld)
            gp, pre = placed((offset * 3) % 8, M, ld + N)
            product(y, ld, pre, ld + N)
            assert torch.equal(y[:, :N], want)
            assert gy.intact() and bool((y[:, N:] == -7.0).all()) and bool((gy.t[:offset] == -7.0).all())
            if gated:
                assert torch.equal(pre[:, :2 * N], want_pre)
                assert gp.intact() and bool((pre[:, 2 * N:] == -7.0).all()) and bool((gp.t[:(offset * 3) % 8] == -7.0).all())
