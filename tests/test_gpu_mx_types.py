"""omc_mx_linear with results of another type than its input: bit for bit quantisation of the input's type followed by a product
with results of the other, for rows quantised inside the product (at most 16) and before it; the values themselves within the
bound of test_gpu_mx.py."""
import numpy as np
import pytest
import torch

import paper_2205_03494_b200 as omc
import mx_reference as mx
from harness import Guarded
from test_gpu_mx import TYPES, check_product, host, stored_matrix, stream, strided

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ty,y_ty", [(a, b) for a in TYPES for b in TYPES if a != b])
@pytest.mark.parametrize("M,N,K", [(1, 300, 512), (5, 777, 1000), (16, 130, 4096), (17, 300, 520), (60, 500, 333), (200, 300, 640), (3000, 700, 300)])
def test_linear_to_another_type(M, N, K, ty, y_ty):
    code, dtype = TYPES[ty]
    y_code, y_dtype = TYPES[y_ty]
    rng = np.random.default_rng(M + 2 * N + K)
    x = torch.from_numpy(rng.standard_normal((M, K)) * 3).to(dtype).double().numpy()
    wc, ws, wv = stored_matrix(rng.standard_normal((N, K)) * 0.1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    nc, ns = omc.mx_sizes(M, K)
    q = torch.empty(nc + ns, dtype=torch.uint8, device="cuda")
    for ld, ldy in ((K, N), (K + 1, N + 1)):
        buf, view = strided(x, dtype, ld)
        want, got = (Guarded(M * ldy, y_dtype, "cuda", fill=-7.0) for _ in range(2))
        omc.mx_quantise(view.data_ptr(), code, M, K, ld, q.data_ptr(), q.data_ptr() + nc, stream=stream())
        omc.mx_matmul(q.data_ptr(), q.data_ptr() + nc, M, wc.data_ptr(), ws.data_ptr(), N, K, want.t.data_ptr(), y_code, ldy, status.data_ptr(),
                      stream=stream())
        space = Guarded(nc + ns, torch.uint8, "cuda", fill=0xFF)
        omc.mx_linear(view.data_ptr(), code, M, K, ld, wc.data_ptr(), ws.data_ptr(), N, got.t.data_ptr(), y_code, ldy, space.t.data_ptr(),
                      status.data_ptr(), stream=stream())
        torch.cuda.synchronize()
        assert int(status[0]) == 0 and got.intact() and want.intact() and space.intact()
        assert torch.equal(got.t, want.t)
        y = got.t[:M * ldy].view(M, ldy)
        assert bool((y[:, N:] == -7.0).all())
        check_product(host(y[:, :N]), mx.quantised(x), wv, y_ty)
