"""The give-up path of the 4-bit products' bounded waits, run in the one form that cannot fault or hang: omc_mx_inject_wait_timeout
makes the first CTA of the next product announce its copies without issuing them, so that its waits run out, or give up the waits
for results while its products are on their way (tensor memory may be let go only after them).  It has to set the status word and end, the other CTAs' results have to be right, nothing may be written outside Y, and the next call gives the same
bits as one before it."""
import numpy as np
import pytest
import torch

import paper_2205_03494_b200 as omc
from harness import Guarded
from test_gpu_mx import stored_matrix, stream

pytestmark = pytest.mark.gpu

# (M, N, K, rows and columns of Y that the first CTA's tiles or its cluster's cover; None: several tiles)
SHAPES = {
    "few rows": (10, 300, 256, 16, 128),
    "few rows, more steps than stages": (20, 19000, 2560, 32, 128),
    "few rows, K divided": (3, 600, 4096, 16, 128),
    "few rows, K divided, more steps than stages": (64, 200, 16384, 64, 128),
    "sixteen rows, K divided, more steps than stages": (9, 200, 16384, 16, 128),
    "tile of 128 rows": (128, 512, 1000, 128, 128),
    "tile of 128 rows, more steps than stages": (300, 600, 2048, 128, 128),
    "tile of 128 rows, K divided": (100, 300, 5000, 128, 128),
    "several tiles of 128 rows": (2300, 2600, 200, None, None),
    "tile of 256 rows": (3000, 1000, 1000, 256, 128),
    "several tiles of 256 rows": (4000, 3000, 4100, None, None),
}


def problem(name, linear):
    M, N, K, tile_m, tile_n = SHAPES[name]
    rng = np.random.default_rng(M + N + K)
    xv = rng.standard_normal((M, K))
    x = torch.from_numpy(xv).to(torch.bfloat16).cuda()
    wc, ws, _ = stored_matrix(rng.standard_normal((N, K)) * 0.1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    space = torch.empty(sum(omc.mx_sizes(M, K)), dtype=torch.uint8, device="cuda")
    codes = omc.mx_sizes(M, K)[0]
    if not linear:
        omc.mx_quantise(x.data_ptr(), omc.BF16, M, K, K, space.data_ptr(), space.data_ptr() + codes, stream=stream())

    def run():
        y = Guarded(M * N, torch.float32, "cuda", fill=-7.0)
        if linear:
            omc.mx_linear(x.data_ptr(), omc.BF16, M, K, K, wc.data_ptr(), ws.data_ptr(), N, y.t.data_ptr(), omc.F32, N, space.data_ptr(),
                          status.data_ptr(), stream=stream())
        else:
            omc.mx_matmul(space.data_ptr(), space.data_ptr() + codes, M, wc.data_ptr(), ws.data_ptr(), N, K, y.t.data_ptr(), omc.F32, N,
                          status.data_ptr(), stream=stream())
        torch.cuda.synchronize()                       # the launch ends by itself
        assert y.intact()
        return y.t[:M * N].view(M, N).clone()
    return run, status, (tile_m, tile_n)


def check(name, linear, inject):
    run, status, (tile_m, tile_n) = problem(name, linear)
    want = run()
    assert int(status[0]) == 0
    inject()
    got = run()
    assert int(status[0]) != 0                         # says that it gave up
    same = got == want
    if tile_m is None:
        assert float(same.double().mean()) > 0.9
    else:
        assert bool(same[tile_m:].all()) and bool(same[:, tile_n:].all())
    if "divided" not in name:                          # (else the other CTAs add up what they have: anything)
        assert bool((got[:3, :128] == -7.0).all())     # nothing was written there
    status.zero_()
    assert torch.equal(run(), want) and int(status[0]) == 0


@pytest.mark.parametrize("linear", [False, True], ids=["matmul", "linear"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_copies_that_never_arrive(name, linear):
    check(name, linear, lambda: omc.mx_inject_wait_timeout(1 << 10, omc.MX_COPIES_MISSING))


@pytest.mark.parametrize("linear", [False, True], ids=["matmul", "linear"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_results_given_up_with_products_on_their_way(name, linear):
    check(name, linear, lambda: omc.mx_inject_wait_timeout(1 << 14, omc.MX_RESULTS_LATE))


def test_injection_argument_checks():
    for polls, what in ((0, 1), ((1 << 16) + 1, 1), (10, 0), (10, 3)):
        assert omc.lib().omc_mx_inject_wait_timeout(polls, what) == -1
