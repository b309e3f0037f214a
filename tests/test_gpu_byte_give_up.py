"""The give-up path of the 8-bit products' bounded waits, run in the one form that cannot fault or hang: omc_byte_inject_wait_timeout makes the first CTA (or
pair of CTAs) of the next product announce its copies without issuing them, so that its waits run out, or give up the waits for results while its products are
on their way.  It has to set the status word and end, the other CTAs' results have to be right, nothing may be written outside Y, and the next call gives
the same bits as one before it."""
import numpy as np
import pytest
import torch

import paper_2205_03494_b200 as omc
from harness import Guarded
from test_gpu_i8 import stored
from test_gpu_mx import stream

pytestmark = pytest.mark.gpu

# (M, N, K, rows and columns of Y that the first CTA's tile, or its cluster's, lies within: no tile is larger than 256 x 256; None: several tiles)
SHAPES = {
    "few rows": (10, 20000, 300, 16, 128),
    "few rows, more steps than stages": (20, 19000, 2560, 32, 128),
    "few rows, K divided": (7, 600, 4096, 16, 128),
    "few rows, K divided, more steps than stages": (64, 200, 16384, 64, 128),
    "a tile an SM": (300, 600, 300, 256, 256),
    "a tile an SM or a pair, more steps than stages": (1100, 1100, 2048, 256, 256),
    "several tiles": (3000, 2000, 1000, None, None),
    "a tile a pair": (2048, 2048, 2048, 256, 256),
    "several tiles of the largest": (4000, 3000, 4100, None, None),
    "rows of Y that start anywhere": (1999, 2001, 2000, 256, 256),
}


def problem(name, gated):
    M, N, K, tile_m, tile_n = SHAPES[name]
    if gated and M * N > 74 * 256 * 128:               # a tile of the gated layer is 256 x 128: the first pair of SMs has several
        tile_m = None
    rng = np.random.default_rng(M + N + K)
    xc, xs, _, _ = stored(rng.standard_normal((M, K)).astype(np.float32))
    wc, ws, _, _ = stored((rng.standard_normal((2 * N if gated else N, K)) * 0.1).astype(np.float32))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run():
        y = Guarded(M * N, torch.float32, "cuda", fill=-7.0)
        if gated:
            omc.byte_gated(xc.data_ptr(), xs.data_ptr(), M, wc.data_ptr(), ws.data_ptr(), N, K, omc.GATE_SIGMOID, y.t.data_ptr(), omc.F32, N, 0, 0,
                           status.data_ptr(), stream=stream())
        else:
            omc.byte_matmul(xc.data_ptr(), xs.data_ptr(), M, wc.data_ptr(), ws.data_ptr(), N, K, y.t.data_ptr(), omc.F32, N, status.data_ptr(), stream=stream())
        torch.cuda.synchronize()                       # the launch ends by itself
        assert y.intact()
        return y.t[:M * N].view(M, N).clone()
    return run, status, (tile_m, tile_n)


def check(name, gated, what, polls):
    run, status, (tile_m, tile_n) = problem(name, gated)
    want = run()
    assert int(status[0]) == 0
    omc.byte_inject_wait_timeout(polls, what)
    got = run()
    assert int(status[0]) != 0                         # says that it gave up
    same = got == want
    if tile_m is None:
        assert float(same.double().mean()) > 0.9
    else:
        assert bool(same[tile_m:].all()) and bool(same[:, tile_n:].all())
    if "divided" not in name:                          # (else the other CTAs add up what they have: anything)
        assert bool((got[:3, :60] == -7.0).all())      # nothing was written there
    status.zero_()
    assert torch.equal(run(), want) and int(status[0]) == 0


@pytest.mark.parametrize("gated", [False, True], ids=["matmul", "gated"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_copies_that_never_arrive(name, gated):
    check(name, gated, omc.BYTE_COPIES_MISSING, 1 << 10)


@pytest.mark.parametrize("gated", [False, True], ids=["matmul", "gated"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_results_given_up_with_products_on_their_way(name, gated):
    check(name, gated, omc.BYTE_RESULTS_LATE, 1 << 14)
