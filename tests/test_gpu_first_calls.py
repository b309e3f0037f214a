"""The first products of a process, made by several threads at once: what the library finds out on a first call (the driver's
tensor-map encoder, the device's SMs, shared memory above the default) it finds out without racing."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..")

PROGRAM = """
import sys, threading
sys.path.insert(0, %r)
import torch
import paper_2205_03494_b200 as omc
M, N, K, threads = 300, 200, 512, 8
torch.manual_seed(0)
x, w = torch.randn(M, K, device="cuda"), torch.randn(N, K, device="cuda")
room = lambda r, c: [torch.empty(n, dtype=torch.uint8, device="cuda") for n in omc.mx_sizes(r, c)]
wq = room(N, K)
ys = [torch.empty(M, N, device="cuda") for _ in range(threads)]
spaces = [torch.empty(sum(omc.mx_sizes(M, K)), dtype=torch.uint8, device="cuda") for _ in range(threads)]
status = torch.zeros(1, dtype=torch.int32, device="cuda")
streams = [torch.cuda.Stream() for _ in range(threads)]
omc.mx_quantise(w.data_ptr(), omc.F32, N, K, K, wq[0].data_ptr(), wq[1].data_ptr())
torch.cuda.synchronize()
start, failed = threading.Barrier(threads), []
def work(i):
    try:
        start.wait()
        omc.mx_linear(x.data_ptr(), omc.F32, M, K, K, wq[0].data_ptr(), wq[1].data_ptr(), N, ys[i].data_ptr(), omc.F32, N, spaces[i].data_ptr(),
                      status.data_ptr(), stream=streams[i].cuda_stream)
    except Exception as e:
        failed.append(e)
ts = [threading.Thread(target=work, args=(i,)) for i in range(threads)]
for t in ts: t.start()
for t in ts: t.join()
torch.cuda.synchronize()
assert not failed, failed
assert int(status[0]) == 0 and all(torch.equal(ys[0], y) for y in ys[1:]) and bool(ys[0].any())
"""


def test_first_products_from_several_threads():
    for _ in range(3):
        subprocess.run([sys.executable, "-c", PROGRAM % ROOT], check=True, timeout=300)
