"""The 8-bit and gated operators together with the store: examples/gated_training_step.py runs, and what each of its steps gives is the definition
(i8_reference.py) applied to what the step before it gave."""
import os
import sys

import numpy as np
import pytest
import torch

import i8_reference as i8
import paper_2205_03494_b200 as omc
from test_gpu_gated import check_gated, codes_of
from test_gpu_i8 import same
from test_gpu_mx import host

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


def test_training_runs_and_a_frame_alone_is_the_frame_in_the_batch():
    import gated_training_step as ex
    losses, block, x = ex.train(rounds=5, frames=400, width_in=256, width=320, width_out=192)
    assert np.isfinite(losses).all() and len(set(losses)) == 5
    assert int(block.status[0]) == 0 and block.plan.status() == 0
    block.load()
    batch = block.forward(x)
    for i in (0, 7, 399):
        # integer sums: the same bits whichever kernel makes them; the gate is the same function of the same FP32 values
        assert torch.equal(block.frame(x[i:i + 1])[0], batch[i])


@pytest.mark.parametrize("frames,k,f,n", [(300, 200, 144, 96), (1000, 128, 272, 130)])
def test_gradients_reach_the_arena(frames, k, f, n):
    import gated_training_step as ex
    block = ex.Block(k, f, n, frames, seed=3)
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((frames, k))).to(torch.bfloat16).cuda()
    dy = torch.from_numpy(rng.standard_normal((frames, n))).to(torch.bfloat16).cuda()
    block.load()
    block.forward(x)
    y = block.y.clone()
    block.backward(dy)
    torch.cuda.synchronize()
    w, wo = host(block.view(block.full, 0)).reshape(2 * f, k), host(block.view(block.full, 1)).reshape(n, f)
    pre = i8.product(*i8.encode(host(x)), *i8.encode(w))
    same(block.pre, pre, torch.bfloat16)
    check_gated(host(block.hidden), pre[:, :f], pre[:, f:], "silu", "bf16")
    h, d = host(block.hidden), host(dy)
    same(y, i8.product(*i8.encode(h), *i8.encode(wo)), torch.bfloat16)
    same(block.dhidden, i8.product(*i8.encode(d), *i8.encode(wo.T)), torch.bfloat16)
    same(block.view(block.grads, 1).view(n, f), i8.product(*i8.encode(d.T), *i8.encode(h.T)), torch.float32)
    # the codes of the gate's gradients: those of omc_gated_backward's values
    dpre = torch.empty(frames, 2 * f, dtype=torch.bfloat16, device="cuda")
    omc.gated_backward(block.dhidden.data_ptr(), f, block.pre.data_ptr(), 2 * f, omc.BF16, frames, f, omc.GATE_SILU, dpre.data_ptr(), 2 * f, stream=block.stream)
    g = host(dpre)
    (gc, gs), (tc, ts) = i8.encode(g), i8.encode(g.T)
    assert np.array_equal(codes_of(block.dpre[0][0][:omc.byte_sizes(frames, 2 * f)[0]].cpu().numpy().view(np.int8), frames, 2 * f), gc)
    same(block.dx, i8.product(gc, gs, *i8.encode(w.T)), torch.bfloat16)
    same(block.view(block.grads, 0).view(2 * f, k), i8.product(tc, ts, *i8.encode(host(x).T)), torch.float32)
    assert int(block.status[0]) == 0
