"""omc_gated_backward's check that dpre shares no element with dy and pre.  Refusals need no GPU; what is accepted runs on one."""
import numpy as np
import pytest
import torch

import paper_2205_03494_b200 as omc
from test_layer_host import A, INVALID, refused

ROWS, F = 40, 24
PITCH = 5 * F + 3


def slices(dy, pre, dpre, pitch=PITCH, base=1 << 20, **more):
    """Arguments of a call on columns of one buffer of FP32 values: first columns of the three matrices."""
    return dict(dict(dy=base + 4 * dy, ld_dy=pitch, pre=base + 4 * pre, ld_pre=pitch, type_=omc.F32, rows=ROWS, F=F, activation=omc.GATE_SILU, dpre=base + 4 * dpre,
                     ld_dpre=pitch), **more)


@pytest.mark.parametrize("dy,pre,dpre", [(0, F, F), (0, F, 3 * F - 1), (0, F, 1), (2 * F - 1, 2 * F, 0), (4 * F, 2 * F + 1, 3), (0, F, PITCH - 2 * F + 1),
                                         (0, 2 * F, 7 * PITCH - 2 * F + 1), (0, F, -2 * F + 1), (3, F + 3, -5 * PITCH + 3 * F)])
def test_columns_that_share_elements_are_refused(dy, pre, dpre):
    refused(INVALID, omc.gated_backward, **slices(dy, pre, dpre))


def test_other_pitches_are_refused_by_their_ranges():
    ok = slices(0, F, 3 * F)
    for bad in (dict(ld_dy=PITCH + 1), dict(ld_pre=PITCH + 2), dict(ld_dpre=PITCH - 1)):
        refused(INVALID, omc.gated_backward, **{**ok, **bad})
    refused(INVALID, omc.gated_backward, **slices(0, F, 3 * F - 1, rows=1, ld_dpre=2 * F, ld_pre=3 * F))      # one row: the row itself


@pytest.mark.gpu
@pytest.mark.parametrize("ty", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("pitch,dy,pre,dpre", [(5 * F, 0, F, 3 * F), (5 * F, 4 * F, 2 * F, 0), (PITCH, 3, F + 3, 3 * F + 3), (PITCH, 2 * F, 0, 3 * F), (PITCH, 2 * F, 3 * F, 5 * F)])
def test_columns_of_one_buffer(pitch, dy, pre, dpre, ty):
    """dy, pre and dpre beside one another in the rows of one buffer (dpre also across the end of a row): the same values as in buffers of their own, and nothing else written."""
    from test_gpu_mx import TYPES, stream
    code, dtype = TYPES[ty]
    gen = torch.Generator(device="cuda").manual_seed(1)
    buf = torch.randn(ROWS + 2, pitch, generator=gen, device="cuda").to(dtype)
    at = lambda first, cols: buf.view(-1)[first:first + ROWS * pitch].view(ROWS, pitch)[:, :cols]
    d, p = at(dy, F).clone(), at(pre, 2 * F).clone()
    own = torch.empty(ROWS, 2 * F, dtype=dtype, device="cuda")
    omc.gated_backward(d.data_ptr(), F, p.data_ptr(), 2 * F, code, ROWS, F, omc.GATE_GELU, own.data_ptr(), 2 * F, stream=stream())
    want = buf.clone()
    want.view(-1)[dpre:dpre + ROWS * pitch].view(ROWS, pitch)[:, :2 * F] = own
    size = buf.element_size()
    omc.gated_backward(buf.data_ptr() + size * dy, pitch, buf.data_ptr() + size * pre, pitch, code, ROWS, F, omc.GATE_GELU, buf.data_ptr() + size * dpre, pitch,
                       stream=stream())
    torch.cuda.synchronize()
    assert torch.equal(buf, want)
