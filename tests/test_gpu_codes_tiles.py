"""Codes along the columns where a CTA of the second kernel has several tiles of rows: the two tiles in shared memory in turn, the rows' factors and marks of both, loads that run over into the
next tile, and the change between loops with and without checks.  Rows and columns with a NaN or an Inf lie in neighbouring tiles and in every other one."""
import numpy as np
import pytest
import torch

import i8_reference as i8
import paper_2205_03494_b200 as omc
from harness import Guarded
from test_gpu_gated import ACTS, check_gradients
from test_gpu_i8 import as_codes, as_scales, check_stored, quantise, room
from test_gpu_mx import TYPES, host, strided, stream

pytestmark = pytest.mark.gpu


def tiles_of_a_cta(rows, cols, ty, halves, whole):
    """Strips of sixteen pieces of sixteen bytes; as many CTAs as are resident at once share the tiles, of 128 rows or 64 of two halves."""
    strips, tiles = -(-cols // (16 * (4 if ty == "f32" else 8))), -(-rows // (128 if halves == 1 else 64))
    resident = 148 * (3 if halves == 2 else 5 if whole else 4)
    shares = min(tiles, max(1, resident // strips))
    return -(-tiles // shares)


def bad_places(rows, tile):
    """Rows in the last tile, the two before it, and further ones at every other tile."""
    last = (rows - 1) // tile
    return [t * tile + 7 * (t % 5) for t in (last, last - 1, last - 2, last - 4, last - 6, 1) if 0 <= t and t * tile + 7 * (t % 5) < rows]


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("rows,F,name", [(1000, 16384, "silu"), (1500, 8200, "gelu"), (1500, 8201, "sigmoid")])
def test_gradients(rows, F, name, ty):
    code, dtype = TYPES[ty]
    assert tiles_of_a_cta(rows, F, ty, 2, F % 8 == 0) > 2
    rng = np.random.default_rng(rows + F)
    dy = rng.standard_normal((rows, F)) * 2.0 ** rng.integers(-4, 3, (rows, 1))
    pre = rng.standard_normal((rows, 2 * F)) * 3
    bad = bad_places(rows, 64)
    d, p = (torch.from_numpy(v).to(dtype).cuda() for v in (dy, pre))
    out = torch.empty(rows, 2 * F, dtype=dtype, device="cuda")
    for marked in (False, True):
        if marked:                                    # a NaN in one column each, and one column with two
            for i, r in enumerate(bad):
                d[r, (i * 131) % 400] = float("nan") if i % 2 else float("inf")
        omc.gated_backward(d.data_ptr(), F, p.data_ptr(), 2 * F, code, rows, F, ACTS[name], out.data_ptr(), 2 * F, stream=stream())
        matrix = host(out)
        if not marked:
            check_gradients(matrix, host(d), host(p)[:, :F], host(p)[:, F:], name, ty)
        else:
            assert sorted(np.nonzero(~np.isfinite(matrix).all(1))[0]) == sorted(bad)
        for along in (True, False):
            q, qt = room(rows, 2 * F), room(2 * F, rows)
            space = Guarded(omc.gated_backward_workspace_bytes(rows, F), torch.uint8, "cuda", fill=0xFF)
            omc.gated_backward(d.data_ptr(), F, p.data_ptr(), 2 * F, code, rows, F, ACTS[name], 0, 0, *([b.t.data_ptr() for b in q] if along else [0, 0]),
                               *[b.t.data_ptr() for b in qt], space.t.data_ptr(), stream=stream())
            torch.cuda.synchronize()
            assert space.intact() and all(b.intact() for b in q + qt)
            if along:
                check_stored((as_codes(q[0], rows, 2 * F), as_scales(q[1], rows)), matrix)
            check_stored((as_codes(qt[0], 2 * F, rows), as_scales(qt[1], 2 * F)), matrix.T)


@pytest.mark.parametrize("ty,rows,cols", [("f16", 3000, 8191), ("bf16", 3000, 8191), ("f32", 3000, 4099), ("bf16", 3001, 16384), ("f32", 2500, 8192)])
def test_matrix(rows, cols, ty):
    code, dtype = TYPES[ty]
    whole = cols * dtype.itemsize % 16 == 0
    assert tiles_of_a_cta(rows, cols, ty, 1, whole) > 2
    rng = np.random.default_rng(rows + cols)
    x = torch.from_numpy(rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-6, 6, (rows, 1))).to(dtype).double().numpy()
    for marked in (False, True):
        if marked:
            for i, r in enumerate(bad_places(rows, 128)):
                x[r, (i * 131) % 400] = np.nan if i % 2 else np.inf
        buf, view = strided(x, dtype, cols)
        for along in (True, False):
            rows_got, cols_got = quantise(view.data_ptr(), code, rows, cols, cols, along, True)
            if along:
                check_stored(rows_got, x)
            check_stored(cols_got, x.T)
