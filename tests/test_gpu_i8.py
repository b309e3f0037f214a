"""omc_byte_quantise / _dequantise / _matmul / _linear against the format's definition in 64 bits (i8_reference.py).  Codes, scales, decoded
values and products have to be equal: the sums are whole numbers, and the roundings after them are fixed."""
import numpy as np
import pytest
import torch

import i8_reference as i8
import paper_2205_03494_b200 as omc
from harness import Guarded
from test_gpu_mx import TYPES, awkward, host, strided, stream

pytestmark = pytest.mark.gpu


def room(rows, cols, fill=0x5A):
    return [Guarded(n, torch.uint8, "cuda", fill=fill) for n in omc.byte_sizes(rows, cols)]


def as_codes(buf, rows, cols):
    n = omc.byte_sizes(rows, cols)[0]
    return buf.t[:n].cpu().numpy().view(np.int8)


def as_scales(buf, rows):
    return buf.t[:4 * rows].cpu().numpy().view(np.float32)


def quantise(x_ptr, code, rows, cols, ld, along, across):
    """Guarded outputs of omc_byte_quantise as host arrays: (codes, scales) or None, (codes_t, scales_t) or None."""
    a, t = (room(rows, cols) if along else None), (room(cols, rows) if across else None)
    ptr = [b.t.data_ptr() for b in a or ()] or [0, 0]
    ptr_t = [b.t.data_ptr() for b in t or ()] or [0, 0]
    space = Guarded(omc.byte_quantise_workspace_bytes(rows, cols), torch.uint8, "cuda", fill=0xFF)
    omc.byte_quantise(x_ptr, code, rows, cols, ld, *ptr, *ptr_t, space.t.data_ptr() if across else 0, stream=stream())
    torch.cuda.synchronize()
    assert space.intact() and all(b.intact() for b in (a or []) + (t or []))
    for bufs, n in ((a, rows), (t, cols)):
        assert not bufs or bool((bufs[1].t[4 * n:omc.byte_sizes(n, 1)[1]] == 0x5A).all())
    return ((as_codes(a[0], rows, cols), as_scales(a[1], rows)) if a else None), ((as_codes(t[0], cols, rows), as_scales(t[1], cols)) if t else None)


def check_stored(got, x):
    codes, scales = i8.encode(x)
    assert np.array_equal(got[1], scales, equal_nan=True)
    assert np.array_equal(got[0], i8.pack(codes))


SHAPES = [(1, 1), (1, 512), (3, 15), (5, 33), (12, 256), (40, 257), (129, 128), (130, 300), (257, 1000), (31, 2048), (300, 129), (1, 2500), (70, 8200),
          (3, 17000), (700, 40)]


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantise(rows, cols, ty):
    """Every group of threads that shares a row, rows too wide for it, tiles cut off on both sides; zeros, subnormals, the largest value, Inf and NaN in
    rows and so in columns; rows on and off 16-byte boundaries."""
    code, dtype = TYPES[ty]
    x = awkward(np.random.default_rng(rows * 7 + cols), rows, cols, dtype)
    for ld, offset in ((cols, 0), (cols + 1, 0), ((cols + 7) // 8 * 8 + 8, 0), ((cols + 7) // 8 * 8, 1)):
        buf, view = strided(x, dtype, ld, offset)
        for along, across in ((True, False), (True, True), (False, True)):
            rows_got, cols_got = quantise(view.data_ptr(), code, rows, cols, ld, along, across)
            if along:
                check_stored(rows_got, x)
            if across:
                check_stored(cols_got, x.T)


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(4000, 1000), (1500, 4111), (20000, 130), (513, 16384), (9000, 36)])
def test_quantise_many_rows(rows, cols, ty):
    """More rows than the first kernel has CTAs, several tiles of a strip in a CTA; every value finite, so that every column has codes."""
    code, dtype = TYPES[ty]
    rng = np.random.default_rng(rows + cols)
    x = torch.from_numpy(rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-6, 6, (rows, 1))).to(dtype).double().numpy()
    buf, view = strided(x, dtype, cols)
    rows_got, cols_got = quantise(view.data_ptr(), code, rows, cols, cols, True, True)
    check_stored(rows_got, x)
    check_stored(cols_got, x.T)


@pytest.mark.parametrize("ty", list(TYPES))
def test_quantise_ties_and_ends(ty):
    """x = s (q + 1/2) where that is a value of the type, its neighbours, and the ends +-127; scales from the smallest numbers to the largest."""
    code, dtype = TYPES[ty]
    half = np.arange(-127, 127) + 0.5
    info = torch.finfo(dtype)
    tops = [127.0 * 2.0 ** e for e in (-14, -3, 0, 5)] + [float(info.max), float(info.tiny), float(info.tiny) * 2.0 ** -6, 3.0]
    rows = []
    for top in tops:
        v = torch.tensor(np.concatenate([[top, -top], half * (top / 127)])).to(dtype)
        rows += [v, torch.nextafter(v, torch.full_like(v, 1e4 if dtype == torch.float16 else 1e30)) * 0.5, torch.nextafter(v, torch.zeros_like(v))]
    x = torch.stack(rows).double().numpy()
    x = np.where(np.isfinite(x), x, 0.0)
    buf, view = strided(x, dtype, x.shape[1])
    rows_got, cols_got = quantise(view.data_ptr(), code, *x.shape, x.shape[1], True, True)
    check_stored(rows_got, x)
    check_stored(cols_got, x.T)


def stored(x, fill=0):
    """Device codes and scales of x, and their host forms."""
    codes, scales = i8.encode(x)
    return torch.from_numpy(i8.pack(codes)).cuda(), torch.from_numpy(scales).cuda(), codes, scales


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 255), (5, 16), (7, 1000), (33, 2049), (2, 9000), (2000, 513), (300, 128)])
def test_dequantise(rows, cols, ty):
    """Every code; scales up to the largest that make the 16-bit types overflow, a NaN row; rows that begin on every kind of address."""
    code, dtype = TYPES[ty]
    rng = np.random.default_rng(rows + cols)
    codes = rng.integers(-128, 128, (rows, cols)).astype(np.int8)
    codes.flat[:min(256, codes.size)] = np.arange(-128, 128)[:min(256, codes.size)]
    scales = (2.0 ** rng.integers(-130, 120, rows) * rng.uniform(1, 2, rows)).astype(np.float32)
    if rows > 2:
        scales[1], codes[1] = np.nan, 0
    with np.errstate(over="ignore"):
        want = torch.from_numpy(i8.values(codes, scales)).to(dtype)
    cd, sd = torch.from_numpy(i8.pack(codes)).cuda(), torch.from_numpy(scales).cuda()
    for ld, offset in ((cols, 0), (cols, 1), (cols + 1, 3), ((cols + 7) // 8 * 8, 0), ((cols + 7) // 8 * 8, 1)):
        g = Guarded(offset + rows * ld, dtype, "cuda", fill=-7.0)
        out = g.t[offset:offset + rows * ld].view(rows, ld)
        omc.byte_dequantise(cd.data_ptr(), sd.data_ptr(), rows, cols, out.data_ptr(), code, ld, stream=stream())
        torch.cuda.synchronize()
        assert g.intact() and bool((out[:, cols:] == -7.0).all()) and bool((g.t[:offset] == -7.0).all())
        assert torch.equal(torch.nan_to_num(out[:, :cols].cpu(), nan=123.0), torch.nan_to_num(want, nan=123.0))


def same(got, want, dtype):
    """got (device matrix) holds the FP32 values `want` rounded to its type."""
    want = torch.from_numpy(np.ascontiguousarray(want)).to(dtype)
    got = got.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got, nan=0.0), torch.nan_to_num(want, nan=0.0))


PRODUCTS = [(1, 128, 256), (1, 1, 1), (2, 130, 64), (3, 777, 1000), (4, 40, 8160), (5, 130, 64), (16, 64, 2048), (17, 777, 1000), (33, 128, 31), (64, 300, 4096),
            (65, 257, 513), (128, 128, 128), (129, 511, 96), (300, 384, 800), (1000, 640, 512), (256, 256, 256), (515, 1030, 2050), (1, 2048, 8192),
            (2300, 2600, 768), (4000, 3000, 4100), (130, 300, 8192), (700, 9000, 600), (100, 129, 5000), (5, 128, 20000), (2304, 2056, 24)]


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_matmul(M, N, K, ty):
    """Every kernel: tiles and K steps cut off on every side, K divided among a cluster's CTAs, several tiles of a pair; rows of Y on 16-byte boundaries, off
    them and wider than the matrix; a row of X that is all zero."""
    code, dtype = TYPES[ty]
    rng = np.random.default_rng(M + 3 * N + K)
    x = rng.standard_normal((M, K)).astype(np.float32) * 2.0 ** rng.integers(-3, 4, (M, 1))
    w = (rng.standard_normal((N, K)) * 0.05).astype(np.float32)
    if M > 1:
        x[M // 2] = 0.0
    xc, xs, xq, xsc = stored(x)
    wc, ws, wq, wsc = stored(w)
    want = i8.product(xq, xsc, wq, wsc)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for ld in (N, N + 3, (N + 7) // 8 * 8):
        g = Guarded(M * ld, dtype, "cuda", fill=-7.0)
        y = g.t[:M * ld].view(M, ld)
        omc.byte_matmul(xc.data_ptr(), xs.data_ptr(), M, wc.data_ptr(), ws.data_ptr(), N, K, y.data_ptr(), code, ld, status.data_ptr(), stream=stream())
        torch.cuda.synchronize()
        assert int(status[0]) == 0 and g.intact()
        same(y[:, :N], want, dtype)
        assert bool((y[:, N:] == -7.0).all())


@pytest.mark.parametrize("M,N,K", [(3, 200, 600), (10, 200, 512), (300, 520, 700), (2500, 2500, 512)])
def test_matmul_scales_of_all_sizes_and_nan(M, N, K):
    """Scales over the whole range of FP32, on one side and the other, products that overflow and that do not although a step between would; NaN scales make
    their row or column NaN, and nothing else; codes of both ends."""
    rng = np.random.default_rng(M)
    xq, wq = rng.integers(-127, 128, (M, K)).astype(np.int8), rng.integers(-128, 128, (N, K)).astype(np.int8)
    xq[0], wq[0] = 127, -128
    xs = (2.0 ** rng.integers(-126, 121, M) * rng.uniform(1, 1.9, M)).astype(np.float32)
    ws = (2.0 ** rng.integers(-126, 121, N) * rng.uniform(1, 1.9, N)).astype(np.float32)
    xs[1], ws[-1] = np.float32(2.0 ** 120), np.float32(2.0 ** -120)
    xs[2], ws[5] = np.nan, np.nan
    t = [torch.from_numpy(a).cuda() for a in (i8.pack(xq), xs, i8.pack(wq), ws)]
    status, y = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty(M, N, device="cuda")
    omc.byte_matmul(t[0].data_ptr(), t[1].data_ptr(), M, t[2].data_ptr(), t[3].data_ptr(), N, K, y.data_ptr(), omc.F32, N, status.data_ptr(), stream=stream())
    same(y, i8.product(xq, xs, wq, ws), torch.float32)
    assert bool(torch.isfinite(y[1, -1])) and int(status[0]) == 0


@pytest.mark.parametrize("M", [1, 20, 300])
def test_matmul_longest_sums(M):
    """K = 2^17 - 1 with every product at its largest: the sums just fit."""
    K, N = (1 << 17) - 1, 130
    xq, wq = np.full((M, K), -128, np.int8), np.full((N, K), -128, np.int8)
    wq[1::2] = 127
    xs, ws = np.linspace(1, 2, M).astype(np.float32), np.linspace(1, 2, N).astype(np.float32)
    t = [torch.from_numpy(a).cuda() for a in (i8.pack(xq), xs, i8.pack(wq), ws)]
    status, y = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty(M, N, device="cuda")
    omc.byte_matmul(t[0].data_ptr(), t[1].data_ptr(), M, t[2].data_ptr(), t[3].data_ptr(), N, K, y.data_ptr(), omc.F32, N, status.data_ptr(), stream=stream())
    total = np.where(np.arange(N) % 2 == 1, -128 * 127 * K, 128 * 128 * K).astype(np.int64)
    want = np.broadcast_to(total.astype(np.float32), (M, N)) * xs[:, None] * ws[None, :]
    same(y, want.astype(np.float32), torch.float32)
    assert int(status[0]) == 0


@pytest.mark.parametrize("ty,y_ty", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("M,N,K", [(1, 2048, 512), (1, 777, 1000), (2, 300, 9000), (3, 130, 96), (4, 512, 8192), (4, 130, 30000), (7, 130, 96), (40, 300, 333),
                                   (700, 600, 520), (2304, 2304, 256)])
def test_linear_is_quantise_then_matmul(M, N, K, ty, y_ty):
    """Bit for bit, for rows on and off 16-byte boundaries, and NaN in one row."""
    (code, dtype), (y_code, y_dtype) = TYPES[ty], TYPES[y_ty]
    rng = np.random.default_rng(M + N + K)
    x = torch.from_numpy(rng.standard_normal((M, K)) * 3).to(dtype).double().numpy()
    if M > 2:
        x[M - 2, K // 2] = np.nan
    wc, ws, wq, wsc = stored((rng.standard_normal((N, K)) * 0.1).astype(np.float32))
    xq, xsc = i8.encode(x)
    want = i8.product(xq, xsc, wq, wsc)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for ld in (K, K + 1, (K + 7) // 8 * 8):
        buf, view = strided(x, dtype, ld)
        g, space = Guarded(M * N, y_dtype, "cuda", fill=-7.0), Guarded(sum(omc.byte_sizes(M, K)), torch.uint8, "cuda", fill=0xFF)
        omc.byte_linear(view.data_ptr(), code, M, K, ld, wc.data_ptr(), ws.data_ptr(), N, g.t.data_ptr(), y_code, N, space.t.data_ptr(), status.data_ptr(),
                      stream=stream())
        torch.cuda.synchronize()
        assert int(status[0]) == 0 and g.intact() and space.intact()
        same(g.t[:M * N].view(M, N), want, y_dtype)


def whole(rng, rows, cols):
    """Whole numbers whose largest magnitude is 127 along either axis: scale 1, and quantising them changes nothing."""
    x = rng.integers(-20, 21, (rows, cols)).astype(np.float64)
    for i in range(max(rows, cols)):
        x[i % rows, i % cols] = 127.0
    return x


def test_backward_products_against_differences():
    """L = sum dY * (X W^T) is linear in X and in W: its differences are its derivatives, exactly, for values that quantisation leaves alone; all sums
    are whole numbers below 2^24."""
    rng = np.random.default_rng(8)
    M, N, K = 96, 160, 224
    x, w, dy = whole(rng, M, K), whole(rng, N, K), whole(rng, M, N)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def both(a):
        t = torch.from_numpy(a).float().cuda()
        bufs = [torch.empty(n, dtype=torch.uint8, device="cuda") for s in (a.shape, a.shape[::-1]) for n in omc.byte_sizes(*s)]
        space = torch.empty(omc.byte_quantise_workspace_bytes(*a.shape), dtype=torch.uint8, device="cuda")
        omc.byte_quantise(t.data_ptr(), omc.F32, *a.shape, a.shape[1], *[b.data_ptr() for b in bufs], space.data_ptr(), stream=stream())
        torch.cuda.synchronize()
        return bufs

    def product(a, rows, b, cols, k):
        y = torch.empty(rows, cols, device="cuda")
        omc.byte_matmul(a[0].data_ptr(), a[1].data_ptr(), rows, b[0].data_ptr(), b[1].data_ptr(), cols, k, y.data_ptr(), omc.F32, cols, status.data_ptr(),
                      stream=stream())
        return host(y)

    qx, qw, qdy = both(x), both(w), both(dy)
    y, dx, dw = product(qx[:2], M, qw[:2], N, K), product(qdy[:2], M, qw[2:], K, N), product(qdy[2:], N, qx[2:], K, M)
    loss = lambda a, b: float((dy * (a @ b.T)).sum())
    assert np.array_equal(y, x @ w.T)
    for _ in range(20):
        m, n, k = rng.integers(M), rng.integers(N), rng.integers(K)
        e = np.zeros_like(x)
        e[m, k] = 0.5
        assert dx[m, k] == (loss(x + e, w) - loss(x - e, w))
        e = np.zeros_like(w)
        e[n, k] = 0.5
        assert dw[n, k] == (loss(x, w + e) - loss(x, w - e))
    assert int(status[0]) == 0


def test_codes_of_the_store_are_an_operand():
    """A variable held as S1I0F7 without the transformation: its packed codes, -128 among them, are W as they stand, with the scale 1 / 128."""
    N, K, M = 96, 160, 130
    rng = np.random.default_rng(3)
    w = rng.uniform(-1.0, 1.0, (N, K)).astype(np.float32)
    w[0, :4] = (-1.0, 1.0, -0.99, 0.0)
    plan = omc.Plan([N * K], [omc.KIND_WEIGHT_MATRIX], (0, 7), flags=omc.PLAN_WEIGHTS_ONLY, fixed=True)
    new = lambda n, t: torch.zeros(max(int(n), 16), dtype=t, device="cuda")
    packed, resid, sb, space = new(plan.packed_bytes, torch.uint8), new(plan.resid_elems, torch.float32), new(2, torch.float32), new(plan.workspace_bytes, torch.uint8)
    full = new(plan.full_elems, torch.float32)
    full[:N * K] = torch.from_numpy(w).cuda().reshape(-1)
    plan.prepare(space.data_ptr(), stream())
    plan.compress(full.data_ptr(), packed.data_ptr(), resid.data_ptr(), sb.data_ptr(), space.data_ptr(), stream())
    xc, xs, xq, xsc = stored(rng.standard_normal((M, K)).astype(np.float32))
    scales, status, y = torch.full((N,), 1.0 / 128, device="cuda"), new(1, torch.int32), torch.empty(M, N, device="cuda")
    omc.byte_matmul(xc.data_ptr(), xs.data_ptr(), M, packed.data_ptr() + plan.packed_off[0], scales.data_ptr(), N, K, y.data_ptr(), omc.F32, N, status.data_ptr(),
                  stream=stream())
    wq = np.clip(np.rint(w.astype(np.float64) * 128), -128, 127).astype(np.int8)
    same(y, i8.product(xq, xsc, wq, np.full(N, 1.0 / 128, np.float32)), torch.float32)


def test_same_bits_every_time_and_on_another_stream():
    rng = np.random.default_rng(1)
    for M, N, K in ((3, 600, 4096), (30, 600, 4096), (700, 900, 1000), (2304, 2304, 1024)):
        xc, xs, _, _ = stored(rng.standard_normal((M, K)).astype(np.float32))
        wc, ws, _, _ = stored(rng.standard_normal((N, K)).astype(np.float32))
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        ys = [torch.empty(M, N, device="cuda") for _ in range(4)]
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        for i, y in enumerate(ys):
            st = side.cuda_stream if i == 3 else stream()
            omc.byte_matmul(xc.data_ptr(), xs.data_ptr(), M, wc.data_ptr(), ws.data_ptr(), N, K, y.data_ptr(), omc.F32, N, status.data_ptr(), stream=st)
        torch.cuda.synchronize()
        assert all(torch.equal(ys[0], y) for y in ys[1:]) and int(status[0]) == 0
