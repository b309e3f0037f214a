"""omc_mx_quantise / _dequantise / _matmul / _linear against the format's definition in 64 bits
(mx_reference.py).  Codes, scales and decoded values must be equal.  Products: the operands' products are exact
in FP32, so the only errors are the K - 1 additions, at most one unit in the last place each (2^-23 of the
running sum, itself at most sum |x||w|), and the final rounding to the output type: the bound is
K 2^-23 sum |x||w| + u |y| with u = 2^-24, 2^-11, 2^-8, plus FP16's smallest subnormal."""
import numpy as np
import pytest
import torch

import paper_2205_03494_b200 as omc
import mx_reference as mx
from harness import Guarded

pytestmark = pytest.mark.gpu

TYPES = {"f32": (omc.F32, torch.float32), "f16": (omc.F16, torch.float16), "bf16": (omc.BF16, torch.bfloat16)}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def stream():
    return torch.cuda.current_stream().cuda_stream


def host(t):
    return t.double().cpu().numpy()


def strided(values, dtype, ld, offset=0):
    """values in a device matrix with `ld` elements from row to row, `offset` elements into its buffer; the rest NaN."""
    rows, cols = values.shape
    buf = torch.full((offset + rows * ld,), float("nan"), dtype=dtype, device="cuda")
    view = buf[offset:].view(rows, ld)[:, :cols]
    view.copy_(torch.from_numpy(values))
    return buf, view


def awkward(rng, rows, cols, dtype):
    """Values over many binades with everything a block can hold: zeros of both signs, subnormals, the type's largest
    value, ties, Inf and NaN (one block each), rows that are zero."""
    x = rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-12, 12, (rows, (cols + 31) // 32)).repeat(32, 1)[:, :cols]
    big, tiny = float(torch.finfo(dtype).max), float(torch.finfo(dtype).tiny)
    x.flat[0] = -0.0
    if rows > 4:
        x[1] = 0.0
        x[2] = rng.standard_normal(cols) * tiny
        x[3] = tiny * 2.0 ** -8                       # subnormal (zero where the type has none that small)
        x[4, : min(cols, 32)] = (np.arange(32) * 0.25 * np.where(np.arange(32) % 3, 1, -1))[:cols]      # every tie
    if rows > 9:
        x[5, cols // 2] = big
        x[6, 0] = -big
        x[7, cols - 1] = np.inf
        x[8, cols // 3] = -np.inf
        x[9, cols // 2] = np.nan
    return torch.from_numpy(x).to(dtype).double().numpy()


def quantise(x_ptr, code, rows, cols, ld, along, across):
    """Guarded outputs of omc_mx_quantise as host arrays: [codes, scales, codes_t, scales_t]."""
    bufs = []
    for want, shape in ((along, (rows, cols)), (across, (cols, rows))):
        for n in omc.mx_sizes(*shape):
            bufs.append(Guarded(n, torch.uint8, "cuda", fill=0x5A) if want else None)
    ptr = [b.t.data_ptr() if b else 0 for b in bufs]
    omc.mx_quantise(x_ptr, code, rows, cols, ld, *ptr, stream=stream())
    torch.cuda.synchronize()
    assert all(b is None or b.intact() for b in bufs)
    sizes = list(omc.mx_sizes(rows, cols)) + list(omc.mx_sizes(cols, rows))
    return [b.t[:n].cpu().numpy() if b else None for b, n in zip(bufs, sizes)]


def check_stored(got, x):
    rows, cols = x.shape
    codes, scales = mx.encode(x)
    packed, _ = mx.pack(codes, scales, cols)
    assert np.array_equal(got[0], packed)
    every = mx.scale_offsets(rows, -(-cols // 256) * 256)        # the blocks behind the last one included: zeros
    want = np.zeros(every.shape, np.uint8)
    want[:, :scales.shape[1]] = scales
    assert np.array_equal(got[1][every], want)


SHAPES = [(1, 1), (1, 512), (3, 31), (5, 33), (12, 256), (40, 257), (129, 128), (130, 300), (257, 1000), (31, 2048), (300, 129)]


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantise(rows, cols, ty):
    code, dtype = TYPES[ty]
    x = awkward(np.random.default_rng(rows * 7 + cols), rows, cols, dtype)
    for ld, offset in ((cols, 0), (cols + 1, 0), ((cols + 7) // 8 * 8 + 8, 0), ((cols + 7) // 8 * 8, 1)):
        buf, view = strided(x, dtype, ld, offset)
        for along, across in ((True, False), (True, True), (False, True)):
            got = quantise(view.data_ptr(), code, rows, cols, ld, along, across)
            if along:
                check_stored(got[:2], x)
            if across:
                check_stored(got[2:], x.T)


@pytest.mark.parametrize("ty", list(TYPES))
def test_dequantise_every_code_and_scale(ty):
    """16 codes x 256 scales; FP32 holds every value (2^-128 to 6 x 2^127 overflows to Inf), the 16-bit types round."""
    code, dtype = TYPES[ty]
    rows, cols = 256, 70
    codes = (np.arange(96)[None, :] * 5 + np.arange(rows)[:, None]).astype(np.uint8) % 16
    codes[:, cols:] = 0
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 3, 1)
    packed, stored = mx.pack(codes, scales, cols, fill=0xFF)
    with np.errstate(over="ignore"):
        want = mx.decode(codes, scales, cols)
    want = torch.from_numpy(want).float().to(dtype)
    cd, sd = torch.from_numpy(packed).cuda(), torch.from_numpy(stored).cuda()
    for ld, offset in ((cols, 0), (72, 0), (80, 3)):
        g = Guarded(offset + rows * ld, dtype, "cuda", fill=-7.0)
        out = g.t[offset:offset + rows * ld].view(rows, ld)
        omc.mx_dequantise(cd.data_ptr(), sd.data_ptr(), rows, cols, out.data_ptr(), code, ld, stream=stream())
        torch.cuda.synchronize()
        assert g.intact()
        assert torch.equal(torch.nan_to_num(out[:, :cols].cpu(), nan=123.0), torch.nan_to_num(want, nan=123.0))
        assert bool((out[:, cols:] == -7.0).all()) and bool((g.t[:offset] == -7.0).all())


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 255), (5, 257), (7, 1000), (33, 2049), (2, 9000), (2000, 513)])
def test_dequantise_wide_rows(rows, cols, ty):
    """Many pieces to a row, rows that begin on every kind of address, last pieces of one value and of 255."""
    code, dtype = TYPES[ty]
    rng = np.random.default_rng(rows + cols)
    cd, sd, want = stored_matrix(rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-6, 6, (rows, 1)))
    for ld, offset in ((cols, 0), (cols, 1), (cols + 1, 3), ((cols + 7) // 8 * 8, 0), ((cols + 7) // 8 * 8, 1)):
        g = Guarded(offset + rows * ld, dtype, "cuda", fill=-7.0)
        out = g.t[offset:offset + rows * ld].view(rows, ld)
        omc.mx_dequantise(cd.data_ptr(), sd.data_ptr(), rows, cols, out.data_ptr(), code, ld, stream=stream())
        torch.cuda.synchronize()
        assert g.intact() and bool((out[:, cols:] == -7.0).all()) and bool((g.t[:offset] == -7.0).all())
        assert torch.equal(out[:, :cols].cpu(), torch.from_numpy(want).float().to(dtype))


def stored_matrix(x, fill=0):
    codes, scales = mx.encode(x)
    packed, s = mx.pack(codes, scales, x.shape[1], fill)
    return torch.from_numpy(packed).cuda(), torch.from_numpy(s).cuda(), mx.decode(codes, scales, x.shape[1])


def check_product(got, x, w, ty):
    k = x.shape[1]
    want = x @ w.T
    bound = k * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T) + UNIT[ty] * np.abs(want) + (2.0 ** -25 if ty == "f16" else 0) + 1e-37
    err = np.abs(got - want)
    assert np.isfinite(got).all()
    assert (err <= bound).all(), float((err / bound).max())


PRODUCTS = [(1, 128, 256), (1, 1, 1), (2, 130, 64), (16, 64, 2048), (17, 777, 1000), (33, 128, 31), (64, 300, 4096), (65, 257, 513),
            (128, 128, 128), (129, 511, 96), (300, 384, 800), (1000, 640, 512), (256, 256, 256), (515, 1030, 2050), (1, 2048, 8192),
            (2300, 2600, 768), (4, 40, 8160), (4000, 3000, 4100), (130, 300, 8192), (700, 9000, 600), (100, 129, 5000)]


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_matmul(M, N, K, ty):
    """Tiles cut off on every side, K steps cut off, K divided among a cluster's CTAs (few tiles, many steps), several
    tiles per CTA; the scale bytes that the layout leaves open hold NaN; a row of X is all zero."""
    code, dtype = TYPES[ty]
    rng = np.random.default_rng(M + 3 * N + K)
    x = rng.standard_normal((M, K)) * 2.0 ** rng.integers(-3, 4, (M, 1))
    w = rng.standard_normal((N, K)) * 0.05
    x[M // 2] = 0.0 if M > 1 else x[0]
    xc, xs, xv = stored_matrix(x, 0xFF)
    wc, ws, wv = stored_matrix(w, 0xFF)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for ld in (N, N + 3):
        g = Guarded(M * ld, dtype, "cuda", fill=-7.0)
        y = g.t[:M * ld].view(M, ld)
        omc.mx_matmul(xc.data_ptr(), xs.data_ptr(), M, wc.data_ptr(), ws.data_ptr(), N, K, y.data_ptr(), code, ld, status.data_ptr(),
                      stream=stream())
        torch.cuda.synchronize()
        assert int(status[0]) == 0 and g.intact()
        check_product(host(y[:, :N]), xv, wv, ty)
        assert bool((y[:, N:] == -7.0).all())
        if M > 1:
            assert not y[M // 2, :N].any()


def test_matmul_scales_of_all_sizes():
    """Scales from 2^-60 to 2^60 on one side, their inverses on the other; differs from block to block."""
    rng = np.random.default_rng(5)
    M, N, K = 200, 300, 640
    e = rng.integers(-60, 61, (1, K // 32)).repeat(32, 1)
    xc, xs, xv = stored_matrix(rng.standard_normal((M, K)) * 2.0 ** e)
    wc, ws, wv = stored_matrix(rng.standard_normal((N, K)) * 2.0 ** -e)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    y = torch.empty(M, N, device="cuda")
    omc.mx_matmul(xc.data_ptr(), xs.data_ptr(), M, wc.data_ptr(), ws.data_ptr(), N, K, y.data_ptr(), omc.F32, N, status.data_ptr(),
                  stream=stream())
    check_product(host(y), xv, wv, "f32")
    assert int(status[0]) == 0


@pytest.mark.parametrize("M,N,K", [(10, 200, 512), (300, 520, 700), (2500, 2500, 512)])
def test_matmul_nan_blocks(M, N, K):
    """A NaN block of X makes its row NaN, one of W its column, and nothing else."""
    rng = np.random.default_rng(M)
    x, w = rng.standard_normal((M, K)), rng.standard_normal((N, K))
    rows, cols = [0, M // 2, M - 1], [3, N - 1]
    for r in rows:
        x[r, (r * 37) % K] = np.nan if r else np.inf
    for c in cols:
        w[c, K - 1] = np.nan
    xc, xs, xv = stored_matrix(x)
    wc, ws, wv = stored_matrix(w)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    y = torch.empty(M, N, device="cuda")
    omc.mx_matmul(xc.data_ptr(), xs.data_ptr(), M, wc.data_ptr(), ws.data_ptr(), N, K, y.data_ptr(), omc.F32, N, status.data_ptr(),
                  stream=stream())
    got = host(y)
    want = np.zeros((M, N), bool)
    want[rows] = True
    want[:, cols] = True
    assert np.array_equal(np.isnan(got), want)
    keep_r, keep_c = ~np.isin(np.arange(M), rows), ~np.isin(np.arange(N), cols)
    check_product(got[keep_r][:, keep_c], xv[keep_r], wv[keep_c], "f32")


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("M,N,K", [(1, 2048, 512), (1, 777, 1000), (7, 130, 96), (16, 512, 8192), (40, 300, 333), (700, 600, 520), (2304, 2304, 256)])
def test_linear_is_quantise_then_matmul(M, N, K, ty):
    """Bit for bit, for rows on and off 16-byte boundaries, and NaN in one row."""
    code, dtype = TYPES[ty]
    rng = np.random.default_rng(M + N + K)
    x = torch.from_numpy(rng.standard_normal((M, K)) * 3).to(dtype).double().numpy()
    if M > 4:
        x[M - 2, K // 2] = np.nan
    wc, ws, _ = stored_matrix(rng.standard_normal((N, K)) * 0.1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    nc, ns = omc.mx_sizes(M, K)
    q = torch.empty(nc + ns, dtype=torch.uint8, device="cuda")
    for ld in (K, K + 1, (K + 7) // 8 * 8):
        buf, view = strided(x, dtype, ld)
        want, g = torch.empty(M, N, dtype=dtype, device="cuda"), Guarded(M * N, dtype, "cuda", fill=-7.0)
        omc.mx_quantise(view.data_ptr(), code, M, K, ld, q.data_ptr(), q.data_ptr() + nc, stream=stream())
        omc.mx_matmul(q.data_ptr(), q.data_ptr() + nc, M, wc.data_ptr(), ws.data_ptr(), N, K, want.data_ptr(), code, N, status.data_ptr(),
                      stream=stream())
        w = Guarded(nc + ns, torch.uint8, "cuda", fill=0xFF)
        omc.mx_linear(view.data_ptr(), code, M, K, ld, wc.data_ptr(), ws.data_ptr(), N, g.t.data_ptr(), code, N, w.t.data_ptr(),
                      status.data_ptr(), stream=stream())
        torch.cuda.synchronize()
        assert int(status[0]) == 0 and g.intact() and w.intact()
        got = g.t[:M * N].view(M, N)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def grid(rng, rows, cols):
    """Values of the format whose blocks, along either axis, all have the scale 1: quantising them changes nothing."""
    x = rng.choice(mx.VALUES, (rows, cols))
    for r in range(rows):
        x[r, r % 32::32] = 4.0
    return x


def test_backward_products_against_differences():
    """L = sum dY * (X W^T) is linear in X and in W: its differences are its derivatives, exactly, for values that
    quantisation leaves alone; all sums are small multiples of 1/8 and exact in FP32."""
    rng = np.random.default_rng(8)
    M, N, K = 96, 160, 224
    x, w, dy = grid(rng, M, K), grid(rng, N, K), grid(rng, M, N)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def both(a):
        t = torch.from_numpy(a).float().cuda()
        bufs = [torch.empty(n, dtype=torch.uint8, device="cuda") for s in (a.shape, a.shape[::-1]) for n in omc.mx_sizes(*s)]
        omc.mx_quantise(t.data_ptr(), omc.F32, *a.shape, a.shape[1], *[b.data_ptr() for b in bufs], stream=stream())
        return bufs

    def product(a, rows, b, cols, k):
        y = torch.empty(rows, cols, device="cuda")
        omc.mx_matmul(a[0].data_ptr(), a[1].data_ptr(), rows, b[0].data_ptr(), b[1].data_ptr(), cols, k, y.data_ptr(), omc.F32, cols,
                      status.data_ptr(), stream=stream())
        return host(y)

    qx, qw, qdy = both(x), both(w), both(dy)
    y = product(qx[:2], M, qw[:2], N, K)
    dx = product(qdy[:2], M, qw[2:], K, N)
    dw = product(qdy[2:], N, qx[2:], K, M)
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


def test_same_bits_every_time_and_on_another_stream():
    rng = np.random.default_rng(1)
    for M, N, K in ((3, 600, 4096), (700, 900, 1000), (2304, 2304, 1024)):
        xc, xs, _ = stored_matrix(rng.standard_normal((M, K)))
        wc, ws, _ = stored_matrix(rng.standard_normal((N, K)))
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        ys = [torch.empty(M, N, device="cuda") for _ in range(4)]
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        for i, y in enumerate(ys):
            st = side.cuda_stream if i == 3 else stream()
            omc.mx_matmul(xc.data_ptr(), xs.data_ptr(), M, wc.data_ptr(), ws.data_ptr(), N, K, y.data_ptr(), omc.F32, N,
                          status.data_ptr(), stream=st)
        torch.cuda.synchronize()
        assert all(torch.equal(ys[0], y) for y in ys[1:]) and int(status[0]) == 0
