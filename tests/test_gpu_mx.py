"""MX blocks on the GPU against the fp64 oracle: codes and scales have to be equal; the rest within bounds derived beside each."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import mx_oracle as mx  # noqa: E402
from paper_2511_04063_amd import binding as B  # noqa: E402

FORMATS = [B.DQ_MXFP4, B.DQ_MXFP8]
TYPES = {B.DQ_F32: torch.float32, B.DQ_BF16: torch.bfloat16}


def rng(seed):
    return np.random.Generator(np.random.Philox(seed))


def up(x, m):
    return -(-x // m) * m


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    c.ensure_workspace(1, 256, 512, B.DQ_F32)
    yield c
    torch.cuda.synchronize()
    c.close()


def view(rows, cols, ld, dtype, fill=float("nan")):
    """A rows x cols view of a filled buffer of rows x ld."""
    buf = torch.full((rows, ld), fill, dtype=dtype, device="cuda")
    return buf, buf[:, :cols]


def stored(rows, n, fmt, more=0):
    """Buffers for codes and scales, every byte 0xee."""
    cb, sb = B.dq_mx_row_bytes(fmt, n)
    return (torch.full((rows, cb + more), 0xEE, dtype=torch.uint8, device="cuda"), torch.full((rows, sb + more), 0xEE, dtype=torch.uint8, device="cuda"))


def block_values(T, n, seed, dtype):
    """Heavy-tailed rows of many magnitudes, with values on ties, on powers of two, zeros, and subnormal blocks; in the type's precision."""
    g = rng(seed)
    X = g.standard_t(3.0, size=(T, n)) * np.exp(2.0 * g.standard_normal((T, 1)))
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.5, -0.25, -2.5, 0.0, -0.0, 0.5, 8.0, 448.0, 464.0, 480.0, 2.0 ** -10, 1.0625])
    at = g.random((T, n)) < 0.3
    X = np.where(at, ties[g.integers(0, ties.size, (T, n))], X)
    X[T // 2] = 0.0
    X[T // 3] *= 2.0 ** -126
    X[T // 4] *= 1e-45
    X[T // 5] *= 2.0 ** 110
    return torch.from_numpy(X).to(torch.float32).to(dtype)


def check_stored(codes, scales, ref_codes, ref_scales, fmt, n):
    cb, sb = B.dq_mx_row_bytes(fmt, n)
    nb = mx.blocks(n)
    got_c, got_s = codes.cpu().numpy(), scales.cpu().numpy()
    assert np.array_equal(got_s[:, :nb], ref_scales)
    assert (got_s[:, nb:sb] == 0).all() and (got_s[:, sb:] == 0xEE).all() and (got_c[:, cb:] == 0xEE).all()
    assert np.array_equal(mx.unpack(got_c[:, :cb], fmt), ref_codes)


SHAPES = [(1, 1), (5, 3), (9, 5), (70, 7), (1, 32), (2, 31), (7, 33), (5, 100), (64, 128), (9, 515), (33, 1000), (3, 2890), (17, 4096), (6, 8200), (300, 40), (4100, 8)]


@pytest.mark.parametrize("T,n", SHAPES)
@pytest.mark.parametrize("xdt", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("fmt", FORMATS)
def test_quantize_and_back(ctx, fmt, xdt, T, n):
    X = block_values(T, n, 100 + T + n, TYPES[xdt])
    _, Xd = view(T, n, up(n, 8) + 8, TYPES[xdt])
    Xd.copy_(X)
    codes, scales = stored(T, n, fmt, more=16)
    ctx.dq_mx_quantize(Xd, xdt, fmt, codes, scales)
    ref_c, ref_s = mx.quantize(X.double().numpy(), fmt)
    check_stored(codes, scales, ref_c, ref_s, fmt, n)
    assert ctx.dq_device_flags() == 0
    ref = torch.from_numpy(mx.values(ref_c, ref_s, n, fmt))
    for ydt, dtype in TYPES.items():
        buf, Y = view(T, n, up(n, 8) + 8, dtype, 7.0)
        ctx.dq_mx_dequantize(fmt, codes, scales, Y, ydt)
        assert torch.equal(Y.cpu(), ref.float().to(dtype))                # one rounding, and that only below 2^-126
        assert (buf[:, n:] == 7.0).all()


@pytest.mark.parametrize("xdt", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("fmt", FORMATS)
def test_quantize_every_bf16_value(ctx, fmt, xdt):
    """Each finite bf16 value in a block with each of some largest values: every rounding, also of subnormals."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    v = bits[torch.isfinite(bits)].float()
    v = v[:-(v.numel() % 31)].reshape(-1, 31)
    rows = [torch.cat([torch.full((v.shape[0], 1), top), v], 1) for top in (0.0, 6.5, 1e30, 2.0 ** -120, 448.0)]
    X = torch.cat(rows).to(TYPES[xdt])
    codes, scales = stored(X.shape[0], 32, fmt)
    ctx.dq_mx_quantize(X.cuda(), xdt, fmt, codes, scales)
    ref_c, ref_s = mx.quantize(X.double().numpy(), fmt)
    check_stored(codes, scales, ref_c, ref_s, fmt, 32)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("xdt", [B.DQ_F32, B.DQ_BF16])
def test_blocks_that_are_not_finite(ctx, xdt, fmt):
    X = torch.randn((5, 200), generator=torch.Generator().manual_seed(1))
    X[1, 70], X[2, 199], X[3, 0] = float("nan"), float("inf"), -float("inf")
    X = X.to(TYPES[xdt])
    codes, scales = stored(5, 200, fmt)
    ctx.dq_mx_quantize(X.cuda(), xdt, fmt, codes, scales)
    ref_c, ref_s = mx.quantize(X.double().numpy(), fmt)
    check_stored(codes, scales, ref_c, ref_s, fmt, 200)
    assert ctx.dq_device_flags() == B.DQ_FLAG_NONFINITE and ctx.dq_device_flags() == 0
    Y = torch.zeros((5, 200), device="cuda")
    ctx.dq_mx_dequantize(fmt, codes, scales, Y, B.DQ_F32)
    ref = mx.values(ref_c, ref_s, 200, fmt)
    assert np.array_equal(np.isnan(Y.cpu().numpy()), np.isnan(ref)) and np.isnan(ref).sum() == 32 + 8 + 32


def test_read_every_code(ctx):
    """All 256 bytes under all 256 scales, in both formats."""
    for fmt in FORMATS:
        n = 512 if fmt == B.DQ_MXFP4 else 256
        cb, sb = B.dq_mx_row_bytes(fmt, n)
        codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1)
        scales = torch.full((256, sb), 0xFF, dtype=torch.uint8)
        scales[:, :n // 32] = torch.arange(256, dtype=torch.uint8)[:, None]
        ref = torch.from_numpy(mx.values(mx.unpack(codes.numpy(), fmt), scales[:, :n // 32].numpy(), n, fmt))
        for ydt, dtype in TYPES.items():
            Y = torch.zeros((256, n), device="cuda", dtype=dtype)
            ctx.dq_mx_dequantize(fmt, codes.cuda(), scales.cuda(), Y, ydt)
            assert torch.equal(torch.nan_to_num(Y.cpu(), nan=12345.0), torch.nan_to_num(ref.float().to(dtype), nan=12345.0))


@pytest.mark.parametrize("xdt", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("fmt", FORMATS)
def test_large_inputs_give_the_codes_of_their_parts(ctx, fmt, xdt):
    """More than the caches hold takes kernels of its own; the rows in parts take those that the oracle has checked."""
    T, n = 4500, 4001 if xdt == B.DQ_BF16 else 3001
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    X, res, H, H2 = (torch.empty((T, up(n, 8)), dtype=TYPES[xdt], device="cuda")[:, :n] for _ in range(4))
    X.copy_(torch.randn((T, n), device="cuda", generator=g))
    res.copy_(torch.randn((T, n), device="cuda", generator=g))
    assert T * n * X.element_size() > 32 << 20 > 1500 * n * X.element_size()
    gain = torch.rand(n, device="cuda", generator=g)
    for norm in (False, True):
        whole, parts = stored(T, n, fmt), stored(T, n, fmt)
        for out, h, bounds in ((whole, H, [(0, T)]), (parts, H2, [(0, 1500), (1500, 3000), (3000, T)])):
            for lo, hi in bounds:
                c, s = out[0][lo:hi], out[1][lo:hi]
                if norm:
                    ctx.dq_mx_rms_norm(X[lo:hi], xdt, res[lo:hi], h[lo:hi], gain, 1e-5, fmt, c, s)
                else:
                    ctx.dq_mx_quantize(X[lo:hi], xdt, fmt, c, s)
        assert torch.equal(whole[0], parts[0]) and torch.equal(whole[1], parts[1])
    assert torch.equal(H, H2)


# ----------------------------------------------------------------------------------- norm
NORM_SHAPES = [(1, 1), (5, 3), (9, 5), (3, 7), (3, 33), (130, 40), (5, 300), (4, 512), (9, 513), (6, 1000), (3, 1024), (5, 2048), (2, 2890), (1, 4096), (7, 4100), (9, 5004), (2, 5120), (5, 5800), (4, 6145), (3, 8192), (0, 64),
               (1030, 700), (1025, 1101), (1029, 1279), (1026, 2046), (1500, 129)]


def norm_reference(X, res, dtype, gain, eps, fmt):
    """h as it is stored, and codes and scales of fp32(norm of h).  The library's 64-bit mean differs from the oracle's by the order of a sum
    of n <= 8192 positive terms, n 2^-53 < 2^-39 relative; that turns a code only where y lies that close to the midpoint of two fp32
    numbers AND one of these is the border of two codes (a tie of 24-bit numbers, about one in 2^21): less than one code in 2^36."""
    h = X if res is None else (X.float() + res.float()).to(dtype)
    with np.errstate(over="ignore"):
        y = mx.rms_norm(h.double().numpy(), gain, eps).astype(np.float32)
    return h, mx.quantize(y, fmt)


@pytest.mark.parametrize("T,n", NORM_SHAPES)
@pytest.mark.parametrize("with_res,with_gain", [(True, False), (False, True), (True, True), (False, False)])
@pytest.mark.parametrize("xdt", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("fmt", FORMATS)
def test_rms_norm(ctx, fmt, xdt, with_res, with_gain, T, n):
    dtype = TYPES[xdt]
    g = rng(500 + T + n)
    X = torch.from_numpy(g.standard_t(3.0, size=(T, n))).to(dtype)
    res = torch.from_numpy(8.0 * g.standard_normal((T, n))).to(dtype) if with_res else None
    if T > 2:
        X[2] = 0
        if with_res:
            res[2] = 0
    gain = (1.0 + 0.3 * g.standard_normal(n)).astype(np.float32) if with_gain else None
    eps = 1e-5 if n % 2 else 0.0
    ld = up(n, 8) + 8
    _, Xd = view(T, n, ld, dtype)
    Xd.copy_(X)
    Rd = None
    if with_res:
        _, Rd = view(T, n, ld + 8, dtype)
        Rd.copy_(res)
    hbuf, H = view(T, n, ld, dtype, 7.0)
    codes, scales = stored(T, n, fmt, more=16)
    ctx.dq_mx_rms_norm(Xd, xdt, Rd, H, None if gain is None else torch.from_numpy(gain).cuda(), eps, fmt, codes, scales)
    h, (ref_c, ref_s) = norm_reference(X, res, dtype, gain, eps, fmt)
    assert torch.equal(H.cpu(), h) and (hbuf[:, n:] == 7.0).all()
    check_stored(codes, scales, ref_c, ref_s, fmt, n)
    assert ctx.dq_device_flags() == 0


@pytest.mark.parametrize("xdt", [B.DQ_F32, B.DQ_BF16])
def test_rms_norm_in_place_and_extremes(ctx, xdt):
    dtype, fmt, T, n = TYPES[xdt], B.DQ_MXFP8, 6, 1500
    g = rng(41)
    X = torch.from_numpy(g.standard_normal((T, n))).to(dtype)
    res = torch.from_numpy(g.standard_normal((T, n))).to(dtype)
    X[0], res[0] = X[0] * 1e30, res[0] * 1e30                  # squares beyond fp32
    X[1], res[1] = X[1] * 1e-30, res[1] * 1e-30                # squares below it
    want_h, (ref_c, ref_s) = norm_reference(X, res, dtype, None, 0.0, fmt)
    for target in ("residual", "x", "none"):
        _, Xd = view(T, n, up(n, 8), dtype)
        _, Rd = view(T, n, up(n, 8), dtype)
        Xd.copy_(X)
        Rd.copy_(res)
        codes, scales = stored(T, n, fmt)
        ctx.dq_mx_rms_norm(Xd, xdt, Rd, {"residual": Rd, "x": Xd, "none": None}[target], None, 0.0, fmt, codes, scales)
        check_stored(codes, scales, ref_c, ref_s, fmt, n)
        assert torch.equal(Rd.cpu(), want_h if target == "residual" else res)
        assert torch.equal(Xd.cpu(), want_h if target == "x" else X)
    assert ctx.dq_device_flags() == 0


def test_rms_norm_of_rows_that_are_not_finite(ctx):
    T, n, fmt = 4, 600, B.DQ_MXFP4
    X = torch.randn((T, n), generator=torch.Generator().manual_seed(2))
    X[1, 77], X[2, 300] = float("nan"), float("inf")
    codes, scales = stored(T, n, fmt)
    ctx.dq_mx_rms_norm(X.cuda(), B.DQ_F32, None, None, None, 1e-6, fmt, codes, scales)
    got = scales.cpu().numpy()[:, :19]
    assert (got[1] == 255).all()                               # the row's root is NaN
    assert got[2, 9] == 255 and (np.delete(got[2], 9) == 0).all()   # the root is infinite: zeros beside inf / inf
    _, (ref_c, ref_s) = norm_reference(X[[0, 3]], None, torch.float32, None, 1e-6, fmt)
    check_stored(codes[[0, 3]], scales[[0, 3]], ref_c, ref_s, fmt, n)
    assert ctx.dq_device_flags() == B.DQ_FLAG_NONFINITE


# ----------------------------------------------------------------------------------- objective
def test_objective_of_many_rows_and_of_many_problems(ctx):
    """More rows than the workgroups of a launch take at once, long and short ones, and so many problems that each gets few workgroups."""
    for b, T, n, some in ((1, 5000, 1201, [0]), (1, 300000, 33, [0]), (20000, 5, 600, [0, 1, 9999, 19999])):
        g = torch.Generator(device="cuda")
        g.manual_seed(n)
        Y = torch.empty((b, T, up(n, 4)), device="cuda")[:, :, :n]
        Y.copy_(torch.randn((b, T, n), device="cuda", generator=g))
        dY, loss = torch.empty((b, T, up(n, 4)), device="cuda")[:, :, :n], torch.empty(b, device="cuda")
        ctx.dq_objective_loss_grad(B.DQ_OBJ_MXFP8, 4, Y, B.DQ_REDUCE_TOKEN_MEAN, loss, dY, B.DQ_F32)
        for i in some:
            ref_loss, ref = mx.objective(Y[i].cpu().numpy(), B.DQ_MXFP8, "mean")
            assert (np.abs(dY[i].double().cpu().numpy() - ref) <= np.abs(ref) * 4 * 2.0 ** -24).all()
            assert abs(loss[i].item() - ref_loss) <= 8 * 2.0 ** -24 * ref_loss


@pytest.mark.parametrize("b,T,n", [(1, 1, 1), (2, 7, 3), (1, 9, 6), (1, 5, 33), (3, 45, 640), (1, 37, 101), (64, 9, 128), (2, 300, 80), (1, 19, 1500), (1, 9, 4096), (1, 5, 8192), (1, 7, 5001), (1, 9001, 530)])
@pytest.mark.parametrize("grad", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("fmt", FORMATS)
def test_objective(ctx, fmt, grad, b, T, n):
    mode = "mean" if (T + n) % 2 else "sum"
    red = B.DQ_REDUCE_TOKEN_MEAN if mode == "mean" else B.DQ_REDUCE_SUM
    obj = B.DQ_OBJ_MXFP4 if fmt == B.DQ_MXFP4 else B.DQ_OBJ_MXFP8
    g = rng(900 + T + n)
    Y = (g.standard_t(3.0, size=(b, T, n)) * 2.0).astype(np.float32)
    Y[0, 0, 0] = 0.0
    if T > 2:
        Y[0, 1] = 0.0
        Y[-1, 2] = 4.0
    ldy, ldd = up(n, 4) + 4, up(n, 8) + 8
    Yd = torch.full((b, T, ldy), float("nan"), device="cuda")
    Yd[:, :, :n] = torch.from_numpy(Y)
    dbuf = torch.full((b, T, ldd), 7.0, dtype=TYPES[grad], device="cuda")
    loss = torch.full((b,), float("nan"), device="cuda")
    only = torch.full((b,), float("nan"), device="cuda")
    ctx.dq_objective_loss_grad(obj, 4, Yd[:, :, :n], red, loss, dbuf[:, :, :n], grad)
    ctx.dq_objective_loss_grad(obj, 4, Yd[:, :, :n], red, only, None, grad)
    assert torch.equal(loss, only)
    assert (dbuf[:, :, n:] == 7.0).all()
    for i in range(b):
        ref_loss, ref = mx.objective(Y[i], fmt, mode)
        got = dbuf[i, :, :n].double().cpu().numpy()
        # y - yhat is exact in fp32 (the two are within a factor of two of each other, or one is zero); 2 c / n has three roundings, the
        # product one, bf16 another; the loss: a square, three sums of positive terms, two factors and a rounding in fp32, the rest in 64 bits
        assert (np.abs(got - ref) <= np.abs(ref) * (4 * 2.0 ** -24 + (2.0 ** -8 if grad == B.DQ_BF16 else 0.0))).all()
        assert abs(loss[i].item() - ref_loss) <= 8 * 2.0 ** -24 * ref_loss
    assert ctx.dq_device_flags() == 0


def test_objective_of_a_block_that_is_not_finite(ctx):
    Y = torch.ones((2, 64), device="cuda")
    Y[1, 40] = float("inf")
    loss, dY = torch.zeros(1, device="cuda"), torch.zeros((2, 64), device="cuda")
    ctx.dq_objective_loss_grad(B.DQ_OBJ_MXFP4, 4, Y, B.DQ_REDUCE_SUM, loss, dY, B.DQ_F32)
    assert torch.isnan(loss).all() and torch.isnan(dY[1, 32:]).all() and not torch.isnan(dY[0]).any() and not torch.isnan(dY[1, :32]).any()
    assert ctx.dq_device_flags() == B.DQ_FLAG_NONFINITE


# ----------------------------------------------------------------------------------- product
def random_matrix(rows, n, fmt, seed, spread=3):
    """Any codes but NaN, scales of 2^-spread .. 2^spread, in buffers whose unused bytes are poison."""
    g = rng(seed)
    cb, sb = B.dq_mx_row_bytes(fmt, n)
    nb = mx.blocks(n)
    codes = g.integers(0, 16 if fmt == B.DQ_MXFP4 else 256, (rows, nb * 32)).astype(np.uint8)
    if fmt == B.DQ_MXFP8:
        codes[(codes & 127) == 127] = 5
    codes[:, n:] = 0
    scales = g.integers(127 - spread, 128 + spread, (rows, nb)).astype(np.uint8)
    cd = torch.full((rows, cb + 32), 0xFF, dtype=torch.uint8, device="cuda")
    sd = torch.full((rows, sb + 16), 0xFF, dtype=torch.uint8, device="cuda")
    cd[:, :cb] = torch.from_numpy(mx.pack(codes, fmt))
    sd[:, :nb] = torch.from_numpy(scales)
    return mx.values(codes, scales, n, fmt), cd, sd


def product_bound(a, b, ref, K, fa, fb, cdt):
    """fp32 sums: at most four instructions for 128 of the reduction and sixteen more to join the parts, each off by 2^-23 of the sum of
    magnitudes.  8-bit operands with a bf16 result: each of eight products loses up to 2^-14 of the largest of them, 2^-11 of their
    magnitudes together.  Then the rounding of the result."""
    s = np.abs(a) @ np.abs(b).T
    eight = B.DQ_MXFP8 in (fa, fb)
    tol = s * (4 * -(-K // 128) + 16) * 2.0 ** -23
    if cdt == B.DQ_BF16:
        tol = tol + np.abs(ref) * 2.0 ** -8 + (s * 2.0 ** -11 if eight else 0.0)
    return tol + 1e-38


PRODUCTS = [(1, 1, 1), (1, 16, 32), (1, 130, 2890), (2, 7, 33), (15, 100, 129), (16, 64, 512), (17, 33, 513), (24, 260, 1000), (33, 16, 4100), (64, 128, 160),
            (65, 70, 96), (129, 257, 640), (130, 515, 100), (257, 129, 384), (300, 500, 1056), (256, 256, 1024), (512, 256, 512), (515, 385, 2080)]


@pytest.mark.parametrize("M,N,K", PRODUCTS)
@pytest.mark.parametrize("cdt", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("fa,fb", [(0, 0), (1, 0), (0, 1), (1, 1)])
def test_gemm_mx(ctx, fa, fb, cdt, M, N, K):
    a, A, As = random_matrix(M, K, fa, 31 * M + K)
    b, Bm, Bs = random_matrix(N, K, fb, 17 * N + K + 1)
    buf, C = view(M, N, up(N, 8) + 8, TYPES[cdt], 7.0)
    ctx.dq_gemm_mx(M, N, K, fa, A, As, fb, Bm, Bs, C, cdt)
    ref = a @ b.T
    got = C.double().cpu().numpy()
    assert (np.abs(got - ref) <= product_bound(a, b, ref, K, fa, fb, cdt)).all()
    assert (buf[:, N:] == 7.0).all()
    again = torch.empty_like(buf)[:, :N]
    ctx.dq_gemm_mx(M, N, K, fa, A, As, fb, Bm, Bs, again, cdt)
    assert torch.equal(C, again)


# Shapes that are multiples of no tile, for each kernel that the size of the result chooses (256, 128 with more and with fewer workgroups than compute
# units, 128 x 64, 64, 64 x 32, up to 16 rows with a long reduction), with reductions of one block, of odd counts of stages and of pieces of 512
@pytest.mark.parametrize("M,N", [(3601, 3570), (2049, 2190), (1701, 1750), (1000, 1601), (801, 1000), (400, 701), (200, 333), (100, 1503), (9, 700)])
@pytest.mark.parametrize("K", [20, 545, 1700, 5200])
@pytest.mark.parametrize("cdt", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("fa,fb", [(0, 0), (1, 0), (0, 1), (1, 1)])
def test_gemm_mx_every_kernel(ctx, fa, fb, cdt, M, N, K):
    _, A, As = random_matrix(M, K, fa, 41 * M + K)
    _, Bm, Bs = random_matrix(N, K, fb, 43 * N + K)
    vals = []
    for rows, fmt, c, s in ((M, fa, A, As), (N, fb, Bm, Bs)):          # read back by the library: that is tested above
        Y = torch.empty((rows, up(K, 8)), device="cuda")[:, :K]
        ctx.dq_mx_dequantize(fmt, c, s, Y, B.DQ_F32)
        vals.append(Y.double())
    buf, C = view(M, N, up(N, 8) + 8, TYPES[cdt], 7.0)
    ctx.dq_gemm_mx(M, N, K, fa, A, As, fb, Bm, Bs, C, cdt)
    ref = vals[0] @ vals[1].t().contiguous()
    s = vals[0].abs() @ vals[1].abs().t().contiguous()
    tol = s * (4 * -(-K // 128) + 16) * 2.0 ** -23 + 1e-38              # as product_bound
    if cdt == B.DQ_BF16:
        tol += ref.abs() * 2.0 ** -8 + (s * 2.0 ** -11 if B.DQ_MXFP8 in (fa, fb) else 0.0)
    assert bool(((C.double() - ref).abs() <= tol).all())
    assert (buf[:, N:] == 7.0).all()
    again = torch.empty_like(buf)[:, :N]
    ctx.dq_gemm_mx(M, N, K, fa, A, As, fb, Bm, Bs, again, cdt)
    assert torch.equal(C, again)


@pytest.mark.parametrize("fa,fb", [(0, 0), (1, 0), (1, 1)])
def test_gemm_of_rows_far_apart(ctx, fa, fb):
    """Rows of A, then of B, 8 MiB apart and more: beyond what the tiles address."""
    M, N, K, far = 70, 50, 700, (1 << 23) + 64
    a, A, As = random_matrix(M, K, fa, 91)
    b, Bm, Bs = random_matrix(N, K, fb, 92)
    ref = a @ b.T
    for spread in ("a", "b"):
        src = A if spread == "a" else Bm
        wide = torch.empty((src.shape[0], far), dtype=torch.uint8, device="cuda")[:, :src.shape[1]]
        wide.copy_(src)
        C = torch.empty((M, up(N, 8)), device="cuda")[:, :N]
        ctx.dq_gemm_mx(M, N, K, fa, wide if spread == "a" else A, As, fb, wide if spread == "b" else Bm, Bs, C, B.DQ_F32)
        assert (np.abs(C.double().cpu().numpy() - ref) <= product_bound(a, b, ref, K, fa, fb, B.DQ_F32)).all()


@pytest.mark.parametrize("cdt", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("fa,fb", [(0, 0), (1, 0), (0, 1), (1, 1)])
@pytest.mark.parametrize("M,N,K", [(5, 40, 600), (30, 41, 600), (100, 1503, 600), (300, 280, 600), (400, 701, 600), (1000, 1601, 600), (1701, 1750, 600), (3601, 3570, 600)])
def test_gemm_of_blocks_that_are_nan(ctx, M, N, K, fa, fb, cdt):
    a, A, As = random_matrix(M, K, fa, 71)
    b, Bm, Bs = random_matrix(N, K, fb, 72)
    As[3, 18] = 255                                            # the last block, cut short
    Bs[N - 2, 0] = 255
    C = torch.zeros((M, up(N, 8)), device="cuda", dtype=TYPES[cdt])[:, :N]
    ctx.dq_gemm_mx(M, N, K, fa, A, As, fb, Bm, Bs, C, cdt)
    bad = torch.isnan(C).cpu().numpy()
    want = np.zeros((M, N), dtype=bool)
    want[3], want[:, N - 2] = True, True
    assert np.array_equal(bad, want)
    ref = a @ b.T
    got = np.where(bad, ref, C.double().cpu().numpy())
    assert (np.abs(got - ref) <= product_bound(a, b, ref, K, fa, fb, cdt)).all()


@pytest.mark.parametrize("fa,fb", [(0, 0), (1, 0), (1, 1)])
def test_gemm_of_normal_values_is_as_near_as_documented(ctx, fa, fb):
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    M, N, K = 300, 400, 2048
    parts, vals = [], []
    for rows, fmt in ((M, fa), (N, fb)):
        X = torch.randn((rows, K), device="cuda", generator=g)
        c, s = stored(rows, K, fmt)
        ctx.dq_mx_quantize(X, B.DQ_F32, fmt, c, s)
        Y = torch.empty_like(X)
        ctx.dq_mx_dequantize(fmt, c, s, Y, B.DQ_F32)
        parts.append((c, s))
        vals.append(Y.double())
    ref = (vals[0] @ vals[1].t().contiguous()).cpu().numpy()
    C = torch.empty((M, N), device="cuda")
    ctx.dq_gemm_mx(M, N, K, fa, *parts[0], fb, *parts[1], C, B.DQ_F32)
    # random signs: 16 steps of four sums, each 2^-24 of a partial sum, add up to a few 2^-24 of the result; 1e-6 is 16 of them
    assert np.linalg.norm(C.double().cpu().numpy() - ref) <= 1e-6 * np.linalg.norm(ref)
    H = torch.empty((M, N), device="cuda", dtype=torch.bfloat16)
    ctx.dq_gemm_mx(M, N, K, fa, *parts[0], fb, *parts[1], H, B.DQ_BF16)
    assert np.linalg.norm(H.double().cpu().numpy() - ref) <= (2.0 ** -8 + 1e-4) * np.linalg.norm(ref)


# ----------------------------------------------------------------------------------- together, and around them
def test_offsets_beyond_32_bits(ctx):
    """Rows so far apart that the last one starts beyond 2^32 bytes (codes) and 2^32 elements (values)."""
    T, n, far = 70000, 96, 65536
    buf = torch.empty((T, far), dtype=torch.bfloat16, device="cuda")
    X = buf[:, :n]
    X.copy_(torch.randn((T, n), device="cuda"))
    cbuf = torch.empty((T, far), dtype=torch.uint8, device="cuda")
    near = stored(T, n, B.DQ_MXFP4)
    ctx.dq_mx_quantize(X, B.DQ_BF16, B.DQ_MXFP4, cbuf[:, :48], near[1])
    ctx.dq_mx_quantize(X.contiguous(), B.DQ_BF16, B.DQ_MXFP4, near[0], near[1])
    assert torch.equal(cbuf[:, :48], near[0])
    H = torch.empty((T, n), dtype=torch.bfloat16, device="cuda")
    ctx.dq_mx_dequantize(B.DQ_MXFP4, near[0], near[1], H, B.DQ_BF16)
    ctx.dq_mx_dequantize(B.DQ_MXFP4, cbuf[:, :48], near[1], X, B.DQ_BF16)
    assert torch.equal(H, X)
    w = stored(40, n, B.DQ_MXFP4)
    ctx.dq_mx_quantize(torch.randn((40, n), device="cuda"), B.DQ_F32, B.DQ_MXFP4, *w)
    C = [torch.empty((T, 40), device="cuda") for _ in range(2)]
    ctx.dq_gemm_mx(T, 40, n, 0, cbuf[:, :48], near[1], 0, *w, C[0], B.DQ_F32)
    ctx.dq_gemm_mx(T, 40, n, 0, *near, 0, *w, C[1], B.DQ_F32)
    assert torch.equal(C[0], C[1])
    ctx.dq_gemm_mx(40, T, n, 0, *w, 0, cbuf[:, :48], near[1], torch.empty((40, T), device="cuda"), B.DQ_F32)
    out = stored(T, n, B.DQ_MXFP4)
    ctx.dq_mx_rms_norm(X, B.DQ_BF16, None, X, None, 1e-5, B.DQ_MXFP4, cbuf[:, :48], out[1])
    ctx.dq_mx_rms_norm(H, B.DQ_BF16, None, None, None, 1e-5, B.DQ_MXFP4, near[0], near[1])
    assert torch.equal(cbuf[:, :48], near[0]) and torch.equal(out[1], near[1])


def test_more_workgroups_than_one_launch_holds(ctx):
    """Calls whose threads would pass 2^32 go in several launches: the norm's 2^22 rows of one workgroup each, the 2^22 strips of a product of rows
    far apart.  Rows repeat every 1024, so every launch has to give what the first one gave."""
    T, n, fmt = (1 << 22) + 1029, 1032, B.DQ_MXFP4
    base = torch.randn((1024, n), device="cuda").bfloat16()
    X = base.repeat(T // 1024 + 1, 1)[:T]
    out, ref = stored(T, n, fmt), stored(1024, n, fmt)
    ctx.dq_mx_rms_norm(X, B.DQ_BF16, X, X, None, 1e-5, fmt, *out)
    H = torch.empty_like(base)
    ctx.dq_mx_rms_norm(base, B.DQ_BF16, base, H, None, 1e-5, fmt, *ref)
    for got, want in ((out[0], ref[0]), (out[1], ref[1]), (X, H)):
        whole = T // 1024 * 1024
        assert (got[:whole].view(-1, 1024, got.shape[1]) == want).all() and torch.equal(got[whole:], want[:T - whole])
    del X, out, got
    M, N, K = (1 << 25) + 1029, 17, 40
    a, A, As = random_matrix(1024, K, fmt, 93)
    b, Bm, Bs = random_matrix(N, K, fmt, 94)
    far = torch.empty((N, (1 << 23) + 64), dtype=torch.uint8, device="cuda")[:, :Bm.shape[1]]
    far.copy_(Bm)
    many = [t.repeat(M // 1024 + 1, 1)[:M] for t in (A, As)]
    C = torch.empty((M, 24), dtype=torch.bfloat16, device="cuda")[:, :N]
    ctx.dq_gemm_mx(M, N, K, fmt, *many, fmt, far, Bs, C, B.DQ_BF16)
    one = torch.empty((1024, 24), dtype=torch.bfloat16, device="cuda")[:, :N]
    ctx.dq_gemm_mx(1024, N, K, fmt, A, As, fmt, far, Bs, one, B.DQ_BF16)
    ref = a @ b.T
    assert (np.abs(one.double().cpu().numpy() - ref) <= product_bound(a, b, ref, K, fmt, fmt, B.DQ_BF16)).all()
    whole = M // 1024 * 1024
    assert (C[:whole].unflatten(0, (-1, 1024)) == one).all() and torch.equal(C[whole:], one[:M - whole])


def layer(c, X, res, H, weights, fmt, bufs, Y):
    """What a linear layer of a rotated model does with its input."""
    c.dq_mx_rms_norm(X, B.DQ_BF16, res, H, None, 1e-5, fmt, *bufs)
    c.dq_gemm_mx(X.shape[0], Y.shape[1], X.shape[1], fmt, *bufs, B.DQ_MXFP4, *weights, Y, B.DQ_BF16)


@pytest.mark.parametrize("T", [1, 70])
@pytest.mark.parametrize("fmt", FORMATS)
def test_calibrate_quantize_norm_multiply(ctx, fmt, T):
    """The operators one after another as they are used: a calibration step on the MX objective, weights rotated and quantised, then norm and
    product, against the same chain in 64 bits from the library's own rotation."""
    n, N, Tc = 192, 136, 320
    g = rng(61)
    acts = (g.standard_t(3.0, size=(Tc, n))).astype(np.float32)
    Z = torch.from_numpy(g.standard_normal((n, n)).astype(np.float32)).cuda()
    R, U, G = (torch.empty((n, n), device="cuda") for _ in range(3))
    Yc, dY = torch.empty((Tc, n), device="cuda"), torch.empty((Tc, n), device="cuda")
    loss, step_loss = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    Xc = torch.from_numpy(acts).cuda()
    obj = B.DQ_OBJ_MXFP4 if fmt == B.DQ_MXFP4 else B.DQ_OBJ_MXFP8
    try:
        ctx.dq_set_objective(obj)
        ctx.dq_qr_orth(Z, R, U)
        ctx.dq_rotate_loss_grad(Xc, B.DQ_F32, R, B.DQ_REDUCE_TOKEN_MEAN, loss, G, Yc, dY)
        Zs = Z.clone()
        ctx.dq_calib_step(Xc, B.DQ_F32, Zs, 1e-2, B.DQ_REDUCE_TOKEN_MEAN, step_loss)
    finally:
        ctx.dq_set_objective(B.DQ_OBJ_WHIP)
    Yh = Yc.cpu().numpy()
    ref_loss, ref_dY = mx.objective(Yh, fmt, "mean")
    assert abs(loss.item() - ref_loss) <= 1e-6 * ref_loss and step_loss.item() == loss.item()
    assert np.abs(dY.cpu().numpy() - ref_dY).max() <= 4 * 2.0 ** -24 * np.abs(ref_dY).max()
    Gr = acts.astype(np.float64).T @ ref_dY
    assert np.linalg.norm(G.cpu().numpy() - Gr) <= 1e-5 * np.linalg.norm(Gr)
    dZ = torch.empty((n, n), device="cuda")
    ctx.dq_qr_backward(R, U, G, dZ)
    assert torch.allclose(Zs, Z - 1e-2 * dZ, rtol=0, atol=1e-6 * float(Z.abs().max()))

    W = torch.from_numpy(g.standard_normal((N, n)).astype(np.float32)).cuda()
    WR = torch.empty((N, n), device="cuda")
    ctx.dq_gemm_f32(N, n, n, 1.0, W, 0, R, 0, 0.0, WR)
    weights = stored(N, n, B.DQ_MXFP4)
    ctx.dq_mx_quantize(WR, B.DQ_F32, B.DQ_MXFP4, *weights)
    X = torch.from_numpy(g.standard_normal((T, n))).to(torch.bfloat16).cuda()
    res = torch.from_numpy(4.0 * g.standard_normal((T, n))).to(torch.bfloat16).cuda()
    H, bufs = torch.empty_like(X), stored(T, n, fmt)
    Y = torch.empty((T, N), dtype=torch.bfloat16, device="cuda")
    layer(ctx, X, res, H, weights, fmt, bufs, Y)
    h, (rc, rs) = norm_reference(X.cpu(), res.cpu(), torch.bfloat16, None, 1e-5, fmt)
    a, b = mx.values(rc, rs, n, fmt), mx.through(WR.cpu().numpy(), B.DQ_MXFP4)
    ref = a @ b.T
    assert torch.equal(H.cpu(), h)
    assert (np.abs(Y.double().cpu().numpy() - ref) <= product_bound(a, b, ref, n, fmt, B.DQ_MXFP4, B.DQ_BF16)).all()
    assert ctx.dq_device_flags() == 0


def test_replayed_graph_and_another_stream():
    """Norm, product and objective captured on a stream of their own; replays between eager work, new inputs each time."""
    T, n, N, fmt = 40, 640, 264, B.DQ_MXFP8
    s = torch.cuda.Stream()
    eager = B.Context()
    eager.ensure_workspace(1, 64, 64, B.DQ_F32)
    with torch.cuda.stream(s):
        c = B.Context()
        c.ensure_workspace(1, 64, 64, B.DQ_F32)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    X, res = (torch.randn((T, n), device="cuda", generator=g).bfloat16() for _ in range(2))
    W = torch.randn((N, n), device="cuda", generator=g)
    weights = stored(N, n, B.DQ_MXFP4)
    eager.dq_mx_quantize(W, B.DQ_F32, B.DQ_MXFP4, *weights)
    H, bufs, Y = torch.empty_like(X), stored(T, n, fmt), torch.empty((T, N), dtype=torch.bfloat16, device="cuda")
    Yf, loss, dY = torch.empty((T, n), device="cuda"), torch.zeros(1, device="cuda"), torch.empty((T, n), device="cuda")

    def work(k, H, bufs, Y, Yf, loss, dY):
        layer(k, X, res, H, weights, fmt, bufs, Y)
        k.dq_mx_dequantize(fmt, *bufs, Yf, B.DQ_F32)
        k.dq_objective_loss_grad(B.DQ_OBJ_MXFP4, 4, Yf, B.DQ_REDUCE_SUM, loss, dY, B.DQ_F32)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        work(c, H, bufs, Y, Yf, loss, dY)
    for i in range(4):
        X.copy_(torch.randn((T, n), device="cuda", generator=g))
        res.copy_(torch.randn((T, n), device="cuda", generator=g) * (i + 1))
        graph.replay()
        H2, bufs2, Y2 = torch.empty_like(X), stored(T, n, fmt), torch.empty_like(Y)
        Yf2, loss2, dY2 = torch.empty_like(Yf), torch.zeros(1, device="cuda"), torch.empty_like(dY)
        work(eager, H2, bufs2, Y2, Yf2, loss2, dY2)
        torch.cuda.synchronize()
        for got, ref in ((H, H2), (bufs[0], bufs2[0]), (bufs[1], bufs2[1]), (Y, Y2), (Yf, Yf2), (loss, loss2), (dY, dY2)):
            assert torch.equal(got, ref)
    c.close()
    eager.close()
