"""MX operators at the ends of their ranges."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import mx_oracle as mx  # noqa: E402
from paper_2511_04063_amd import binding as B  # noqa: E402
from test_gpu_mx import TYPES, product_bound, random_matrix, rng, stored, up, view  # noqa: E402

PAIRS = [(0, 0), (1, 0), (0, 1), (1, 1)]


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    c.ensure_workspace(1, 256, 512, B.DQ_F32)
    yield c
    torch.cuda.synchronize()
    c.close()


# ----------------------------------------------------------------------------------- objective
@pytest.mark.parametrize("grad", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("obj,fmt", [(B.DQ_OBJ_MXFP4, mx.MXFP4), (B.DQ_OBJ_MXFP8, mx.MXFP8)])
@pytest.mark.parametrize("where", ["large", "small"])
def test_objective_whose_squares_leave_fp32(ctx, obj, fmt, grad, where):
    """Errors whose squares, or sums of four of them, lie beyond fp32's largest or below its smallest normal number, and a loss that does not.
    The bounds are those of ordinary rows: the sums are formed in 64 bits, so only the roundings of the loss and of the gradient count."""
    g = rng(77)
    if where == "large":
        T, n, mode = 6, 4096, "mean"
        Y = g.standard_normal((T, n)).astype(np.float32)
        # one block a row: with e4m3 errors reach 2^-4 of the values, with e2m1 a quarter
        Y[:, 64:96] *= np.float32(2.0 ** 68 if fmt == mx.MXFP8 else 2.0 ** 66)
        Y[0, 64:68] = np.float32(1.06 * 2.0 ** 71 if fmt == mx.MXFP8 else 1.24 * 2.0 ** 68)
    else:
        T, n, mode = 3000, 96, "sum"
        Y = (g.standard_normal((T, n)) * 2.0 ** (-63 if fmt == mx.MXFP8 else -64)).astype(np.float32)
    ref_loss, ref = mx.objective(Y, fmt, mode)
    e2 = (ref / (2.0 / n * (1.0 / T if mode == "mean" else 1.0))) ** 2
    largest = np.finfo(np.float32).max
    assert (e2.reshape(T, -1, 4).sum(-1).max() > largest if where == "large" else e2.max() < 2.0 ** -126) and 2.0 ** -126 < ref_loss < largest
    buf = torch.empty((T, up(n, 8)), dtype=TYPES[grad], device="cuda")[:, :n]
    loss = torch.zeros(1, device="cuda")
    red = B.DQ_REDUCE_TOKEN_MEAN if mode == "mean" else B.DQ_REDUCE_SUM
    ctx.dq_objective_loss_grad(obj, 4, torch.from_numpy(Y).cuda(), red, loss, buf, grad)
    assert abs(loss.item() - ref_loss) <= 8 * 2.0 ** -24 * ref_loss
    assert (np.abs(buf.double().cpu().numpy() - ref) <= np.abs(ref) * (4 * 2.0 ** -24 + (2.0 ** -8 if grad == B.DQ_BF16 else 0.0))).all()
    assert ctx.dq_device_flags() == 0


# ----------------------------------------------------------------------------------- product
def spread_matrices(M, N, K, fa, fb, seed, together, every):
    """Matrices whose scales run over the whole range, block by block of the reduction, while those of A and B together stay near `together`: all
    products are ordinary numbers.  `every`: only each so many blocks of the reduction leave the middle."""
    _, A, As = random_matrix(M, K, fa, seed)
    _, Bm, Bs = random_matrix(N, K, fb, seed + 1)
    nb, g = mx.blocks(K), rng(seed + 2)
    lo, hi = -127 + max(together, 0), 127 + min(together, 0)
    to_a = g.integers(lo, hi + 1, nb)
    to_a[:2] = lo, hi
    if every > 1:
        to_a[np.arange(nb) % every != every - 1] = together // 2
    out = []
    for rows, fmt, codes, scales, mid in ((M, fa, A, As, to_a), (N, fb, Bm, Bs, together - to_a)):
        byte = np.clip(mid[None, :] + 127 + g.integers(-2, 3, (rows, nb)), 0, 254).astype(np.uint8)
        cb = B.dq_mx_row_bytes(fmt, K)[0]
        if rows > 3:                                            # blocks of zeros, under scales of both ends
            codes[rows // 2, :cb] = 0
            byte[rows // 2, 0::2], byte[rows // 2, 1::2] = 0, 254
        scales[:, :nb] = torch.from_numpy(byte)
        out.append(mx.values(mx.unpack(codes[:, :cb].cpu().numpy(), fmt), byte, K, fmt))
    return out[0], A, As, out[1], Bm, Bs


# one for every kernel that the sizes choose (the last two: 256 x 256 tiles, 32 columns a workgroup)
@pytest.mark.parametrize("M,N", [(5, 40), (30, 41), (24, 700), (100, 1503), (300, 280), (400, 701), (1000, 1601), (1701, 1750), (3601, 3570), (3, 8209)])
@pytest.mark.parametrize("K", [70, 1700])
@pytest.mark.parametrize("together,every", [(0, 1), (-100, 1), (90, 1), (0, 7)])
@pytest.mark.parametrize("cdt", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("fa,fb", PAIRS)
def test_gemm_of_any_scales(ctx, fa, fb, cdt, together, every, K, M, N):
    a, A, As, b, Bm, Bs = spread_matrices(M, N, K, fa, fb, 7 * M + K, together, every)
    C = torch.full((M, up(N, 8)), float("nan"), dtype=TYPES[cdt], device="cuda")[:, :N]
    ctx.dq_gemm_mx(M, N, K, fa, A, As, fb, Bm, Bs, C, cdt)
    if M * N > 100000:                     # only the reference and its bound are formed by a library: fp64, on the GPU
        ad, bd = torch.from_numpy(a).cuda(), torch.from_numpy(b).cuda().t().contiguous()
        ref, s = (ad @ bd).cpu().numpy(), (ad.abs() @ bd.abs()).cpu().numpy()
    else:
        ref, s = a @ b.T, np.abs(a) @ np.abs(b).T
    tol = s * (4 * -(-K // 128) + 16) * 2.0 ** -23                      # as product_bound
    if cdt == B.DQ_BF16:
        tol += np.abs(ref) * 2.0 ** -8 + (s * 2.0 ** -11 if B.DQ_MXFP8 in (fa, fb) else 0.0)
    got = C.double().cpu().numpy()
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= tol + 1e-38).all()
    again = torch.empty((M, up(N, 8)), dtype=TYPES[cdt], device="cuda")[:, :N]
    ctx.dq_gemm_mx(M, N, K, fa, A, As, fb, Bm, Bs, again, cdt)
    assert torch.equal(C, again)


@pytest.mark.parametrize("M,N", [(5, 400), (30, 300), (24, 700), (100, 1503), (300, 400), (400, 701), (1000, 1601), (1701, 1750)])
@pytest.mark.parametrize("fa,fb", [(1, 0), (0, 1), (1, 1)])
def test_gemm_of_large_scales_is_as_near_as_of_small_ones(ctx, fa, fb, M, N):
    """Normal values, A's times 2^60 and B's times 2^-60: 32 steps of 64, each eight sums.  256 roundings of at most 2^-24 of C's norm, of independent signs,
    add up to 16 of them; summed to 14 bits eight at a time they would be off by 4e-6 (8 x 4 bits) to 1.5e-5 (8 x 8)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(M)
    K, parts, vals = 2048, [], []
    for rows, fmt, factor in ((M, fa, 2.0 ** 60), (N, fb, 2.0 ** -60)):
        X = torch.randn((rows, K), device="cuda", generator=g) * factor
        c, s = stored(rows, K, fmt)
        ctx.dq_mx_quantize(X, B.DQ_F32, fmt, c, s)
        Y = torch.empty_like(X)
        ctx.dq_mx_dequantize(fmt, c, s, Y, B.DQ_F32)
        parts.append((c, s))
        vals.append(Y.double())
    ref = vals[0] @ vals[1].t().contiguous()
    C = torch.empty((M, up(N, 4)), device="cuda")[:, :N]
    ctx.dq_gemm_mx(M, N, K, fa, *parts[0], fb, *parts[1], C, B.DQ_F32)
    assert float(torch.linalg.norm(C.double() - ref)) <= 2e-6 * float(torch.linalg.norm(ref))


@pytest.mark.parametrize("M,N,K", [(8, 4000, 2048), (30, 1000, 2048), (300, 400, 2048), (300, 400, 16384), (2300, 2100, 1024), (3600, 3500, 512)])
@pytest.mark.parametrize("fa,fb", PAIRS)
def test_gemm_of_normal_values_before_the_rounding_to_bf16(ctx, fa, fb, M, N, K):
    """How far a bf16 result is off before its rounding, from the elements that it rounds otherwise than the exact product does.  Where two values e apart
    lie in cells of u, they are rounded apart, by u, with a chance of e / u; so the squared distance D^2 of the two rounded results comes to
    sum |e| u <= ||e|| ||u|| <= 1e-4 ||C|| 2^-7 ||C|| where e is within the documented 1e-4 of C's norm (u <= 2^-7 |c|).  Counts of some hundred and more such
    elements: a fifth more for their scatter.  For 4 x 4 bits, whose sums are fp32, 1e-5 is allowed in place of 1e-4."""
    g = torch.Generator(device="cuda")
    g.manual_seed(M + K)
    parts, vals = [], []
    for rows, fmt in ((M, fa), (N, fb)):
        X = torch.randn((rows, K), device="cuda", generator=g)
        c, s = stored(rows, K, fmt)
        ctx.dq_mx_quantize(X, B.DQ_F32, fmt, c, s)
        Y = torch.empty_like(X)
        ctx.dq_mx_dequantize(fmt, c, s, Y, B.DQ_F32)
        parts.append((c, s))
        vals.append(Y.double())
    ref = vals[0] @ vals[1].t().contiguous()
    H = torch.empty((M, up(N, 8)), device="cuda", dtype=torch.bfloat16)[:, :N]
    ctx.dq_gemm_mx(M, N, K, fa, *parts[0], fb, *parts[1], H, B.DQ_BF16)
    apart = H.double() - ref.bfloat16().double()
    norm = float(torch.linalg.norm(ref))
    bound = (1e-4 if B.DQ_MXFP8 in (fa, fb) else 1e-5) * 2.0 ** -7 * 1.2
    assert float(torch.linalg.norm(apart)) ** 2 <= bound * norm ** 2


@pytest.mark.parametrize("M,N", [(8, 400), (30, 1000), (300, 400), (2300, 2100)])
@pytest.mark.parametrize("cdt", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("fa,fb", PAIRS)
def test_gemm_whose_large_products_cancel(ctx, fa, fb, cdt, M, N):
    """A channel that stands far above the others meets weights that cancel it: the documented bound goes with the sum of magnitudes, not with C."""
    K = 1024
    g = rng(M)
    a, b = g.standard_normal((M, K)), g.standard_normal((N, K))
    a[:, 0::64], b[:, 1::64] = 300.0, -b[:, 0::64]
    a[:, 1::64] = a[:, 0::64]
    parts, vals = [], []
    for rows, fmt, x in ((M, fa, a), (N, fb, b)):
        c, s = stored(rows, K, fmt)
        ctx.dq_mx_quantize(torch.from_numpy(x).float().cuda(), B.DQ_F32, fmt, c, s)
        Y = torch.empty((rows, K), device="cuda")
        ctx.dq_mx_dequantize(fmt, c, s, Y, B.DQ_F32)
        parts.append((c, s))
        vals.append(Y.double().cpu().numpy())
    ref = vals[0] @ vals[1].T
    C = torch.empty((M, up(N, 8)), device="cuda", dtype=TYPES[cdt])[:, :N]
    ctx.dq_gemm_mx(M, N, K, fa, *parts[0], fb, *parts[1], C, cdt)
    got = C.double().cpu().numpy()
    assert (np.abs(got - ref) <= product_bound(*vals, ref, K, fa, fb, cdt)).all()


# up to 16 rows against 8192 columns and more: 32 columns a workgroup
@pytest.mark.parametrize("M,N,K", [(1, 8200, 1000), (9, 8209, 545), (16, 9001, 4096), (3, 8193, 31)])
@pytest.mark.parametrize("cdt", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("fa,fb", PAIRS)
def test_gemm_of_few_rows_and_many_columns(ctx, fa, fb, cdt, M, N, K):
    a, A, As = random_matrix(M, K, fa, 5 * M + K)
    b, Bm, Bs = random_matrix(N, K, fb, 3 * N + K)
    buf, C = view(M, N, up(N, 8) + 8, TYPES[cdt], 7.0)
    ctx.dq_gemm_mx(M, N, K, fa, A, As, fb, Bm, Bs, C, cdt)
    ref = a @ b.T
    assert (np.abs(C.double().cpu().numpy() - ref) <= product_bound(a, b, ref, K, fa, fb, cdt)).all()
    assert (buf[:, N:] == 7.0).all()
    As[M - 1, (K - 1) // 32] = 255                              # the last block, cut short
    Bs[N - 2, 0] = 255
    bad = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    bad[M - 1], bad[:, N - 2] = True, True
    D = torch.empty_like(buf)[:, :N]
    ctx.dq_gemm_mx(M, N, K, fa, A, As, fb, Bm, Bs, D, cdt)
    assert torch.equal(torch.isnan(D), bad)
    got = torch.where(bad, torch.from_numpy(ref).cuda(), D.double()).cpu().numpy()
    assert (np.abs(got - ref) <= product_bound(a, b, ref, K, fa, fb, cdt)).all()


@pytest.mark.parametrize("cdt", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("fa,fb", PAIRS)
def test_gemm_of_rows_far_apart_and_many_columns(ctx, fa, fb, cdt):
    """Rows of A, then of B, 8 MiB apart and more: B's last one starts 64 GiB behind the first."""
    M, N, K, far = 37, 8209, 700, (1 << 23) + 64
    a, A, As = random_matrix(M, K, fa, 91)
    b, Bm, Bs = random_matrix(N, K, fb, 92)
    ref = a @ b.T
    for spread in ("a", "b"):
        src = A if spread == "a" else Bm
        wide = torch.empty((src.shape[0], far), dtype=torch.uint8, device="cuda")[:, :src.shape[1]]
        wide.copy_(src)
        C = torch.empty((M, up(N, 8)), dtype=TYPES[cdt], device="cuda")[:, :N]
        ctx.dq_gemm_mx(M, N, K, fa, wide if spread == "a" else A, As, fb, wide if spread == "b" else Bm, Bs, C, cdt)
        assert (np.abs(C.double().cpu().numpy() - ref) <= product_bound(a, b, ref, K, fa, fb, cdt)).all()
        del wide


@pytest.mark.parametrize("cdt", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("fa,fb", PAIRS)
@pytest.mark.parametrize("M", [9, 40, 300])
def test_gemm_whose_last_rows_of_b_start_beyond_32_bits(ctx, M, fa, fb, cdt):
    """The product of rows of B 64 KiB apart gives the bits of the same rows close together."""
    N, K, far = 70001, 96, 65536
    _, A, As = random_matrix(M, K, fa, 81)
    _, Bm, Bs = random_matrix(N, K, fb, 82)
    wide = torch.empty((N, far), dtype=torch.uint8, device="cuda")
    wide[:, :Bm.shape[1]] = Bm
    scales = wide[:, 32768:32768 + Bs.shape[1]]
    scales.copy_(Bs)
    C = [torch.empty((M, up(N, 8)), dtype=TYPES[cdt], device="cuda")[:, :N] for _ in range(2)]
    ctx.dq_gemm_mx(M, N, K, fa, A, As, fb, Bm, Bs, C[0], cdt)
    ctx.dq_gemm_mx(M, N, K, fa, A, As, fb, wide[:, :Bm.shape[1]], scales, C[1], cdt)
    assert torch.equal(C[0], C[1])
    vals = []
    for rows, fmt, c, s in ((M, fa, A, As), (4001, fb, Bm[N - 4001:], Bs[N - 4001:])):
        Y = torch.empty((rows, K), device="cuda")
        ctx.dq_mx_dequantize(fmt, c, s, Y, B.DQ_F32)
        vals.append(Y.double().cpu().numpy())
    ref = vals[0] @ vals[1].T
    got = C[1][:, N - 4001:].double().cpu().numpy()
    assert (np.abs(got - ref) <= product_bound(vals[0], vals[1], ref, K, fa, fb, cdt)).all()
