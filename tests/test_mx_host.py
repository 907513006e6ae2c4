"""What the MX entry points refuse before anything is launched.  No GPU: a context of zeros stands in, which none of these calls gets to use."""

import ctypes
import os

import pytest

from paper_2511_04063_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2511_04063_amd.build import build_library
        build_library(verbose=False)
    return B.load_library()


@pytest.fixture(scope="module")
def ctx():
    store = ctypes.create_string_buffer(1 << 16)
    return ctypes.c_void_p(ctypes.addressof(store)), store


MOST = 2 ** 31 - 1024
P, Q, ODD = 1 << 20, 1 << 21, (1 << 20) + 8            # never dereferenced


def test_row_bytes(lib):
    assert B.dq_mx_row_bytes(B.DQ_MXFP4, 1) == (16, 16) and B.dq_mx_row_bytes(B.DQ_MXFP8, 32) == (32, 16)
    assert B.dq_mx_row_bytes(B.DQ_MXFP4, 513) == (17 * 16, 32) and B.dq_mx_row_bytes(B.DQ_MXFP8, 4096) == (4096, 128)
    assert B.dq_mx_row_bytes(B.DQ_MXFP8, 2 ** 31 - 1) == (2 ** 31, 2 ** 26)
    out = ctypes.c_size_t(0)
    assert lib.dq_mx_row_bytes(0, 8, None, ctypes.byref(out)) == B.DQ_ERR_NULL
    assert lib.dq_mx_row_bytes(0, 0, ctypes.byref(out), ctypes.byref(out)) == B.DQ_ERR_SHAPE
    assert lib.dq_mx_row_bytes(2, 8, ctypes.byref(out), ctypes.byref(out)) == B.DQ_ERR_DTYPE


def changed(base, **more):
    return list({**base, **more}.values())


def test_quantize_refuses(lib, ctx):
    ok = dict(ctx=ctx[0], T=4, n=40, X=P, xdt=B.DQ_F32, ldx=40, fmt=B.DQ_MXFP4, codes=Q, ldc=32, scales=Q, lds=16)
    call = lib.dq_mx_quantize
    assert call(*changed(ok)) == B.DQ_ERR_WORKSPACE                       # everything else is right
    for status, wrong in [(B.DQ_ERR_NULL, dict(ctx=None)), (B.DQ_ERR_NULL, dict(X=None)), (B.DQ_ERR_NULL, dict(codes=None)),
                          (B.DQ_ERR_NULL, dict(scales=None)), (B.DQ_ERR_SHAPE, dict(T=-1)), (B.DQ_ERR_SHAPE, dict(n=0)),
                          (B.DQ_ERR_SHAPE, dict(ldx=36)), (B.DQ_ERR_SHAPE, dict(ldc=16)), (B.DQ_ERR_SHAPE, dict(fmt=B.DQ_MXFP8)),
                          (B.DQ_ERR_SHAPE, dict(n=520, ldx=520, ldc=272)), (B.DQ_ERR_DTYPE, dict(xdt=2)), (B.DQ_ERR_DTYPE, dict(fmt=2)),
                          (B.DQ_ERR_DTYPE, dict(fmt=-1)), (B.DQ_ERR_ALIGN, dict(X=ODD)), (B.DQ_ERR_ALIGN, dict(codes=ODD)),
                          (B.DQ_ERR_ALIGN, dict(scales=ODD)), (B.DQ_ERR_ALIGN, dict(ldx=42)), (B.DQ_ERR_ALIGN, dict(ldc=40)),
                          (B.DQ_ERR_ALIGN, dict(lds=24)), (B.DQ_ERR_ALIGN, dict(xdt=B.DQ_BF16, ldx=44))]:
        assert call(*changed(ok, **wrong)) == status, wrong
    assert call(*changed(ok, T=0, X=None)) == B.DQ_OK
    far = dict(ldx=2 ** 32, ldc=2 ** 32, lds=2 ** 32)
    for size in ("T", "n"):
        assert call(*changed(ok, **far, **{size: MOST})) == B.DQ_ERR_WORKSPACE
        assert call(*changed(ok, **far, **{size: MOST + 1})) == B.DQ_ERR_UNSUPPORTED


def test_dequantize_refuses(lib, ctx):
    ok = dict(ctx=ctx[0], T=4, n=40, fmt=B.DQ_MXFP4, codes=Q, ldc=32, scales=Q, lds=16, Y=P, ydt=B.DQ_F32, ldy=40)
    for status, wrong in [(B.DQ_ERR_NULL, dict(ctx=None)), (B.DQ_ERR_NULL, dict(Y=None)), (B.DQ_ERR_NULL, dict(codes=None)),
                          (B.DQ_ERR_NULL, dict(scales=None)), (B.DQ_ERR_SHAPE, dict(T=-1)), (B.DQ_ERR_SHAPE, dict(n=0)),
                          (B.DQ_ERR_SHAPE, dict(ldy=36)), (B.DQ_ERR_SHAPE, dict(ldc=16)), (B.DQ_ERR_SHAPE, dict(lds=0)),
                          (B.DQ_ERR_DTYPE, dict(ydt=2)), (B.DQ_ERR_DTYPE, dict(fmt=2)), (B.DQ_ERR_ALIGN, dict(Y=ODD)),
                          (B.DQ_ERR_ALIGN, dict(codes=ODD)), (B.DQ_ERR_ALIGN, dict(ldy=42)), (B.DQ_ERR_ALIGN, dict(ydt=B.DQ_BF16, ldy=44))]:
        assert lib.dq_mx_dequantize(*changed(ok, **wrong)) == status, wrong
    assert lib.dq_mx_dequantize(*changed(ok, T=0, Y=None)) == B.DQ_OK
    for size in ("T", "n"):
        assert lib.dq_mx_dequantize(*changed(ok, **{size: MOST + 1})) == B.DQ_ERR_UNSUPPORTED


def test_rms_norm_refuses(lib, ctx):
    ok = dict(ctx=ctx[0], T=4, n=40, X=P, xdt=B.DQ_BF16, ldx=40, res=Q, ldr=48, H=Q + 4096, ldh=40, gain=Q, eps=1e-5, fmt=B.DQ_MXFP8, codes=Q,
              ldc=64, scales=Q, lds=16)
    call = lib.dq_mx_rms_norm
    assert call(*changed(ok)) == B.DQ_ERR_WORKSPACE
    assert call(*changed(ok, res=None, ldr=0, H=None, ldh=0, gain=None, eps=0.0)) == B.DQ_ERR_WORKSPACE
    assert call(*changed(ok, H=P)) == B.DQ_ERR_WORKSPACE and call(*changed(ok, H=Q, ldh=48)) == B.DQ_ERR_WORKSPACE
    for status, wrong in [(B.DQ_ERR_NULL, dict(ctx=None)), (B.DQ_ERR_NULL, dict(X=None)), (B.DQ_ERR_NULL, dict(codes=None)),
                          (B.DQ_ERR_NULL, dict(scales=None)), (B.DQ_ERR_SHAPE, dict(T=-1)), (B.DQ_ERR_SHAPE, dict(n=0)),
                          (B.DQ_ERR_UNSUPPORTED, dict(n=B.DQ_MAX_N + 1)), (B.DQ_ERR_UNSUPPORTED, dict(T=MOST + 1)), (B.DQ_ERR_SHAPE, dict(eps=-1e-6)), (B.DQ_ERR_SHAPE, dict(eps=float("nan"))),
                          (B.DQ_ERR_SHAPE, dict(eps=float("inf"))), (B.DQ_ERR_SHAPE, dict(ldr=32)), (B.DQ_ERR_SHAPE, dict(ldh=32)),
                          (B.DQ_ERR_SHAPE, dict(H=Q, ldh=40)), (B.DQ_ERR_SHAPE, dict(H=P, ldh=48)), (B.DQ_ERR_SHAPE, dict(ldc=32)),
                          (B.DQ_ERR_DTYPE, dict(xdt=2)), (B.DQ_ERR_DTYPE, dict(fmt=2)), (B.DQ_ERR_ALIGN, dict(res=ODD)), (B.DQ_ERR_ALIGN, dict(H=ODD)),
                          (B.DQ_ERR_ALIGN, dict(gain=Q + 4)), (B.DQ_ERR_ALIGN, dict(ldx=44)), (B.DQ_ERR_ALIGN, dict(scales=ODD))]:
        assert call(*changed(ok, **wrong)) == status, wrong
    assert call(*changed(ok, T=0, X=None)) == B.DQ_OK


def test_gemm_refuses(lib, ctx):
    ok = dict(ctx=ctx[0], M=4, N=12, K=40, fa=B.DQ_MXFP8, A=P, lda=64, As=P, ldas=16, fb=B.DQ_MXFP4, B=Q, ldb=32, Bs=Q, ldbs=16, C=P, cdt=B.DQ_BF16,
              ldc=16)
    for status, wrong in [(B.DQ_ERR_NULL, dict(ctx=None)), (B.DQ_ERR_NULL, dict(A=None)), (B.DQ_ERR_NULL, dict(As=None)), (B.DQ_ERR_NULL, dict(B=None)),
                          (B.DQ_ERR_NULL, dict(Bs=None)), (B.DQ_ERR_NULL, dict(C=None)), (B.DQ_ERR_SHAPE, dict(M=-1)), (B.DQ_ERR_SHAPE, dict(N=-1)),
                          (B.DQ_ERR_SHAPE, dict(K=0)), (B.DQ_ERR_SHAPE, dict(lda=48)), (B.DQ_ERR_SHAPE, dict(ldb=16)), (B.DQ_ERR_SHAPE, dict(ldc=8)),
                          (B.DQ_ERR_SHAPE, dict(K=520, lda=544, ldb=272)), (B.DQ_ERR_DTYPE, dict(fa=2)), (B.DQ_ERR_DTYPE, dict(fb=-1)),
                          (B.DQ_ERR_DTYPE, dict(cdt=2)), (B.DQ_ERR_ALIGN, dict(A=ODD)), (B.DQ_ERR_ALIGN, dict(Bs=ODD)), (B.DQ_ERR_ALIGN, dict(ldas=20)),
                          (B.DQ_ERR_ALIGN, dict(ldc=12)), (B.DQ_ERR_ALIGN, dict(C=ODD))]:
        assert lib.dq_gemm_mx(*changed(ok, **wrong)) == status, wrong
    for size, most in (("M", 2 ** 26), ("N", 2 ** 26), ("K", MOST)):
        assert lib.dq_gemm_mx(*changed(ok, **{size: most + 1})) == B.DQ_ERR_UNSUPPORTED
    assert lib.dq_gemm_mx(*changed(ok, M=0, A=None)) == B.DQ_OK and lib.dq_gemm_mx(*changed(ok, N=0)) == B.DQ_OK


def test_objectives_are_checked_like_the_others(lib, ctx):
    for obj in (B.DQ_OBJ_MXFP4, B.DQ_OBJ_MXFP8):
        assert lib.dq_objective_loss_grad(None, obj, 4, 1, 8, 8, P, 8, 0, P, P, 0, 8) == B.DQ_ERR_NULL
        assert lib.dq_objective_loss_grad(ctx[0], obj, 4, 1, 8, 8, P, 8, 0, Q, Q, 0, 8) == B.DQ_ERR_WORKSPACE
        assert lib.dq_objective_loss_grad(ctx[0], obj, 4, 1, 8, B.DQ_MAX_N + 8, P, B.DQ_MAX_N + 8, 0, Q, Q, 0, B.DQ_MAX_N + 8) == B.DQ_ERR_UNSUPPORTED
        assert lib.dq_objective_loss_grad(ctx[0], obj, 4, 1, 8, 8, P, 8, 0, Q, Q, 2, 8) == B.DQ_ERR_DTYPE
    assert lib.dq_objective_loss_grad(ctx[0], 6, 4, 1, 8, 8, P, 8, 0, Q, Q, 0, 8) == B.DQ_ERR_DTYPE
    assert lib.dq_objective_loss_grad(ctx[0], -1, 4, 1, 8, 8, P, 8, 0, Q, Q, 0, 8) == B.DQ_ERR_DTYPE
