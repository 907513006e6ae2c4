// Product of two MX matrices on the matrix cores:  C (M x N) = A B^T, A (M x K) and B (N x K) rows of MX blocks, C fp32 or bf16.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 codes by 16 x 128 codes and applies the block scales itself (four lanes hold a row's
// four blocks; lane l: row l % 16, block l / 16).  4-bit operands: 16 bytes a lane, its block.  8-bit ones: two times 16 bytes, k = 16 g .. and
// k = 64 + 16 g .. for g = l / 16, while the lane's scale is still that of block g.  B is passed as the first operand, so a lane ends up with four
// neighbouring columns of one row of C: register v holds C[m = l % 16][n = 4 (l / 16) + v].
//
// Eight products at a time (k = 8 j .. 8 j + 7) are summed inside the instruction with about 14 bits below the largest of them when an operand has 8-bit
// codes: normal values come out with an error of 1.5e-5 of the result's norm (8 x 8 bits) or 4e-6 (8 x 4), far below a bf16 result's rounding;
// 4 x 4 bits show none.  A caller who asks for fp32 gets fp32 sums: there 8-bit operands (and what they meet) go to the bf16 matrix cores,
// value times scale being exact in bf16.
#include "dq_mx.h"

namespace dq {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// operand format as the instruction counts it
template <int F> constexpr int kMfmaFormat = F == DQ_MXFP4 ? 4 : 0;
template <int F> constexpr int kStepBytes = F == DQ_MXFP4 ? 64 : 128;       // 128 codes

template <int F> struct Codes { i32x4 a; i32x4 b; };
template <> struct Codes<DQ_MXFP4> { i32x4 a; };

template <int F>
__device__ __forceinline__ i32x8 operand(const Codes<F>& c) {
    if constexpr (F == DQ_MXFP4) return __builtin_shufflevector(c.a, c.a, 0, 1, 2, 3, -1, -1, -1, -1);
    else return __builtin_shufflevector(c.a, c.b, 0, 1, 2, 3, 4, 5, 6, 7);
}

template <int FA, int FB>
__device__ __forceinline__ f32x4 mfma_mx(const Codes<FA>& a, const Codes<FB>& b, f32x4 c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand<FA>(a), operand<FB>(b), c, kMfmaFormat<FA>, kMfmaFormat<FB>, 0, sa, 0, sb);
}

// this lane's codes of 128 of a row (`step` counts 128s); blocks from nb on are zeros and are not read
template <int F, bool WIDE>
__device__ __forceinline__ Codes<F> load_codes(const unsigned char* row, int step, int g, int nb) {
    const i32x4 zero = {0, 0, 0, 0};
    Codes<F> c;
    const unsigned char* p = row + (long)step * kStepBytes<F>;
    if constexpr (F == DQ_MXFP4) {
        c.a = 4 * step + g < nb ? *reinterpret_cast<const i32x4*>(p + 16 * g) : zero;
    } else if constexpr (WIDE) {
        const bool in = 4 * step + g < nb;
        c.a = in ? *reinterpret_cast<const i32x4*>(p + 32 * g) : zero;
        c.b = in ? *reinterpret_cast<const i32x4*>(p + 32 * g + 16) : zero;
    } else {
        c.a = 4 * step + g / 2 < nb ? *reinterpret_cast<const i32x4*>(p + 16 * g) : zero;
        c.b = 4 * step + 2 + g / 2 < nb ? *reinterpret_cast<const i32x4*>(p + 64 + 16 * g) : zero;
    }
    return c;
}
__device__ __forceinline__ unsigned load_scale(const unsigned char* row, int step, int g, int nb) {
    return 4 * step + g < nb ? row[4 * step + g] : 0u;
}

// codes [8 j, 8 j + 8) of this lane's 32 (loaded WIDE), times their scale, in bf16
template <int F, int J>
__device__ __forceinline__ bf16x8 values8(const Codes<F>& c, unsigned byte) {
    const float s = mx_scale(byte);
    unsigned w[4];
    if constexpr (F == DQ_MXFP4) {
        const unsigned u = (unsigned)c.a[J];
        w[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 0));
        w[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 1));
        w[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 2));
        w[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 3));
    } else {
        const unsigned u = (unsigned)(J < 2 ? c.a[2 * J] : c.b[2 * J - 4]), v = (unsigned)(J < 2 ? c.a[2 * J + 1] : c.b[2 * J - 3]);
        w[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, s, false));
        w[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, s, true));
        w[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, s, false));
        w[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, s, true));
    }
    i32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = byte == 255u ? 0x7fc07fc0 : (int)w[i];
    return __builtin_bit_cast(bf16x8, r);
}

template <int FA, int FB>
__device__ __forceinline__ f32x4 mfma_values(const Codes<FA>& a, const Codes<FB>& b, f32x4 c, unsigned sa, unsigned sb) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values8<FA, 0>(a, sa), values8<FB, 0>(b, sb), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values8<FA, 1>(a, sa), values8<FB, 1>(b, sb), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values8<FA, 2>(a, sa), values8<FB, 2>(b, sb), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(values8<FA, 3>(a, sa), values8<FB, 3>(b, sb), c, 0, 0, 0);
}

template <class OUT>
__device__ __forceinline__ void store4(OUT* dst, int left, f32x4 v) {
    if constexpr (sizeof(OUT) == 4) {
        store_quad(dst, left, make_float4(v[0], v[1], v[2], v[3]));
    } else {
        const mx_f32x2 a = {v[0], v[1]}, b = {v[2], v[3]};
        const unsigned w0 = __builtin_bit_cast(unsigned, __builtin_convertvector(a, mx_bf16x2));
        const unsigned w1 = __builtin_bit_cast(unsigned, __builtin_convertvector(b, mx_bf16x2));
        if (left >= 4) {
            *reinterpret_cast<uint2*>(dst) = make_uint2(w0, w1);
        } else {
            dst[0] = (bf16_t)w0;
            if (left > 1) dst[1] = (bf16_t)(w0 >> 16);
            if (left > 2) dst[2] = (bf16_t)w1;
        }
    }
}

// ---- straight from memory: a workgroup of 8 wavefronts makes 16 MT rows x 16 columns of C, each wavefront taking every eighth 128 of the
// reduction; the eight sums are added in order through LDS.
template <int FA, int FB, class OUT, int MT>
__global__ __launch_bounds__(512) void gemm_mx_direct_kernel(GemmMx g) {
    constexpr bool EXACT = sizeof(OUT) == 4 && (FA == DQ_MXFP8 || FB == DQ_MXFP8);
    __shared__ f32x4 part[8][MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * (16 * MT);
    const int nb = (int)((g.K + 31L) / 32), steps = (nb + 3) / 4;
    const int nr = n0 + r < g.N ? n0 + r : g.N - 1;
    const unsigned char* pb = g.B + (long)nr * g.ldb;
    const unsigned char* sb = g.Bs + (long)nr * g.ldbs;
    const unsigned char* pa[MT];
    const unsigned char* sa[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int mr = m0 + 16 * i + r < g.M ? m0 + 16 * i + r : g.M - 1;
        pa[i] = g.A + (long)mr * g.lda;
        sa[i] = g.As + (long)mr * g.ldas;
    }
    f32x4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int t = wave; t < steps; t += 8) {
        const Codes<FB> b = load_codes<FB, EXACT>(pb, t, q, nb);
        const unsigned eb = load_scale(sb, t, q, nb);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const Codes<FA> a = load_codes<FA, EXACT>(pa[i], t, q, nb);
            const unsigned ea = load_scale(sa[i], t, q, nb);
            if constexpr (EXACT) acc[i] = mfma_values<FB, FA>(b, a, acc[i], eb, ea);
            else acc[i] = mfma_mx<FB, FA>(b, a, acc[i], (int)eb, (int)ea);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) part[wave][i][lane] = acc[i];
    __syncthreads();
    if (wave < MT) {
        f32x4 c = part[0][wave][lane];
#pragma unroll
        for (int k = 1; k < 8; ++k) c += part[k][wave][lane];
        const int m = m0 + 16 * wave + r, n = n0 + 4 * q;
        if (m < g.M && n < g.N) store4(static_cast<OUT*>(g.C) + (long)m * g.ldc + n, g.N - n, c);
    }
}

template <int FA, int FB, class OUT>
hipError_t launch_types(const GemmMx& g, hipStream_t s) {
    const unsigned gx = (unsigned)((g.N + 15L) / 16);
    if (g.M <= 16) hipLaunchKernelGGL((gemm_mx_direct_kernel<FA, FB, OUT, 1>), dim3(gx, 1), dim3(512), 0, s, g);
    else hipLaunchKernelGGL((gemm_mx_direct_kernel<FA, FB, OUT, 4>), dim3(gx, (unsigned)((g.M + 63L) / 64)), dim3(512), 0, s, g);
    return hipGetLastError();
}

template <int FA, int FB>
hipError_t launch_out(const GemmMx& g, hipStream_t s) {
    return g.c_is_bf16 ? launch_types<FA, FB, bf16_t>(g, s) : launch_types<FA, FB, float>(g, s);
}

}  // namespace

hipError_t launch_gemm_mx(const GemmMx& g, hipStream_t s) {
    if (g.M <= 0 || g.N <= 0) return hipSuccess;
    if (g.fa == DQ_MXFP4) return g.fb == DQ_MXFP4 ? launch_out<DQ_MXFP4, DQ_MXFP4>(g, s) : launch_out<DQ_MXFP4, DQ_MXFP8>(g, s);
    return g.fb == DQ_MXFP4 ? launch_out<DQ_MXFP8, DQ_MXFP4>(g, s) : launch_out<DQ_MXFP8, DQ_MXFP8>(g, s);
}

}  // namespace dq
