// Product of two MX matrices on the matrix cores:  C (M x N) = A B^T, A (M x K) and B (N x K) rows of MX blocks, C fp32 or bf16.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 codes by 16 x 128 codes and applies the block scales itself (four lanes hold a row's
// four blocks; lane l: row l % 16, block l / 16).  4-bit operands: 16 bytes a lane, its block.  8-bit ones: two times 16 bytes, k = 16 g .. and
// k = 64 + 16 g .. for g = l / 16, while the lane's scale is still that of block g.  B is passed as the first operand, so a lane ends up with four
// neighbouring columns of one row of C: register v holds C[m = l % 16][n = 4 (l / 16) + v].
//
// Eight products at a time (k = 8 j .. 8 j + 7) are summed inside the instruction with about 14 bits below the largest of them when an operand has 8-bit
// codes, an error of at most 2^-11 of the magnitudes that are summed.  Normal values come out with 1.5e-5 of the result's norm (8 x 8 bits) or 4e-6 (8 x 4), of
// K = 512 as of 16384, a hundredth of what a bf16 result's rounding makes; where a channel 300 times the others meets weights that cancel it, 3.3e-3, twice
// the rounding.  4 x 4 bits show none.  A bf16 result takes it, for 2.2 times the rate of the exact route below.  A caller who asks for fp32 gets fp32 sums: there 8-bit operands (and what they meet) go to the bf16 matrix cores,
// as value times scale times 2^20, which bf16 holds exactly for scales below 2^17 (2^-127 2^-9 2^20 is a normal number; 2^31 products of two largest
// ones stay below 2^121), and the sums lose the 2^40 at the end.  A wavefront that meets a larger scale, which takes values of 2^19 (4 bits) or 2^25 and
// more, forms its sums again: by the scaled instruction, which holds any scales, with all but one of each eight codes of A masked, eight times, so that
// nothing is lost (8192^3 of 8 x 8 bits 870 us, with large scales everywhere 5.8 ms).
#include "dq_mx.h"

namespace dq {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
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

constexpr int kLift = 20;                                    // the fp32 route's values are 2^20 times what they stand for
constexpr float kLower = 1.f / (1L << 2 * kLift);
constexpr unsigned kLargeScale = 127u + 17u;                 // scale bytes from here on, but 255, are too large for it
// nonzero where one of the four scale bytes of a word is: its highest bit and one of the next three, and not all of them
__device__ __forceinline__ unsigned large_scales(unsigned w) { return w & (w << 1 | w << 2 | w << 3) & ~((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ bool large_scale(unsigned byte) { return byte - kLargeScale < 255u - kLargeScale; }
static_assert(kLargeScale == 0x90u, "large_scales looks at these bits");

// codes [8 j, 8 j + 8) of this lane's 32 (loaded WIDE), times their scale and 2^20, in bf16; scale 255 makes the conversions' results NaN
template <int F, int J>
__device__ __forceinline__ bf16x8 values8(const Codes<F>& c, unsigned byte) {
    const float s = __uint_as_float(((byte < 255u - kLift ? byte : 255u - kLift) + kLift) << 23);
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
    for (int i = 0; i < 4; ++i) r[i] = (int)w[i];
    return __builtin_bit_cast(bf16x8, r);
}

template <int FA, int FB>
__device__ __forceinline__ f32x4 mfma_values(const Codes<FA>& a, const Codes<FB>& b, f32x4 c, unsigned sa, unsigned sb) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values8<FA, 0>(a, sa), values8<FB, 0>(b, sb), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values8<FA, 1>(a, sa), values8<FB, 1>(b, sb), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values8<FA, 2>(a, sa), values8<FB, 2>(b, sb), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(values8<FA, 3>(a, sa), values8<FB, 3>(b, sb), c, 0, 0, 0);
}

// of each eight neighbouring codes the j-th alone
template <int F>
__device__ __forceinline__ Codes<F> one_of_eight(Codes<F> c, int j) {
    if constexpr (F == DQ_MXFP4) {
#pragma unroll
        for (int w = 0; w < 4; ++w) c.a[w] &= (int)(0xfu << (4 * j));
    } else {
        const unsigned m[2] = {j < 4 ? 0xffu << (8 * j) : 0u, j < 4 ? 0u : 0xffu << (8 * (j - 4))};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            c.a[w] &= (int)m[w & 1];
            c.b[w] &= (int)m[w & 1];
        }
    }
    return c;
}

// This lane's codes and scale of 64 of a row, as the 32 x 32 x 64 instruction takes them; as load_codes
template <int F>
__device__ __forceinline__ Codes<F> load_codes64(const unsigned char* row, int step, int q, int nb) {
    const i32x4 zero = {0, 0, 0, 0};
    const unsigned char* p = row + (long)step * (kStepBytes<F> / 2) + 16 * q;
    Codes<F> c;
    if constexpr (F == DQ_MXFP4) {
        c.a = 2 * step + q < nb ? *reinterpret_cast<const i32x4*>(p) : zero;
    } else {
        c.a = *reinterpret_cast<const i32x4*>(p);
        c.b = 2 * step + 1 < nb ? *reinterpret_cast<const i32x4*>(p + 32) : zero;
    }
    return c;
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

// ---- straight from memory, for small products: a workgroup of 8 wavefronts makes 16 MT rows x 16 NT columns of C.  Each wavefront takes every
// eighth piece of 512 of the reduction (a row's 16 scales, one load) and has all of a piece's operands under way at once; the eight sums are added in
// order through LDS.  Bound by one latency from launch to store: 1 x 4096, 4096 of 4 x 4 bits 4.0 us, of which a kernel of no work takes 2 and the 8.9
// MB of B, at the rate of a large copy, 1.7; 300 x 300, 300 3.0.
template <int FA, int FB, class OUT, int MT, int NT>
__global__ __launch_bounds__(512) void gemm_mx_direct_kernel(GemmMx g, int tiles_n) {
    constexpr bool EXACT = sizeof(OUT) == 4 && (FA == DQ_MXFP8 || FB == DQ_MXFP8);
    __shared__ f32x4 part[8][MT * NT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int n0 = (int)(blockIdx.x % (unsigned)tiles_n) * (16 * NT), m0 = (int)(blockIdx.x / (unsigned)tiles_n) * (16 * MT);
    const int nb = (int)((g.K + 31L) / 32);
    const unsigned char *pa[MT], *sa[MT], *pb[NT], *sb[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int row = m0 + 16 * i + r < g.M ? m0 + 16 * i + r : g.M - 1;
        pa[i] = g.A + (long)row * g.lda;
        sa[i] = g.As + (long)row * g.ldas;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int row = n0 + 16 * j + r < g.N ? n0 + 16 * j + r : g.N - 1;
        pb[j] = g.B + (long)row * g.ldb;
        sb[j] = g.Bs + (long)row * g.ldbs;
    }
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    bool large = false;
    for (int piece = wave; 16 * piece < nb; piece += 8) {
        Codes<FA> a[4][MT];
        Codes<FB> b[4][NT];
        i32x4 ea[MT], eb[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) eb[j] = *reinterpret_cast<const i32x4*>(sb[j] + 16L * piece);
#pragma unroll
        for (int i = 0; i < MT; ++i) ea[i] = *reinterpret_cast<const i32x4*>(sa[i] + 16L * piece);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int j = 0; j < NT; ++j) b[t][j] = load_codes<FB, EXACT>(pb[j], 4 * piece + t, q, nb);
#pragma unroll
            for (int i = 0; i < MT; ++i) a[t][i] = load_codes<FA, EXACT>(pa[i], 4 * piece + t, q, nb);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const bool in = 16 * piece + 4 * t + q < nb;          // what lies behind a row's last scale may be anything
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const unsigned xa = in ? (unsigned)ea[i][t] >> (8 * q) : 0u;
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const unsigned xb = in ? (unsigned)eb[j][t] >> (8 * q) : 0u;
                    if constexpr (EXACT) {
                        large |= large_scale(xa & 255u) || large_scale(xb & 255u);
                        acc[i][j] = mfma_values<FB, FA>(b[t][j], a[t][i], acc[i][j], xb & 255u, xa & 255u);
                    } else acc[i][j] = mfma_mx<FB, FA>(b[t][j], a[t][i], acc[i][j], (int)xb, (int)xa);
                }
            }
        }
    }
    if constexpr (EXACT) {
        const bool again = __any(large);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] *= kLower;
        if (again) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    f32x4 c = {0.f, 0.f, 0.f, 0.f};
                    for (int step = 4 * wave; 4 * step < nb; step += step % 4 == 3 ? 29 : 1) {
                        const int block = 4 * step + q;
                        const int xa = block < nb ? sa[i][block] : 0, xb = block < nb ? sb[j][block] : 0;
                        const Codes<FA> a = load_codes<FA, false>(pa[i], step, q, nb);
                        const Codes<FB> b = load_codes<FB, false>(pb[j], step, q, nb);
                        for (int k = 0; k < 8; ++k) c = mfma_mx<FB, FA>(b, one_of_eight<FA>(a, k), c, xb, xa);
                    }
                    acc[i][j] = c;
                }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) part[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    if (wave < MT * NT) {
        f32x4 c = part[0][wave][lane];
#pragma unroll
        for (int k = 1; k < 8; ++k) c += part[k][wave][lane];
        const int m = m0 + wave / NT * 16 + r, n = n0 + wave % NT * 16 + 4 * q;
        if (m < g.M && n < g.N) store4(static_cast<OUT*>(g.C) + (long)m * g.ldc + n, g.N - n, c);
    }
}

template <int FA, int FB, class OUT, int MT, int NT>
hipError_t launch_direct(const GemmMx& g, hipStream_t s) {
    const long tn = (g.N + 16L * NT - 1) / (16 * NT), tm = (g.M + 16L * MT - 1) / (16 * MT);
    // a launch counts its threads in 32 bits: 2^31 of them at a time
    const long band = tn < (1L << 22) ? (1L << 22) / tn : 1;
    for (long first = 0; first < tm; first += band) {
        const long strips = tm - first < band ? tm - first : band, row = 16 * MT * first;
        GemmMx p = g;
        p.A = g.A + row * g.lda;
        p.As = g.As + row * g.ldas;
        p.C = static_cast<OUT*>(g.C) + row * g.ldc;
        p.M = (int)(g.M - row < 16 * MT * strips ? g.M - row : 16 * MT * strips);
        hipLaunchKernelGGL((gemm_mx_direct_kernel<FA, FB, OUT, MT, NT>), dim3((unsigned)(strips * tn)), dim3(512), 0, s, p, (int)tn);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---- tiles through LDS: a workgroup of 2 x 2 wavefronts makes 64 MI x 64 NI of C, a wavefront 32 MI x 32 NI of it in 32 x 32 x 64 instructions
// (lane l: row l % 32, block l / 32; 8-bit operands k = 16 g .. and k = 32 + 16 g .. for g = l / 32).
//
// The reduction goes in stages of 128 (of 256 where both operands have 4 bits: rows of 128 bytes, whole cache lines; with half of one a transfer the
// requests doubled, and the path to memory was busy 77 % of the time instead of 54).  kStages of them are on their way or in LDS; a lane's 16 bytes
// travel from memory into LDS without passing registers.  What a wavefront waits for in the last step of stage i: its own parts of stage i + 1, with
// kStages - 2 later stages still travelling, then a barrier; behind it stage i + 1 is complete in LDS, and every wavefront has read the last of stage i,
// whose place the parts of stage i + kStages take.
// The fragments of a step of 64 are read during the step before it.  Scales come in pieces of 16 a row, for 512 of the reduction, the same way.
//
// What bounds it.  256 x 256 tiles: the steps, at the clock that the matrix cores' power leaves.  8192^3 of 4 x 4 bits takes 250 to 260 us (4.3 PFLOP/s), of
// 8 x 4 364 (3.0), of 8 x 8 388 (2.8; the library's product of plain fp8 matrices 398): the matrix cores are busy 58, 74 and 69 % of the cycles, and the
// clock falls from 2.4 to 1.8 and 1.95 GHz.  4 x 4 bits, K from 1024 to 8192 in two and in four rounds of tiles, take 9 us once (launch, operands from HBM,
// the last tiles' ends), 4.3 a round and 0.44 a step of 64, 800 to 860 cycles of which the matrix cores need 512: 56 of the 75 us of 8192 x 4096, K 4096 are steps.
// fp32 results of 8-bit operands: bf16 arithmetic, 8192^3 870 us (1.26 PFLOP/s; the library's bf16 product 1.30).  Few tiles: latency of the loads.
//
// LDS holds rows of 64 or 128 bytes as they are in memory, 16-byte chunk c at place c ^ swizzle(row): eight lanes in a row read from
// different banks, and so do sixteen (no conflicts are counted).
template <int CHUNKS>
__device__ __forceinline__ int swizzle(int row) {
    const int b0 = row & 1, b1 = (row >> 1) & 1, b2 = (row >> 2) & 1, b3 = (row >> 3) & 1;
    if constexpr (CHUNKS == 4) return (b1 ^ b3) | (b2 << 1);
    else return (b0 ^ b3) | (b1 << 1) | (b2 << 2);
}

// 16 bytes a lane from base + offset to LDS at `to` + 16 lane; not waited for.  (M0 is a register that the compiler sets itself before each use.)
__device__ __forceinline__ void to_lds(const unsigned char* base, unsigned offset, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void to_lds(const unsigned char* from, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}
// all but the last N of this wavefront's transfers have arrived, its LDS reads are done, and every wavefront has come as far
template <int N>
__device__ __forceinline__ void arrived() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <int FA, int FB, int MI, int NI, int WAVES, int GROUPS, int ROOM>
struct TileShape {
    static constexpr int kThreads = 64 * WAVES, kPiece = 16 * kThreads;
    static constexpr int TM = 64 * MI, TN = 16 * WAVES * NI;
    static constexpr int SUBS = FA == DQ_MXFP4 && FB == DQ_MXFP4 ? 4 : 2;                    // steps of 64 in a stage
    static constexpr int RA = kStepBytes<FA> / 2 * SUBS, RB = kStepBytes<FB> / 2 * SUBS;        // bytes of a row in a stage
    static constexpr int CA = RA / 16, CB = RB / 16;                                         // chunks
    static constexpr int PA = TM * RA / kPiece, kPieces = PA + TN * RB / kPiece;
    static constexpr int kStageBytes = kPieces * kPiece;
    static constexpr int kScaleSets = MI < 4 ? 2 : 1, kScaleBytes = (TM + TN + 63) / 64 * 1024;
    static constexpr int kStages = (ROOM * 1024 / GROUPS - kScaleSets * kScaleBytes) / kStageBytes;
    static constexpr int kLds = kStages * kStageBytes + kScaleSets * kScaleBytes;
    static_assert(kStages >= 2, "two stages have to fit");
    // pieces sent for up to the j-th step behind the barrier: in the first of two steps, in the first two of four
    static constexpr int sent(int j) { return j < 0 ? 0 : SUBS == 4 && j == 0 ? kPieces / 2 : kPieces; }
    // transfers that a wavefront may have under way behind stage i + 1; in front of the first read of new scales, no more than were sent for since
    // those scales, which were sent for behind the first barrier of the 512 before (of the 512 before that, with two sets)
    static constexpr int kBehind = (kStages - 2) * kPieces < 60 ? (kStages - 2) * kPieces : 60;
    static constexpr int kSinceScales = ((kScaleSets - 1) * 8 / SUBS + 8 / SUBS - 1) * kPieces - sent(0);
    static constexpr int kBehindScales = kBehind < kSinceScales ? kBehind : kSinceScales;
};

template <int FA, int FB, class OUT, int MI, int NI, int WAVES, int GROUPS, int ROOM>
__global__ __launch_bounds__(64 * WAVES * GROUPS) void gemm_mx_tile_kernel(GemmMx g, int tiles_m, int tiles_n) {
    using S = TileShape<FA, FB, MI, NI, WAVES, GROUPS, ROOM>;
    constexpr bool EXACT = sizeof(OUT) == 4 && (FA == DQ_MXFP8 || FB == DQ_MXFP8);
    constexpr int NP = S::kPieces, NST = S::kStages, SUBS = S::SUBS, BLOCKS = 2 * SUBS;      // blocks of a row in a stage
    __shared__ __attribute__((aligned(1024))) unsigned char all_smem[S::kLds * GROUPS];
    // GROUPS sets of WAVES wavefronts, each with its own part of LDS and every GROUPS-th piece of 512 of the reduction
    const int group = __builtin_amdgcn_readfirstlane((int)threadIdx.x / S::kThreads);
    const int tid = (int)threadIdx.x % S::kThreads, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 31, q = lane >> 5;
    unsigned char* const smem = all_smem + group * S::kLds;

    // XCD-aware tile order (see gemm_f32.hip): the workgroups resident on an XCD form a block of tiles 8 high
    const int nt = tiles_m * tiles_n;
    const int bid = blockIdx.x;
    const int q8 = nt >> 3, r8 = nt & 7;
    const int xcd = bid & 7;
    const int pid = xcd * q8 + (xcd < r8 ? xcd : r8) + (bid >> 3);
    const int band = 8 * tiles_n;
    const int first_m = pid / band * 8;
    const int gsz = (tiles_m - first_m) < 8 ? (tiles_m - first_m) : 8;
    const int m0 = (first_m + (pid % band) % gsz) * S::TM, n0 = (pid % band) / gsz * S::TN;

    const int nb = (int)((g.K + 31L) / 32), stages = (nb + BLOCKS - 1) / BLOCKS;
    constexpr int PER = 8 / SUBS;                  // stages of 512
    const int pieces = (nb + 15) / 16, local_stages = (pieces + GROUPS - 1) / GROUPS * PER;
    auto whole_piece = [&](int piece) { return GROUPS == 1 ? piece : piece * GROUPS + group; };      // of this group's
    const unsigned smem_at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem);
    constexpr int kScalesAt = NST * S::kStageBytes;

    // this thread's transfers: row and chunk in a tile, as an offset from the tile's first row
    const unsigned char* const baseA = g.A + (long)m0 * g.lda;
    const unsigned char* const baseB = g.B + (long)n0 * g.ldb;
    unsigned offA[S::PA], offB[NP - S::PA];
    int chunkA, chunkB;          // the same for all of a thread's rows, which are 16 or a multiple of it apart
    {
        constexpr int rows = S::kThreads / S::CA;
        const int at = tid / S::CA;
        chunkA = (tid % S::CA) ^ swizzle<S::CA>(at);
#pragma unroll
        for (int p = 0; p < S::PA; ++p) {
            const int row = m0 + p * rows + at < g.M ? p * rows + at : g.M - 1 - m0;
            offA[p] = (unsigned)((long)row * g.lda) + 16u * chunkA;
        }
    }
    {
        constexpr int rows = S::kThreads / S::CB;
        const int at = tid / S::CB;
        chunkB = (tid % S::CB) ^ swizzle<S::CB>(at);
#pragma unroll
        for (int p = 0; p < NP - S::PA; ++p) {
            const int row = n0 + p * rows + at < g.N ? p * rows + at : g.N - 1 - n0;
            offB[p] = (unsigned)((long)row * g.ldb) + 16u * chunkB;
        }
    }
    constexpr int SP = (S::TM + S::TN + S::kThreads - 1) / S::kThreads;
    const unsigned char* scale_row[SP];
#pragma unroll
    for (int p = 0; p < SP; ++p) {
        const int i = p * S::kThreads + tid;
        if (i < S::TM) {
            const int row = m0 + i < g.M ? m0 + i : g.M - 1;
            scale_row[p] = g.As + (long)row * g.ldas;
        } else {
            const int row = n0 + i - S::TM < g.N ? n0 + i - S::TM : g.N - 1;
            scale_row[p] = g.Bs + (long)row * g.ldbs;
        }
    }
    // Piece p of a stage (A's rows, then B's) into the stage's place at `place` in LDS.  In the last stage, which stands in for all behind it too, a chunk of a
    // block that the row does not have is replaced by the row's first one of the stage: its scale counts as 2^-127 in both operands, which makes nothing
    // of any number, and a NaN in it has made the row NaN before.
    const unsigned backA = BLOCKS * (stages - 1) + chunkA / (S::CA / BLOCKS) < nb ? 0u : 16u * chunkA;
    const unsigned backB = BLOCKS * (stages - 1) + chunkB / (S::CB / BLOCKS) < nb ? 0u : 16u * chunkB;
    struct Source { const unsigned char *a, *b; unsigned back_a, back_b; };
    auto source = [&](int local) {
        int t = GROUPS == 1 ? local : whole_piece(local / PER) * PER + local % PER;
        const bool end = t >= stages - 1;
        t = end ? stages - 1 : t;
        return Source{baseA + (long)t * S::RA, baseB + (long)t * S::RB, end ? backA : 0u, end ? backB : 0u};
    };
    auto fetch = [&](const Source& f, int p, int place) {
        const bool a = p < S::PA;
        to_lds(a ? f.a : f.b, a ? offA[a ? p : 0] - f.back_a : offB[a ? 0 : p - S::PA] - f.back_b, smem_at + place + p * S::kPiece + wave * 1024);
    };
    auto fetch_scales = [&](int chunk) {
        const unsigned to = smem_at + kScalesAt + (S::kScaleSets == 1 ? 0 : (chunk & 1) * S::kScaleBytes) + wave * 1024;
        chunk = whole_piece(chunk);
        chunk = 16 * chunk < nb ? chunk : (nb - 1) / 16;
#pragma unroll
        for (int p = 0; p < SP; ++p)
            if ((S::TM + S::TN) % S::kThreads == 0 || p * S::kThreads + wave * 64 < S::TM + S::TN) to_lds(scale_row[p] + 16L * chunk, to + p * S::kPiece);
    };

    const int wm = wave / (WAVES / 2) * 32 * MI, wn = wave % (WAVES / 2) * 32 * NI;
    // where this lane's 16 bytes of a fragment are, from the start of the fragment's rows: chunks by step, in its two halves for 8 bits
    auto lane_at = [&](auto fc, auto cc, int row_bytes, int u, int half) {
        constexpr int F = decltype(fc)::value, C = decltype(cc)::value;
        const int c = F == DQ_MXFP4 ? 2 * u + q : EXACT ? 4 * u + 2 * q + half : 4 * u + 2 * half + q;
        return r * row_bytes + 16 * (c ^ swizzle<C>(r));
    };
    // a step's multiplications go row by row of A's fragments, so that the next step's can be read over each as soon as its row is done
    Codes<FA> fa[MI];
    Codes<FB> fb[2][NI];
    int lanesA[SUBS][2], lanesB[SUBS][2];
#pragma unroll
    for (int u = 0; u < SUBS; ++u)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            lanesA[u][half] = wm * S::RA + lane_at(std::integral_constant<int, FA>{}, std::integral_constant<int, S::CA>{}, S::RA, u, half);
            lanesB[u][half] = S::TM * S::RA + wn * S::RB + lane_at(std::integral_constant<int, FB>{}, std::integral_constant<int, S::CB>{}, S::RB, u, half);
        }
    // fragment k (A's, then B's) of step u of the stage at `place`
    auto read_fragment = [&](int k, int set, int u, int place) {
        const unsigned char* at = smem + place;
        if (k < MI) {
            Codes<FA>& c = fa[k < MI ? k : 0];
            c.a = *reinterpret_cast<const i32x4*>(at + lanesA[u][0] + 32 * k * S::RA);
            if constexpr (FA == DQ_MXFP8) c.b = *reinterpret_cast<const i32x4*>(at + lanesA[u][1] + 32 * k * S::RA);
        } else {
            const int j = k < MI ? 0 : k - MI;
            Codes<FB>& c = fb[set][j];
            c.a = *reinterpret_cast<const i32x4*>(at + lanesB[u][0] + 32 * j * S::RB);
            if constexpr (FB == DQ_MXFP8) c.b = *reinterpret_cast<const i32x4*>(at + lanesB[u][1] + 32 * j * S::RB);
        }
    };

    // Scales of 512 of the reduction.  Rows i and i + 1 of fragments: the lanes of the lower half read 16 bytes of a row of fragment i, those of
    // the upper half of fragment i + 1; bytes of even blocks and of odd ones are put together, and the halves exchanged, so that byte t of
    // word pair sc[i] is, in each lane, the scale of its block in step t.
    constexpr int FR = MI + NI;
    i32x4 raw[(FR + 1) / 2];
    int sc[FR][2];
    unsigned large = 0u;
    auto frag_row = [&](int k) { return k < MI ? wm + 32 * k : S::TM + wn + 32 * (k - MI); };
    auto read_scales = [&](int chunk) {
        const unsigned char* at = smem + kScalesAt + (S::kScaleSets == 1 ? 0 : (chunk & 1) * S::kScaleBytes);
#pragma unroll
        for (int k = 0; k < FR; k += 2) {
            const int row = q == 0 ? frag_row(k) : frag_row(k + 1 < FR ? k + 1 : k);
            raw[k / 2] = *reinterpret_cast<const i32x4*>(at + 16 * (row + r));
        }
    };
    auto place_scales = [&](int chunk) {
        unsigned keep[4];            // what lies behind the row's last scale may be anything
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int have = nb - 16 * whole_piece(chunk) - 4 * w;
            keep[w] = have >= 4 ? ~0u : have <= 0 ? 0u : (1u << (8 * have)) - 1u;
        }
#pragma unroll
        for (int k = 0; k < FR; k += 2) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const unsigned lo = (unsigned)raw[k / 2][2 * w] & keep[2 * w], hi = (unsigned)raw[k / 2][2 * w + 1] & keep[2 * w + 1];
                if constexpr (EXACT) large |= large_scales(lo) | large_scales(hi);
                const unsigned even = __builtin_amdgcn_perm(hi, lo, 0x06040200u), odd = __builtin_amdgcn_perm(hi, lo, 0x07050301u);
                const auto x = __builtin_amdgcn_permlane32_swap(even, odd, false, false);
                sc[k][w] = (int)x[0];
                if (k + 1 < FR) sc[k + 1 < FR ? k + 1 : k][w] = (int)x[1];
            }
        }
    };

    f32x16 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

    // the s-th product of fragments of step T of a piece of 512
    auto multiply = [&](auto tc, int s) {
        constexpr int T = decltype(tc)::value;
        const int i = s / NI, j = (i & 1) ? NI - 1 - s % NI : s % NI;
        const Codes<FA>& a = fa[i];
        const Codes<FB>& b = fb[T & 1][j];
        if constexpr (EXACT) {
            const unsigned ea = ((unsigned)sc[i][T / 4] >> (8 * (T & 3))) & 255u, eb = ((unsigned)sc[MI + j][T / 4] >> (8 * (T & 3))) & 255u;
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values8<FB, 0>(b, eb), values8<FA, 0>(a, ea), acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values8<FB, 1>(b, eb), values8<FA, 1>(a, ea), acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values8<FB, 2>(b, eb), values8<FA, 2>(a, ea), acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values8<FB, 3>(b, eb), values8<FA, 3>(a, ea), acc[i][j], 0, 0, 0);
        } else {
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand<FB>(b), operand<FA>(a), acc[i][j], kMfmaFormat<FB>, kMfmaFormat<FA>,
                                                                        T & 3, sc[MI + j][T / 4], T & 3, sc[i][T / 4]);
        }
    };

    // Step T of the eight of a piece of 512.  Behind the barrier in the last step of a stage its place is filled again (and in the next step, if a stage has
    // four); that step also reads the next stage's first fragments.  No branches: the instructions stay where they are written, each
    // transfer and read behind a multiplication of its own.
    int place = 0, freed = (NST - 1) * S::kStageBytes;
    Source from = source(NST - 1);
    auto step = [&](auto tc, int stage) {
        constexpr int T = decltype(tc)::value, u = T & 1, sub = T % SUBS;
        constexpr bool last = sub == SUBS - 1;
        if constexpr (last) {
            arrived<T == 7 ? S::kBehindScales : S::kBehind>();
            freed = place;
            place = place == (NST - 1) * S::kStageBytes ? 0 : place + S::kStageBytes;
            from = source(stage + NST);
            if constexpr (T == 7) read_scales(stage * SUBS / 8 + 1);
        }
        constexpr int j = last ? 0 : sub + 1, first = S::sent(j - 1), count = S::sent(j) - first;        // transfers of this step
        constexpr int SLOTS = MI * NI;
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            const int i = s / NI;
            multiply(tc, s);
            if (s < NI) read_fragment(MI + s, 1 - u, last ? 0 : sub + 1, place);
            if (s % NI == NI - 1) read_fragment(i, 0, last ? 0 : sub + 1, place);
#pragma unroll
            for (int k = first + count * s / SLOTS; k < first + count * (s + 1) / SLOTS; ++k)
                fetch(from, k, freed);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (T == SUBS - 1) fetch_scales(stage * SUBS / 8 + S::kScaleSets);
        if constexpr (T == 7) place_scales(stage * SUBS / 8 + 1);
    };

#pragma unroll
    for (int c = 0; c < S::kScaleSets; ++c) fetch_scales(c);
#pragma unroll
    for (int t = 0; t < NST; ++t)
#pragma unroll
        for (int p = 0; p < (t + 1 < NST ? NP : S::sent(0)); ++p) fetch(source(t), p, t * S::kStageBytes);
    constexpr int kFirst = (NST - 2) * NP + S::sent(0);
    arrived<(kFirst < 60 ? kFirst : 60)>();
    read_scales(0);
#pragma unroll
    for (int k = 0; k < FR; ++k) read_fragment(k, 0, 0, 0);
    place_scales(0);
    for (int stage = 0; stage < local_stages; stage += PER) {
        step(std::integral_constant<int, 0>{}, stage);
        step(std::integral_constant<int, 1>{}, stage + 1 / SUBS);
        step(std::integral_constant<int, 2>{}, stage + 2 / SUBS);
        step(std::integral_constant<int, 3>{}, stage + 3 / SUBS);
        step(std::integral_constant<int, 4>{}, stage + 4 / SUBS);
        step(std::integral_constant<int, 5>{}, stage + 5 / SUBS);
        step(std::integral_constant<int, 6>{}, stage + 6 / SUBS);
        step(std::integral_constant<int, 7>{}, stage + 7 / SUBS);
    }
    arrived<0>();        // nothing may still be on its way into LDS when the workgroup ends

    if constexpr (EXACT) {
        const bool again = __any(large != 0u);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] *= kLower;
        if (again) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) {
                    const int m = m0 + wm + 32 * i + r, n = n0 + wn + 32 * j + r;
                    const long row_a = m < g.M ? m : g.M - 1, row_b = n < g.N ? n : g.N - 1;
                    const unsigned char *pa = g.A + row_a * g.lda, *pb = g.B + row_b * g.ldb, *sa = g.As + row_a * g.ldas, *sb = g.Bs + row_b * g.ldbs;
                    f32x16 c;
#pragma unroll
                    for (int v = 0; v < 16; ++v) c[v] = 0.f;
                    for (int step = 8 * group; 2 * step < nb; step += step % 8 == 7 ? 8 * GROUPS - 7 : 1) {
                        const int block = 2 * step + q;
                        const int xa = block < nb ? sa[block] : 0, xb = block < nb ? sb[block] : 0;
                        const Codes<FA> a = load_codes64<FA>(pa, step, q, nb);
                        const Codes<FB> b = load_codes64<FB>(pb, step, q, nb);
                        for (int k = 0; k < 8; ++k)
                            c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand<FB>(b), operand<FA>(one_of_eight<FA>(a, k)), c, kMfmaFormat<FB>,
                                                                                kMfmaFormat<FA>, 0, xb, 0, xa);
                    }
                    acc[i][j] = c;
                }
        }
    }

    // the groups' sums, added in order
    if constexpr (GROUPS > 1) {
        static_assert(64 * WAVES * MI * NI * 64 <= S::kLds, "a group's sums have to fit its part of LDS");
        f32x4* const mine = reinterpret_cast<f32x4*>(smem);
        if (group > 0) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        mine[((i * NI + j) * 4 + v) * S::kThreads + tid] = f32x4{acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]};
        }
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int other = 1; other < GROUPS; ++other) {
            const f32x4* const from_group = reinterpret_cast<const f32x4*>(all_smem + other * S::kLds);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const f32x4 x = from_group[((i * NI + j) * 4 + v) * S::kThreads + tid];
#pragma unroll
                        for (int y = 0; y < 4; ++y) acc[i][j][4 * v + y] += x[y];
                    }
        }
    }

    // Register 4 x + y of a lane holds C[m = r][n = 8 x + 4 q + y]; lanes of the two halves exchange groups of four, so that each has eight columns
    // in a row: lower half 16 x .., upper half 16 x + 8 ..  They pass through LDS, 32 rows of a wavefront at a time, and leave as whole rows of its tile.
    // While 32 rows are on their way back from LDS the next 32 are written to it.
    constexpr int CR = 32 * NI * (int)sizeof(OUT), CC = CR / 16, E = 16 / (int)sizeof(OUT);
    static_assert(2 * WAVES * 32 * CR <= S::kLds, "twice 32 rows of every wavefront have to fit");
    const auto chunk_at = [](int row, int c) { return row * CR + 16 * (c ^ swizzle<(CC < 8 ? 4 : 8)>(row)); };
    const auto put_rows = [&](int i) {
        unsigned char* const slab = smem + (2 * wave + (i & 1)) * 32 * CR;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                unsigned w[8];
                constexpr int W = sizeof(OUT) == 4 ? 4 : 2;       // words of four values
                if constexpr (sizeof(OUT) == 4) {
#pragma unroll
                    for (int v = 0; v < 8; ++v) w[v] = __float_as_uint(acc[i][j][8 * x + v]);
                } else {
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const mx_f32x2 pair = {acc[i][j][8 * x + 2 * v], acc[i][j][8 * x + 2 * v + 1]};
                        w[v] = __builtin_bit_cast(unsigned, __builtin_convertvector(pair, mx_bf16x2));
                    }
                }
#pragma unroll
                for (int v = 0; v < W; ++v) {
                    const auto e = __builtin_amdgcn_permlane32_swap(w[v], w[v + W], false, false);
                    w[v] = e[0];
                    w[v + W] = e[1];
                }
                const int c = (32 * j + 16 * x + 8 * q) / E;
                *reinterpret_cast<uint4*>(slab + chunk_at(r, c)) = make_uint4(w[0], w[1], w[2], w[3]);
                if constexpr (sizeof(OUT) == 4) *reinterpret_cast<uint4*>(slab + chunk_at(r, c + 1)) = make_uint4(w[4], w[5], w[6], w[7]);
            }
        }
    };
    OUT* const C = static_cast<OUT*>(g.C);
    const bool inside = m0 + S::TM <= g.M && n0 + S::TN <= g.N;
    const auto send_rows = [&](int i) {
        const unsigned char* const slab = smem + (2 * wave + (i & 1)) * 32 * CR;
        uint4 w[CC / 2];
#pragma unroll
        for (int p = 0; p < CC / 2; ++p) w[p] = *reinterpret_cast<const uint4*>(slab + chunk_at((64 * p + lane) / CC, (64 * p + lane) % CC));
        const int m = m0 + wm + 32 * i + lane / CC, n = n0 + wn + E * (lane % CC);
        OUT* const to = C + (long)m * g.ldc + n;
        if (inside) {
#pragma unroll
            for (int p = 0; p < CC / 2; ++p) *reinterpret_cast<uint4*>(to + (long)(64 / CC * p) * g.ldc) = w[p];
            return;
        }
#pragma unroll
        for (int p = 0; p < CC / 2; ++p) {
            if (m + 64 / CC * p >= g.M || n >= g.N) continue;
            OUT* const at = to + (long)(64 / CC * p) * g.ldc;
            if (n + E <= g.N) {
                *reinterpret_cast<uint4*>(at) = w[p];
            } else {
                const unsigned u[4] = {w[p].x, w[p].y, w[p].z, w[p].w};
#pragma unroll
                for (int v = 0; v < E - 1; ++v)
                    if (n + v < g.N) {
                        if constexpr (sizeof(OUT) == 4) at[v] = __uint_as_float(u[v]);
                        else at[v] = (bf16_t)(v & 1 ? u[v / 2] >> 16 : u[v / 2] & 0xffffu);
                    }
            }
        }
    };
#pragma unroll
    for (int i = 0; i <= MI; ++i) {
        if (i < MI) put_rows(i < MI ? i : 0);
        asm volatile("" ::: "memory");       // lanes read what other lanes of their wavefront wrote
        if (i > 0) send_rows(i - 1);
        asm volatile("" ::: "memory");
    }
}

template <int FA, int FB, class OUT, int MI, int NI, int WAVES, int GROUPS, int ROOM>
hipError_t launch_tile(const GemmMx& g, hipStream_t s) {
    using S = TileShape<FA, FB, MI, NI, WAVES, GROUPS, ROOM>;
    const long tm = (g.M + (long)S::TM - 1) / S::TM, tn = (g.N + (long)S::TN - 1) / S::TN;
    if (tm * tn > 0x7fffffffL) return hipErrorInvalidValue;
    hipLaunchKernelGGL((gemm_mx_tile_kernel<FA, FB, OUT, MI, NI, WAVES, GROUPS, ROOM>), dim3((unsigned)(tm * tn)), dim3(S::kThreads * GROUPS), 0, s, g, (int)tm, (int)tn);
    return hipGetLastError();
}

// Which kernel, by what each takes for C = M x N, K (us of the kernel alone, operands in the caches; 4 x 4 bits and bf16 unless said):
//   straight from memory, 16 rows, against 64 x 32 tiles   1 x 4096, 4096: 4.0, 6.1;  1 x 4096, 16384: 8.2, 11.8;  16 x 4096, 8192 (8 x 8): 11.1, 12.3;
//                                                   16 x 8192, 4096: 6.0, 6.3;  but 16 x 8192, 8192: 9.3, 8.2, and 1 x 8192, 8192 (8 x 8) 15.6, 13.3
//                                                   (one row of 8 x 4 bits against 8192 columns, K 8192, would gain by it: 8.3, 10.2)
//   the same, 32 rows x 16 (256 workgroups at most)   17 x 1000, 2000 (8 x 4): 3.8, 5.7;  300 x 300, 300 (8 x 8, fp32): 3.9, 7.3;  24 x 4096, 4096 (8 x 4): 7.2,
//                                                   7.4;  but 24 x 8192, 2048 (512): 7.9, 6.1, and 64 x 1000, 8192 (8 x 4): 12.5, 9.8
//   the same, 32 rows x 32 (256 workgroups at most)   24 x 8192, 2048 (8 x 4): 5.5, 6.1;  512 x 512, 512 (8 x 8, fp32): 5.0, 7.4;  but 24 x 8192, 4096 (8 x
//                                                   4): 8.7, 8.1, and 1000 x 1000, 256 (1024): 8.4, 5.6
//   64 x 32 tiles, 4 groups against 64 x 64, 2      128 x 4096, 4096: 6.8, 7.4;  256 x 4096, 4096 (512 and 256 workgroups): 12.2, 8.4
//   64 x 64 tiles against 128 x 64, 2 groups        256 x 4096, 4096: 8.4, 9.9;  512 x 4096, 4096 (512 and 256 workgroups): 12.1, 10.8
//   128 x 64 tiles against 128 x 128                512 x 4096, 4096 (256 and 128 workgroups): 10.8, 12.3;  1024 x 4096, 4096: 19.3, 14.4
//   128 x 128 tiles, all of LDS against half          operands not in the L2s: 1024 x 4096, 4096 (256 workgroups): 17.1, 22.1;  2048 x 4096, 4096 (512): 32.5, 29.3
//   128 x 128 tiles against 256 x 256               2048 x 4096, 4096 (512 and 128 workgroups): 25.0, 29.0
// that is, the largest tile that still gives most compute units a workgroup, by results of up to 8192 columns.  Tiles are counted, whatever part of their rows
// exists: 24 x 14336, 4096 (8 x 4) takes 11.5 us in tiles of 128 x 64, 24 x 28672, 8192 27.6 in 128 x 128 and 1 x 128256, 8192 167 in 256 x 256, where B at the
// rate of a large copy takes 6, 24 and 105.  (256 x 128 tiles in between: 24.3 for the last, but 39.7 against 37.6 for
// 2560 x 4096, and 46.6 against 40.8 for 4096 x 4096, 1024 in bf16 arithmetic.)  A kernel of no work takes 2 us, one of 64 in the reduction 4 to 5.
template <int FA, int FB, class OUT>
hipError_t launch_types(const GemmMx& g, hipStream_t s) {
    constexpr bool exact = sizeof(OUT) == 4 && (FA == DQ_MXFP8 || FB == DQ_MXFP8);
    const bool near_rows = g.lda < (1L << 23) && g.ldb < (1L << 23);       // the tiles address their rows by 32-bit offsets
    const auto tiles = [&](long tm, long tn) { return ((g.M + tm - 1) / tm) * ((g.N + tn - 1) / tn); };
    if (!near_rows || (g.M <= 16 && (g.K <= 4096 || tiles(16, 16) <= 256))) {
        // 32 columns a workgroup as soon as that gives every compute unit one: 16 x 8192, K 4096 6.4 -> 5.6 us, 8 x 8 bits 10.3 -> 8.6 (one row 4.8 and 4.9, 7.4 and
        // 7.2; but one row against 14336 columns, 8 x 8 bits, 13.7 -> 14.6)
        return g.N >= 32 * 256 ? launch_direct<FA, FB, OUT, 1, 2>(g, s) : launch_direct<FA, FB, OUT, 1, 1>(g, s);
    }
    if (g.K <= 4096 && tiles(32, 16) <= 256) return launch_direct<FA, FB, OUT, 2, 1>(g, s);
    if (g.K <= 2560 && tiles(32, 32) <= 256) return launch_direct<FA, FB, OUT, 2, 2>(g, s);
    constexpr long most = 192;
    if (!exact && tiles(256, 256) >= most) {
        // Eight wavefronts to a tile for 4 x 4 bits (8192^3, when it was chosen: 324 us with four, 299), four for the others, whose fragments do not leave registers
        // for two wavefronts a SIMD (8 x 8 bits: 429 us, 476 with eight).
        if constexpr (FA == DQ_MXFP4 && FB == DQ_MXFP4) return launch_tile<FA, FB, OUT, 4, 2, 8, 1, 160>(g, s);
        else if constexpr (!exact) return launch_tile<FA, FB, OUT, 4, 4, 4, 1, 160>(g, s);
    }
    if (tiles(128, 128) > 256) return launch_tile<FA, FB, OUT, 2, 2, 4, 1, 80>(g, s);         // two workgroups a compute unit
    if (tiles(128, 128) >= most) return launch_tile<FA, FB, OUT, 2, 2, 4, 1, 160>(g, s);
    if (tiles(128, 64) >= most) return launch_tile<FA, FB, OUT, 2, 1, 4, 2, 160>(g, s);
    if (tiles(64, 64) >= most) return launch_tile<FA, FB, OUT, 1, 1, 4, 2, 80>(g, s);
    return launch_tile<FA, FB, OUT, 1, 1, 2, 4, 160>(g, s);
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
