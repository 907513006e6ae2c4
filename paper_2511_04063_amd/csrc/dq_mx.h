// Microscaled (MX) blocks: 32 consecutive values of a row share a scale 2^E, E + 127 in a byte; a value is a 4-bit float (e2m1: 0, 0.5, 1,
// 1.5, 2, 3, 4, 6) or an 8-bit one (e4m3, largest 448).  Device code shared by the quantiser, the norm, the objective and the product.
#pragma once

#include <type_traits>

#include "dq_internal.h"
#include "dq_wave.h"

namespace dq {
namespace {

typedef float mx_f32x2 __attribute__((ext_vector_type(2)));
typedef short mx_i16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));

constexpr unsigned kMxInf = 0x7f800000u;     // |v| as an integer from here on: an infinity or a NaN

// E + 127 of a block from the bits of its largest magnitude: floor(log2 a) is the exponent field of a, E = max(floor(log2 a) - emax, -127)
// with emax the exponent of the largest representable value (6 = 1.5 2^2, 448 = 1.75 2^8); below the normal numbers E is -127 anyway.
// 255 stands for a NaN.
template <int F>
__device__ __forceinline__ unsigned mx_scale_byte(unsigned top) {
    constexpr int emax = F == DQ_MXFP4 ? 2 : 8;
    const int e = (int)(top >> 23) - emax;
    return top >= kMxInf ? 255u : (unsigned)(e > 0 ? e : 0);
}
// 2^E as a float (2^-127 is subnormal; the conversions take it)
__device__ __forceinline__ float mx_scale(unsigned byte) { return __uint_as_float(byte == 0u ? 0x00400000u : byte << 23); }

// largest of the LANES lanes that hold a block (4 or 8 neighbours, aligned)
template <int LANES>
__device__ __forceinline__ unsigned mx_group_max(unsigned v) {
    const auto other = [](unsigned x, auto off) { return __float_as_uint(lane_xor<decltype(off)::value>(__uint_as_float(x))); };
    unsigned o = other(v, std::integral_constant<int, 1>{});
    v = v > o ? v : o;
    o = other(v, std::integral_constant<int, 2>{});
    v = v > o ? v : o;
    if constexpr (LANES == 8) {
        o = other(v, std::integral_constant<int, 4>{});
        v = v > o ? v : o;
    }
    return v;
}

// Codes of NV fp32 values (NV = 4 or 8) of a block with that scale byte, in value order from the lowest bits: NV / 8 words of 4-bit codes
// (half a word for NV = 4) or NV / 4 words of 8-bit ones.  The conversions divide by the scale, round to nearest even and, to 4 bits,
// saturate; to 8 bits they give a NaN from 464 scales on, so the values are clamped to 448 scales first.
template <int F, int NV>
__device__ __forceinline__ void mx_encode(const float (&v)[NV], unsigned byte, unsigned (&out)[F == DQ_MXFP4 ? (NV + 7) / 8 : NV / 4]) {
    const bool bad = byte == 255u;
    const float s = mx_scale(byte);
    if constexpr (F == DQ_MXFP4) {
        unsigned w = 0u;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
        if constexpr (NV == 8) {
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
        }
        out[0] = bad ? 0u : w;
    } else {
        const float lim = bad ? 0.f : __uint_as_float(((byte + 8u) << 23) | 0x600000u);      // 448 scales
#pragma unroll
        for (int i = 0; i < NV / 4; ++i) {
            mx_i16x2 q = {0, 0};
            q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, __builtin_amdgcn_fmed3f(v[4 * i], -lim, lim),
                                                         __builtin_amdgcn_fmed3f(v[4 * i + 1], -lim, lim), s, false);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, __builtin_amdgcn_fmed3f(v[4 * i + 2], -lim, lim),
                                                         __builtin_amdgcn_fmed3f(v[4 * i + 3], -lim, lim), s, true);
            out[i] = bad ? 0u : __builtin_bit_cast(unsigned, q);
        }
    }
}

// The four values that codes [4 q, 4 q + 4) of `w` (one word of 8-bit codes; for 4-bit ones q selects the half) stand for.
template <int F, int Q>
__device__ __forceinline__ void mx_decode4(unsigned w, float s, float (&v)[4]) {
    mx_f32x2 a, b;
    if constexpr (F == DQ_MXFP4) {
        a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2 * Q);
        b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2 * Q + 1);
    } else {
        a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, false);
        b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, true);
    }
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}

}  // namespace
}  // namespace dq
