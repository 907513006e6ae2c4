// Quantisation to MX blocks and back, the RMS norm with the residual's addition that ends in MX blocks, and the objective that measures the
// MX quantiser's error with its gradient.  All are passes over token rows bound by HBM: a thread moves 16 bytes of input at a time (4 fp32
// or 8 bf16 values), the 8 or 4 lanes that share a block exchange its largest magnitude by DPP, and the codes leave from the same registers.
#include "dq_mx.h"

namespace dq {
namespace {

template <class T> struct Piece;                       // what one 16-byte access holds
template <> struct Piece<float> { static constexpr int V = 4; };
template <> struct Piece<bf16_t> { static constexpr int V = 8; };

__device__ __forceinline__ float bf16_value(unsigned bits) { return __uint_as_float(bits << 16); }
__device__ __forceinline__ unsigned bf16_pair(float a, float b) {
    const mx_f32x2 v = {a, b};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(v, mx_bf16x2));
}

// The piece of a row at src with `left` columns to the row's end (possibly none); columns behind it read as zeros.  Nothing behind the
// row's end is touched.
__device__ __forceinline__ void load_piece(const float* src, int left, float (&v)[4]) {
    if (left >= 4) {
        const float4 q = *reinterpret_cast<const float4*>(src);
        v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < left ? src[i] : 0.f;
    }
}
__device__ __forceinline__ void load_piece(const bf16_t* src, int left, float (&v)[8]) {
    if (left >= 8) {
        const uint4 q = *reinterpret_cast<const uint4*>(src);
        const unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = bf16_value(w[i] & 0xffffu);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? bf16_value(src[i]) : 0.f;
    }
}
__device__ __forceinline__ void store_piece(float* dst, int left, const float (&v)[4]) {
    if (left >= 4) {
        *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) dst[i] = v[i];
    }
}
template <int NV>
__device__ __forceinline__ void store_piece(bf16_t* dst, int left, const float (&v)[NV]) {
    unsigned w[NV / 2];
#pragma unroll
    for (int i = 0; i < NV / 2; ++i) w[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
    if (left >= NV) {
        if constexpr (NV == 8) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < left) dst[i] = (bf16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu);
    }
}

template <int NV>
__device__ __forceinline__ unsigned piece_top(const float (&v)[NV]) {
    unsigned top = 0u;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const unsigned u = __float_as_uint(v[i]) & 0x7fffffffu;
        top = top > u ? top : u;
    }
    return top;
}

// Codes of piece `unit` of a row (V values each) and, from the first lane of a block, its scale; the row's last block also fills the scales
// up to a multiple of 16.
template <int F, int NV>
__device__ __forceinline__ void put_blocks(const float (&v)[NV], int unit, int nb, unsigned char* codes, unsigned char* scales, unsigned* flags) {
    constexpr int LANES = 32 / NV;
    const unsigned byte = mx_scale_byte<F>(mx_group_max<LANES>(piece_top(v)));
    unsigned w[F == DQ_MXFP4 ? (NV + 7) / 8 : NV / 4];
    mx_encode<F, NV>(v, byte, w);
    if constexpr (F == DQ_MXFP4) {
        if constexpr (NV == 8) reinterpret_cast<unsigned*>(codes)[unit] = w[0];
        else reinterpret_cast<unsigned short*>(codes)[unit] = (unsigned short)w[0];
    } else {
        if constexpr (NV == 8) reinterpret_cast<uint2*>(codes)[unit] = make_uint2(w[0], w[1]);
        else reinterpret_cast<unsigned*>(codes)[unit] = w[0];
    }
    if (unit % LANES == 0) {
        const int block = unit / LANES;
        scales[block] = (unsigned char)byte;
        if (block == nb - 1)
            for (int i = nb; i & 15; ++i) scales[i] = 0;
        if (byte == 255u) atomicOr(flags, DQ_FLAG_NONFINITE);
    }
}

// Threads over rows of `upr` pieces: `rg` whole rows side by side in a workgroup where they are short (rg * upr <= 256), else tiles of 256
// pieces along a row (blockIdx.x); rows are walked in steps of rg * gridDim.y, so that a thread stays at its column.
struct Walk { int upr, rg; };
__device__ __forceinline__ bool walk_start(const Walk& w, int& row, int& unit) {
    if (w.rg > 1) {
        const int r = (int)threadIdx.x / w.upr;
        unit = (int)threadIdx.x - r * w.upr;
        row = (int)blockIdx.y * w.rg + r;
        return r < w.rg;
    }
    unit = (int)(blockIdx.x * 256 + threadIdx.x);
    row = (int)blockIdx.y;
    return unit < w.upr;
}

template <class IN, int F>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const IN* __restrict__ X, long ldx, int T, int n, int nb, unsigned char* __restrict__ codes,
                                                          long ldc, unsigned char* __restrict__ scales, long lds, Walk w, unsigned* flags) {
    constexpr int V = Piece<IN>::V;
    int row, unit;
    if (!walk_start(w, row, unit)) return;
    const int step = w.rg * (int)gridDim.y, left = n - unit * V;
    for (long r = row; r < T; r += step) {
        float v[V];
        load_piece(X + r * ldx + (long)unit * V, left, v);
        put_blocks<F, V>(v, unit, nb, codes + r * ldc, scales + r * lds, flags);
    }
}

template <class OUT, int F>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const unsigned char* __restrict__ codes, long ldc, const unsigned char* __restrict__ scales,
                                                            long lds, int T, int n, OUT* __restrict__ Y, long ldy, Walk w) {
    constexpr int V = Piece<OUT>::V, LANES = 32 / V;
    int row, unit;
    if (!walk_start(w, row, unit)) return;
    const int step = w.rg * (int)gridDim.y, left = n - unit * V;
    if (left <= 0) return;
    for (long r = row; r < T; r += step) {
        const unsigned char* src = codes + r * ldc;
        const unsigned byte = scales[r * lds + unit / LANES];
        const float s = mx_scale(byte);
        float v[V];
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            float t[4];
            if constexpr (F == DQ_MXFP4) {
                const unsigned word = V == 8 ? reinterpret_cast<const unsigned*>(src)[unit]
                                             : (unsigned)reinterpret_cast<const unsigned short*>(src)[unit];
                if (q == 0) mx_decode4<F, 0>(word, s, t); else mx_decode4<F, 1>(word, s, t);
            } else {
                mx_decode4<F, 0>(reinterpret_cast<const unsigned*>(src)[unit * (V / 4) + q], s, t);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * q + i] = byte == 255u ? __uint_as_float(0x7fc00000u) : t[i];
        }
        store_piece(Y + r * ldy + (long)unit * V, left, v);
    }
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
    return v;
}

// 1 / sqrt(m) to 64 bits from the machine's estimate by two Newton steps; a row of zeros without an epsilon gives zeros
__device__ __forceinline__ double inverse_root(double m) {
    if (!(m > 0.0)) return m == 0.0 ? 0.0 : __builtin_nan("");
    if (m == __builtin_inf()) return 0.0;
    double r = __builtin_amdgcn_rsq(m);
    r = r * (1.5 - 0.5 * m * r * r);
    return r * (1.5 - 0.5 * m * r * r);
}

// One token row per TPR threads, P pieces each:  h = x + res (rounded to the stored type: the norm is that of what is stored),
// y = fp32(h / sqrt(mean h^2 + eps) * gain), then MX blocks of y.  The mean and y are formed in 64 bits and rounded once: a difference in
// the last bit of y flips codes next to a border, and a row's sum in 32 bits moves every value of the row.  H may be X or res.
template <class IN, int F, int P, int TPR>
__global__ __launch_bounds__(256) void mx_rms_norm_kernel(const IN* X, long ldx, const IN* res, long ldr, IN* H, long ldh, const float* __restrict__ gain,
                                                          float eps, int T, int n, int nb, unsigned char* __restrict__ codes, long ldc,
                                                          unsigned char* __restrict__ scales, long lds, unsigned* flags) {
    constexpr int V = Piece<IN>::V, ROWS = 256 / TPR;
    __shared__ double part[4];
    const int t = (int)threadIdx.x % TPR;
    const long row = (long)blockIdx.x * ROWS + (int)threadIdx.x / TPR;
    const bool live = row < T;
    float h[P][V];
    double ss = 0.0;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int c = (p * TPR + t) * V, left = live ? n - c : 0;
        if (left > 0) {
            load_piece(X + row * ldx + c, left, h[p]);
            if (res != nullptr) {
                float r[V];
                load_piece(res + row * ldr + c, left, r);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    h[p][i] += r[i];
                    if constexpr (V == 8) h[p][i] = (float)(__bf16)h[p][i];
                }
            }
            if (H != nullptr) store_piece(H + row * ldh + c, left, h[p]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) h[p][i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) ss += (double)h[p][i] * (double)h[p][i];
    }
    ss = wave_sum(ss);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = ss;
        __syncthreads();
        ss = (part[0] + part[1]) + (part[2] + part[3]);
    }
    if (!live) return;
    const double f = inverse_root(ss / (double)n + (double)eps);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int unit = p * TPR + t, c = unit * V;
        if (c >= nb * 32) continue;                       // lanes of a block go together
        float y[V];
        if (gain != nullptr) {
            float g[V];
            if constexpr (V == 4) {
                load_piece(gain + c, n - c, g);
            } else {
                float g0[4], g1[4];
                load_piece(gain + c, n - c, g0);
                load_piece(gain + c + 4, n - c - 4, g1);
#pragma unroll
                for (int i = 0; i < 4; ++i) { g[i] = g0[i]; g[4 + i] = g1[i]; }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = (float)((double)h[p][i] * f * (double)g[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = (float)((double)h[p][i] * f);
        }
        put_blocks<F, V>(y, unit, nb, codes + row * ldc, scales + row * lds, flags);
    }
}

// Squared error of the MX quantiser and its derivative:  loss_t = (1/n) sum_i (y_i - yhat_i)^2,  dY_i = c (2/n) (y_i - yhat_i).  yhat is
// constant around almost every y (the scale is a power of two), so this is the derivative wherever there is one.
template <int F, bool BF16OUT>
__global__ __launch_bounds__(256) void mx_objective_kernel(const float* __restrict__ Y, long ldy, int T, int n, float scale, void* __restrict__ dYv,
                                                           long lddy, double* __restrict__ partials, long sy, long sdy, Walk w) {
    __shared__ double tot[4];
    Y += (long)blockIdx.y * sy;
    const float f = scale * 2.f / (float)n;
    const int xt = w.rg > 1 ? 1 : (w.upr + 255) / 256;
    const long groups = ((long)T + w.rg - 1) / w.rg;
    double acc = 0.0;
    for (long item = blockIdx.x; item < groups * xt; item += gridDim.x) {
        const long group = item / xt;
        const int r_in = w.rg > 1 ? (int)threadIdx.x / w.upr : 0;
        const int unit = w.rg > 1 ? (int)threadIdx.x - r_in * w.upr : (int)(item - group * xt) * 256 + (int)threadIdx.x;
        const long row = group * w.rg + r_in;
        const int left = n - unit * 4;
        if (r_in >= w.rg || unit >= w.upr || row >= T) continue;
        float v[4];
        load_piece(Y + row * ldy + (long)unit * 4, left, v);
        const unsigned byte = mx_scale_byte<F>(mx_group_max<8>(piece_top(v)));
        unsigned code[1];
        mx_encode<F, 4>(v, byte, code);
        float e[4];
        mx_decode4<F, 0>(code[0], mx_scale(byte), e);
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e[i] = byte == 255u ? __uint_as_float(0x7fc00000u) : v[i] - e[i];
            ss += e[i] * e[i];
            e[i] *= f;
        }
        acc += (double)ss;
        if (dYv != nullptr && left > 0) {
            if constexpr (BF16OUT) store_piece<4>(static_cast<bf16_t*>(dYv) + (long)blockIdx.y * sdy + row * lddy + (long)unit * 4, left, e);
            else store_piece(static_cast<float*>(dYv) + (long)blockIdx.y * sdy + row * lddy + (long)unit * 4, left, e);
        }
    }
    acc = wave_sum(acc);
    if ((threadIdx.x & 63) == 0) tot[threadIdx.x >> 6] = acc;
    __syncthreads();
    if (threadIdx.x == 0) partials[(long)blockIdx.y * gridDim.x + blockIdx.x] = ((tot[0] + tot[1]) + (tot[2] + tot[3])) / (double)n;
}

Walk make_walk(int n, int V) {
    Walk w;
    w.upr = (int)((n + 31L) / 32) * (32 / V);
    w.rg = w.upr <= 128 ? 256 / w.upr : 1;
    return w;
}
dim3 walk_grid(const Walk& w, int T) {
    const long groups = ((long)T + w.rg - 1) / w.rg;
    const long xt = w.rg > 1 ? 1 : (w.upr + 255) / 256;
    long gy = 16384 / xt;
    gy = gy < 1 ? 1 : gy < groups ? gy : groups;
    return dim3((unsigned)xt, (unsigned)gy);
}

template <class IN, int F, int P, int TPR>
hipError_t norm_launch(const MxNorm& m, hipStream_t s) {
    constexpr int rows = 256 / TPR;
    hipLaunchKernelGGL((mx_rms_norm_kernel<IN, F, P, TPR>), dim3((unsigned)(((long)m.T + rows - 1) / rows)), dim3(256), 0, s,
                       static_cast<const IN*>(m.X), m.ldx, static_cast<const IN*>(m.res), m.ldr, static_cast<IN*>(m.H), m.ldh, m.gain, m.eps, m.T,
                       m.n, (m.n + 31) / 32, m.codes, m.ldc, m.scales, m.lds, m.flags);
    return hipGetLastError();
}
template <class IN, int F>
hipError_t norm_shape(const MxNorm& m, hipStream_t s) {
    if constexpr (Piece<IN>::V == 8) {
        if (m.n <= 512) return norm_launch<IN, F, 1, 64>(m, s);
        if (m.n <= 1024) return norm_launch<IN, F, 2, 64>(m, s);
        if (m.n <= 2048) return norm_launch<IN, F, 1, 256>(m, s);
        if (m.n <= 4096) return norm_launch<IN, F, 2, 256>(m, s);
        if (m.n <= 8192) return norm_launch<IN, F, 4, 256>(m, s);
    } else {
        if (m.n <= 512) return norm_launch<IN, F, 2, 64>(m, s);
        if (m.n <= 1024) return norm_launch<IN, F, 4, 64>(m, s);
        if (m.n <= 2048) return norm_launch<IN, F, 2, 256>(m, s);
        if (m.n <= 4096) return norm_launch<IN, F, 4, 256>(m, s);
        if (m.n <= 8192) return norm_launch<IN, F, 8, 256>(m, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_mx_quantize(const void* X, int x_is_bf16, long ldx, int T, int n, int format, unsigned char* codes, long ldc, unsigned char* scales,
                              long lds, unsigned* flags, hipStream_t s) {
    if (T < 1 || n < 1) return hipSuccess;
    const Walk w = make_walk(n, x_is_bf16 ? 8 : 4);
    const int nb = (int)((n + 31L) / 32);
#define DQ_GO(IN, F)                                                                                                                              \
    hipLaunchKernelGGL((mx_quantize_kernel<IN, F>), walk_grid(w, T), dim3(256), 0, s, static_cast<const IN*>(X), ldx, T, n, nb, codes, ldc, scales, \
                       lds, w, flags)
    if (x_is_bf16) { if (format == DQ_MXFP4) DQ_GO(bf16_t, DQ_MXFP4); else DQ_GO(bf16_t, DQ_MXFP8); }
    else { if (format == DQ_MXFP4) DQ_GO(float, DQ_MXFP4); else DQ_GO(float, DQ_MXFP8); }
#undef DQ_GO
    return hipGetLastError();
}

hipError_t launch_mx_dequantize(int format, const unsigned char* codes, long ldc, const unsigned char* scales, long lds, int T, int n, void* Y,
                                int y_is_bf16, long ldy, hipStream_t s) {
    if (T < 1 || n < 1) return hipSuccess;
    const Walk w = make_walk(n, y_is_bf16 ? 8 : 4);
#define DQ_GO(OUT, F)                                                                                                                        \
    hipLaunchKernelGGL((mx_dequantize_kernel<OUT, F>), walk_grid(w, T), dim3(256), 0, s, codes, ldc, scales, lds, T, n, static_cast<OUT*>(Y), \
                       ldy, w)
    if (y_is_bf16) { if (format == DQ_MXFP4) DQ_GO(bf16_t, DQ_MXFP4); else DQ_GO(bf16_t, DQ_MXFP8); }
    else { if (format == DQ_MXFP4) DQ_GO(float, DQ_MXFP4); else DQ_GO(float, DQ_MXFP8); }
#undef DQ_GO
    return hipGetLastError();
}

hipError_t launch_mx_rms_norm(const MxNorm& m, hipStream_t s) {
    if (m.T < 1) return hipSuccess;
    if (m.x_is_bf16) return m.format == DQ_MXFP4 ? norm_shape<bf16_t, DQ_MXFP4>(m, s) : norm_shape<bf16_t, DQ_MXFP8>(m, s);
    return m.format == DQ_MXFP4 ? norm_shape<float, DQ_MXFP4>(m, s) : norm_shape<float, DQ_MXFP8>(m, s);
}

hipError_t launch_mx_objective(int format, const float* Y, long ldy, int T, int n, float scale, void* dY, int dy_is_bf16, long lddy, double* partials,
                               int grid, hipStream_t s, int batch, long stride_y, long stride_dy) {
    if (batch < 1 || T < 1) return hipSuccess;
    const Walk w = make_walk(n, 4);
#define DQ_GO(F, BF) \
    hipLaunchKernelGGL((mx_objective_kernel<F, BF>), dim3(grid, batch), dim3(256), 0, s, Y, ldy, T, n, scale, dY, lddy, partials, stride_y, stride_dy, w)
    if (format == DQ_MXFP4) { if (dy_is_bf16) DQ_GO(DQ_MXFP4, true); else DQ_GO(DQ_MXFP4, false); }
    else { if (dy_is_bf16) DQ_GO(DQ_MXFP8, true); else DQ_GO(DQ_MXFP8, false); }
#undef DQ_GO
    return hipGetLastError();
}

}  // namespace dq
