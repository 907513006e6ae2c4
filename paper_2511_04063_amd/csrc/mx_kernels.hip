// Quantisation to MX blocks and back, the RMS norm with the residual's addition that ends in MX blocks, and the objective that measures the
// MX quantiser's error with its gradient.  All are passes over token rows bound by HBM: a thread moves 16 bytes of input at a time (4 fp32
// or 8 bf16 values), the 8 or 4 lanes that share a block exchange its largest magnitude by DPP, and the codes leave from the same registers.
#include "dq_mx.h"

namespace dq {
namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

template <class T> struct Piece;                       // what one 16-byte access holds, and the access at any element
template <> struct Piece<float> { static constexpr int V = 4; typedef u32x4 Anywhere __attribute__((aligned(4))); };
template <> struct Piece<bf16_t> { static constexpr int V = 8; typedef u32x4 Anywhere __attribute__((aligned(2))); };

__device__ __forceinline__ unsigned bf16_pair(float a, float b) {
    const mx_f32x2 v = {a, b};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(v, mx_bf16x2));
}

// What a 16-byte access brings: raw until all of a thread's are under way.
__device__ __forceinline__ void unpack(const uint4& q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
}
__device__ __forceinline__ void unpack(const uint4& q, float (&v)[8]) {
    const unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
// The piece of V values at column c of a row of n; what lies behind the row's end reads as zero and is not touched.  In place of a piece that is not
// whole the row's last V values are read, and shifted to their place afterwards (the norm of 8192 x 1100 in bf16: 20.6 us with such values read one by one,
// 17.1).  TINY: rows shorter than a piece, value by value.
// STREAM: past the caches, for what is read once by a kernel that writes less than it reads (quantiser 8192 x 8192 42 -> 34 us, objective 8192 x 4096
// 39 -> 35; the norm, which writes as much, 50 -> 52).
template <bool STREAM, bool TINY, class T>
__device__ __forceinline__ uint4 load_whole(const T* row, int c, int n) {
    if constexpr (TINY) return make_uint4(0u, 0u, 0u, 0u);
    const typename Piece<T>::Anywhere* at = reinterpret_cast<const typename Piece<T>::Anywhere*>(row + (c + Piece<T>::V <= n ? c : n - Piece<T>::V));
    const u32x4 q = STREAM ? __builtin_nontemporal_load(at) : *at;
    return make_uint4(q.x, q.y, q.z, q.w);
}
template <bool TINY, class T>
__device__ __forceinline__ void finish_piece(uint4& q, const T* row, int c, int n) {
    constexpr int V = Piece<T>::V, BITS = 128 / V;
    const int over = c + V - n;        // values behind the end
    if constexpr (TINY) {
        unsigned w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (c + i < n) {
                if constexpr (V == 4) w[i] = __float_as_uint(row[c + i]);
                else w[i / 2] |= (unsigned)row[c + i] << (16 * (i & 1));
            }
        q = make_uint4(w[0], w[1], w[2], w[3]);
    } else if (over > 0) {
        const int by = BITS * over;
        const unsigned long long lo = (unsigned long long)q.y << 32 | q.x, hi = (unsigned long long)q.w << 32 | q.z;
        const unsigned long long low = by < 64 ? lo >> by | hi << (64 - by) : by < 128 ? hi >> (by - 64) : 0ull, high = by < 64 ? hi >> by : 0ull;
        q = make_uint4((unsigned)low, (unsigned)(low >> 32), (unsigned)high, (unsigned)(high >> 32));
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

// Threads over all pieces of all rows, `upr` a row: a workgroup takes `run` times 256 neighbouring ones, then as many 256 `run` times the grid further
// on (objective 8192 x 4096, bf16 gradient: 40.7 us with 256 at a time, 34.1).  A step of a thread is so many rows and pieces.
struct Step { unsigned rows; int units; };
struct Walk { int upr, run; Step near, far; };
struct Place { unsigned row; int unit; };
__device__ __forceinline__ Place walk_start(const Walk& w) {
    const unsigned item = blockIdx.x * (256u * w.run) + threadIdx.x, row = item / (unsigned)w.upr;
    return Place{row, (int)(item - row * (unsigned)w.upr)};
}
__device__ __forceinline__ Place walk_next(const Walk& w, const Place& at, const Step& s) {
    const int unit = at.unit + s.units;
    return unit < w.upr ? Place{at.row + s.rows, unit} : Place{at.row + s.rows + 1, unit - w.upr};
}

// Bound by HBM; U pieces of a thread under way at a time, or their latency shows (8192 x 8192 bf16 to 4 bits, 170 MB, 30.5 us: 5.6 TB/s, a
// large copy reaches 5.3; 333 x 2890, 5 MB: 3.5 us, 2 of them a kernel's own).
template <class IN, int F, bool TINY>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const IN* __restrict__ X, long ldx, int T, int n, int nb, unsigned char* __restrict__ codes,
                                                          long ldc, unsigned char* __restrict__ scales, long lds, Walk w, unsigned* flags) {
    constexpr int V = Piece<IN>::V, U = 4;
    Place at = walk_start(w);
    while (at.row < (unsigned)T) {
        uint4 q[U];
        Place p[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            p[k] = at;
            const bool in = at.row < (unsigned)T;
            q[k] = load_whole<true, TINY>(X + (long)(in ? at.row : 0u) * ldx, in ? at.unit * V : 0, n);
            at = walk_next(w, at, k < U - 1 ? w.near : w.far);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (p[k].row >= (unsigned)T) break;
            finish_piece<TINY>(q[k], X + (long)p[k].row * ldx, p[k].unit * V, n);
            float v[V];
            unpack(q[k], v);
            put_blocks<F, V>(v, p[k].unit, nb, codes + (long)p[k].row * ldc, scales + (long)p[k].row * lds, flags);
        }
    }
}

// Bound by the writes: 8192 x 8192 from 4 bits to bf16, 35 MB read and 134 MB written, in 25.7 us (6.6 TB/s; a fill reaches 6.9).  Stores past the
// caches were slower (34 us).
template <class OUT, int F>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const unsigned char* __restrict__ codes, long ldc, const unsigned char* __restrict__ scales,
                                                            long lds, int T, int n, OUT* __restrict__ Y, long ldy, Walk w) {
    constexpr int V = Piece<OUT>::V, LANES = 32 / V;
    for (Place at = walk_start(w); at.row < (unsigned)T; at = walk_next(w, at, w.far)) {
        const int left = n - at.unit * V;
        if (left <= 0) continue;
        const unsigned char* src = codes + (long)at.row * ldc;
        const float s = mx_scale(scales[(long)at.row * lds + at.unit / LANES]);      // of 255 an infinity, which makes the conversions' results NaN
        float v[V];
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            float t[4];
            if constexpr (F == DQ_MXFP4) {
                const unsigned word = V == 8 ? reinterpret_cast<const unsigned*>(src)[at.unit]
                                             : (unsigned)reinterpret_cast<const unsigned short*>(src)[at.unit];
                if (q == 0) mx_decode4<F, 0>(word, s, t); else mx_decode4<F, 1>(word, s, t);
            } else {
                mx_decode4<F, 0>(reinterpret_cast<const unsigned*>(src)[at.unit * (V / 4) + q], s, t);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * q + i] = t[i];
        }
        store_piece(Y + (long)at.row * ldy + (long)at.unit * V, left, v);
    }
}

template <int OFF>
__device__ __forceinline__ double lane_xor_double(double v) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = __float_as_uint(lane_xor<OFF>(__uint_as_float((unsigned)u))), hi = __float_as_uint(lane_xor<OFF>(__uint_as_float((unsigned)(u >> 32))));
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double v) {
    v += lane_xor_double<1>(v); v += lane_xor_double<2>(v); v += lane_xor_double<8>(v);
    v += lane_xor_double<4>(v); v += lane_xor_double<16>(v); v += lane_xor_double<32>(v);
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

template <bool PAST, class T>
__device__ __forceinline__ void store_sum(T* to, const uint4& q) {
    const u32x4 w = {q.x, q.y, q.z, q.w};
    if constexpr (PAST) __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(to));
    else *reinterpret_cast<u32x4*>(to) = w;
}

// One token row per TPR threads, P pieces each:  h = x + res (rounded to the stored type: the norm is that of what is stored),
// y = fp32(h / sqrt(mean h^2 + eps) * gain), then MX blocks of y.  The mean and y are formed in 64 bits and rounded once: a difference in
// the last bit of y flips codes next to a border, and a row's sum in 32 bits moves every value of the row.  H may be X or res.
// A row is read once and stays in registers, all of its loads under way together.  Bound by HBM: 8192 x 4096 bf16 with the residual to
// 8 bits, 235 MB, 36.5 us in a row (6.4 TB/s) and 45 where what reads the codes runs between (5.2); one token of 4096 2.6 us, a kernel of no
// work takes 2.
template <class IN, int F, int P, int TPR, bool PAST, bool TINY>
__global__ __launch_bounds__(256) void mx_rms_norm_kernel(const IN* X, long ldx, const IN* res, long ldr, IN* H, long ldh, const float* __restrict__ gain,
                                                          float eps, int T, int n, int nb, unsigned char* __restrict__ codes, long ldc,
                                                          unsigned char* __restrict__ scales, long lds, unsigned* flags) {
    constexpr int V = Piece<IN>::V, ROWS = 256 / TPR;
    __shared__ double part[4];
    const int t = (int)threadIdx.x % TPR;
    const long row = (long)blockIdx.x * ROWS + (int)threadIdx.x / TPR, at = row < T ? row : T - 1;
    const bool live = row < T;
    uint4 q[P], z[P];
#pragma unroll
    for (int p = 0; p < P; ++p) q[p] = load_whole<false, TINY>(X + at * ldx, (p * TPR + t) * V, n);
    if (res != nullptr) {
#pragma unroll
        for (int p = 0; p < P; ++p) z[p] = load_whole<false, TINY>(res + at * ldr, (p * TPR + t) * V, n);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int c = (p * TPR + t) * V;
            finish_piece<TINY>(q[p], X + at * ldx, c, n);
            finish_piece<TINY>(z[p], res + at * ldr, c, n);
            float h[V], r[V];
            unpack(q[p], h);
            unpack(z[p], r);
#pragma unroll
            for (int i = 0; i < V; ++i) h[i] += r[i];
            if constexpr (V == 8) q[p] = make_uint4(bf16_pair(h[0], h[1]), bf16_pair(h[2], h[3]), bf16_pair(h[4], h[5]), bf16_pair(h[6], h[7]));
            else q[p] = make_uint4(__float_as_uint(h[0]), __float_as_uint(h[1]), __float_as_uint(h[2]), __float_as_uint(h[3]));
        }
    } else {
#pragma unroll
        for (int p = 0; p < P; ++p) finish_piece<TINY>(q[p], X + at * ldx, (p * TPR + t) * V, n);
    }
    double ss = 0.0;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int c = (p * TPR + t) * V;
        if (H != nullptr && live) {
            if (c + V <= n) {
                store_sum<PAST>(H + row * ldh + c, q[p]);
            } else if (c < n) {
                const unsigned w[4] = {q[p].x, q[p].y, q[p].z, q[p].w};
#pragma unroll
                for (int i = 0; i < V - 1; ++i)
                    if (c + i < n) {
                        if constexpr (V == 4) H[row * ldh + c + i] = __uint_as_float(w[i]);
                        else H[row * ldh + c + i] = (bf16_t)(w[i / 2] >> (16 * (i & 1)));
                    }
            }
        }
        float h[V];
        unpack(q[p], h);
#pragma unroll
        for (int i = 0; i < V; ++i) ss += (double)h[i] * (double)h[i];
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
        float h[V], y[V];
        unpack(q[p], h);
        if (gain != nullptr) {
            float g[V];
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                uint4 u = load_whole<false, TINY>(gain, c + i, n);
                finish_piece<TINY>(u, gain, c + i, n);
                float g4[4];
                unpack(u, g4);
#pragma unroll
                for (int k = 0; k < 4; ++k) g[i + k] = g4[k];
            }
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = (float)((double)h[i] * f * (double)g[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = (float)((double)h[i] * f);
        }
        put_blocks<F, V>(y, unit, nb, codes + row * ldc, scales + row * lds, flags);
    }
}

// Squared error of the MX quantiser and its derivative:  loss_t = (1/n) sum_i (y_i - yhat_i)^2,  dY_i = c (2/n) (y_i - yhat_i).  yhat is
// constant around almost every y (the scale is a power of two), so this is the derivative wherever there is one.  Squares and sums in 64 bits: in 32 an
// error of 2^64 would make the loss infinite where the mean is not.
//
// Bound by HBM: 8192 x 4096 with a bf16 gradient, 201 MB, 34.1 us (5.9 TB/s); 64 problems of 2048 x 128 with an fp32 one, 134 MB, 24.9 us (5.4 TB/s); 10
// of 2849 x 648 32 us (53 with a row a workgroup at a time).
template <int F, bool BF16OUT, bool TINY>
__global__ __launch_bounds__(256) void mx_objective_kernel(const float* __restrict__ Y, long ldy, int T, int n, float scale, void* __restrict__ dYv,
                                                           long lddy, double* __restrict__ partials, long sy, long sdy, Walk w) {
    constexpr int U = 4;
    __shared__ double tot[4];
    Y += (long)blockIdx.y * sy;
    const float f = scale * 2.f / (float)n;
    double acc = 0.0;
    Place at = walk_start(w);
    while (at.row < (unsigned)T) {
        uint4 q[U];
        Place p[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            p[k] = at;
            const bool in = at.row < (unsigned)T;
            q[k] = load_whole<true, TINY>(Y + (long)(in ? at.row : 0u) * ldy, in ? at.unit * 4 : 0, n);
            at = walk_next(w, at, k < U - 1 ? w.near : w.far);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (p[k].row >= (unsigned)T) break;
            const long row = p[k].row;
            const int c = p[k].unit * 4;
            finish_piece<TINY>(q[k], Y + row * ldy, c, n);
            float v[4], e[4];
            unpack(q[k], v);
            const unsigned byte = mx_scale_byte<F>(mx_group_max<8>(piece_top(v)));
            unsigned code[1];
            mx_encode<F, 4>(v, byte, code);
            mx_decode4<F, 0>(code[0], mx_scale(byte), e);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e[i] = v[i] - e[i];          // NaN in a block of scale 255
                acc += (double)e[i] * (double)e[i];
                e[i] *= f;
            }
            if (dYv != nullptr && c < n) {
                if constexpr (BF16OUT) store_piece<4>(static_cast<bf16_t*>(dYv) + (long)blockIdx.y * sdy + row * lddy + c, n - c, e);
                else store_piece(static_cast<float*>(dYv) + (long)blockIdx.y * sdy + row * lddy + c, n - c, e);
            }
        }
    }
    acc = wave_sum(acc);
    if ((threadIdx.x & 63) == 0) tot[threadIdx.x >> 6] = acc;
    __syncthreads();
    if (threadIdx.x == 0) partials[(long)blockIdx.y * gridDim.x + blockIdx.x] = ((tot[0] + tot[1]) + (tot[2] + tot[3])) / (double)n;
}

int pieces_of(int n, int V) { return (int)((n + 31L) / 32) * (32 / V); }
// neighbouring pieces only where every workgroup gets `batch` times 256 of them
Walk make_walk(int T, int upr, int batch, long grid) {
    const int run = (long)T * upr >= 256 * batch * grid ? batch : 1;
    const long near = run > 1 ? 256 : 256 * grid, far = run > 1 ? 256 * (batch * grid - (batch - 1)) : 256 * grid;
    return Walk{upr, run, {(unsigned)(near / upr), (int)(near % upr)}, {(unsigned)(far / upr), (int)(far % upr)}};
}
// at most 16384 workgroups, and each `batch` pieces a thread where that leaves 2048 of them, eight for every compute unit
long walk_grid(int T, int upr, int batch) {
    const long tiles = ((long)T * upr + 255) / 256;
    long g = (tiles + batch - 1) / batch;
    g = g < 2048 ? 2048 : g > 16384 ? 16384 : g;
    return g < tiles ? g : tiles;
}

// The norm's sum leaves past the caches where the input alone is more than the L2s hold (32 MB), so that little of it would be found there when it is
// next wanted, behind a layer: 8192 x 4096 (bf16, 67 MB) 50 -> 45 us.  Of less, and of all codes, what follows reads them in the caches (the quantiser
// itself gains 34 -> 32 us at 8192 x 8192 by codes past them, and what reads those next loses 7).
bool past_caches(int T, int n, int is_bf16) { return (long)T * n * (is_bf16 ? 2 : 4) > (32L << 20); }

template <class IN, int F, int P, int TPR, bool TINY = false>
hipError_t norm_launch(const MxNorm& m, hipStream_t s) {
    constexpr int ROWS = 256 / TPR;
    const bool past = past_caches(m.T, m.n, m.x_is_bf16);
    // a launch counts its threads in 32 bits: 2^30 of them at a time
    for (long first = 0; first < m.T; first += (1L << 22) * ROWS) {
        const long left = m.T - first, rows = left < (1L << 22) * ROWS ? left : (1L << 22) * ROWS;
        const IN *X = static_cast<const IN*>(m.X) + first * m.ldx, *res = m.res != nullptr ? static_cast<const IN*>(m.res) + first * m.ldr : nullptr;
        IN* H = m.H != nullptr ? static_cast<IN*>(m.H) + first * m.ldh : nullptr;
#define DQ_GO(PAST)                                                                                                                          \
    hipLaunchKernelGGL((mx_rms_norm_kernel<IN, F, P, TPR, PAST, TINY>), dim3((unsigned)((rows + ROWS - 1) / ROWS)), dim3(256), 0, s, X, m.ldx, res, \
                       m.ldr, H, m.ldh, m.gain, m.eps, (int)rows, m.n, (m.n + 31) / 32, m.codes + first * m.ldc, m.ldc,                       \
                       m.scales + first * m.lds, m.lds, m.flags)
        if (past) DQ_GO(true); else DQ_GO(false);
#undef DQ_GO
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
// Pieces of a thread: as many as a row has, since others cost loads of what is there already and registers (1023 x 5004 fp32: 8 pieces 14.7 us, 5
// pieces 13.4).
template <class IN, int F, int TPR>
hipError_t norm_pieces(const MxNorm& m, hipStream_t s) {
    constexpr int V = Piece<IN>::V;
    switch ((m.n + TPR * V - 1) / (TPR * V)) {
        case 1: return norm_launch<IN, F, 1, TPR>(m, s);
        case 2: return norm_launch<IN, F, 2, TPR>(m, s);
        case 3: return norm_launch<IN, F, 3, TPR>(m, s);
        case 4: return norm_launch<IN, F, 4, TPR>(m, s);
        case 5: if constexpr (V == 4) return norm_launch<IN, F, 5, TPR>(m, s); break;
        case 6: if constexpr (V == 4 && TPR == 256) return norm_launch<IN, F, 6, TPR>(m, s); break;
        case 7: if constexpr (V == 4 && TPR == 256) return norm_launch<IN, F, 7, TPR>(m, s); break;
        case 8: if constexpr (V == 4 && TPR == 256) return norm_launch<IN, F, 8, TPR>(m, s); break;
    }
    return hipErrorInvalidValue;
}
// A wavefront a row where 4 pieces a lane in bf16, 5 in fp32, are enough (8192 rows: 1100 in bf16 24.4 us a workgroup a row, 17.1; 1500 26.4, 20.3; 1030
// in fp32 26.0, 24.1; but 1500 in fp32 29.3, 30.4), unless there are few rows (400 x 1000 fp32: 4.4, 3.4 a workgroup a row; 600 x 1500 bf16 5.2, 4.5).
template <class IN, int F>
hipError_t norm_shape(const MxNorm& m, hipStream_t s) {
    constexpr int V = Piece<IN>::V;
    if (m.n < V) return norm_launch<IN, F, 1, 64, true>(m, s);
    return m.n <= 64 * V || (m.n <= 64 * V * (V == 8 ? 4 : 5) && m.T > 1024) ? norm_pieces<IN, F, 64>(m, s) : norm_pieces<IN, F, 256>(m, s);
}

}  // namespace

hipError_t launch_mx_quantize(const void* X, int x_is_bf16, long ldx, int T, int n, int format, unsigned char* codes, long ldc, unsigned char* scales,
                              long lds, unsigned* flags, hipStream_t s) {
    if (T < 1 || n < 1) return hipSuccess;
    const int V = x_is_bf16 ? 8 : 4, upr = pieces_of(n, V);
    const long grid = walk_grid(T, upr, 4);
    const Walk w = make_walk(T, upr, 4, grid);
    const int nb = (int)((n + 31L) / 32);
#define DQ_GO(IN, F, TINY)                                                                                                                      \
    hipLaunchKernelGGL((mx_quantize_kernel<IN, F, TINY>), dim3((unsigned)grid), dim3(256), 0, s, static_cast<const IN*>(X), ldx, T, n, nb, codes, \
                       ldc, scales, lds, w, flags)
#define DQ_FORMAT(IN, TINY) do { if (format == DQ_MXFP4) DQ_GO(IN, DQ_MXFP4, TINY); else DQ_GO(IN, DQ_MXFP8, TINY); } while (0)
    if (x_is_bf16) { if (n < V) DQ_FORMAT(bf16_t, true); else DQ_FORMAT(bf16_t, false); }
    else { if (n < V) DQ_FORMAT(float, true); else DQ_FORMAT(float, false); }
#undef DQ_FORMAT
#undef DQ_GO
    return hipGetLastError();
}

hipError_t launch_mx_dequantize(int format, const unsigned char* codes, long ldc, const unsigned char* scales, long lds, int T, int n, void* Y,
                                int y_is_bf16, long ldy, hipStream_t s) {
    if (T < 1 || n < 1) return hipSuccess;
    const int upr = pieces_of(n, y_is_bf16 ? 8 : 4);
    const long grid = walk_grid(T, upr, 1);
    const Walk w = make_walk(T, upr, 1, grid);
#define DQ_GO(OUT, F)                                                                                                                        \
    hipLaunchKernelGGL((mx_dequantize_kernel<OUT, F>), dim3((unsigned)grid), dim3(256), 0, s, codes, ldc, scales, lds, T, n, static_cast<OUT*>(Y), \
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

// four pieces a thread, fewer in a small problem
int mx_objective_grid(int T, int n) {
    const long tiles = ((long)T * pieces_of(n, 4) + 255) / 256, few = tiles < 32 ? tiles : 32, g = (tiles + 3) / 4;
    return (int)(g < few ? few : g < 2048 ? g : 2048);
}

hipError_t launch_mx_objective(int format, const float* Y, long ldy, int T, int n, float scale, void* dY, int dy_is_bf16, long lddy, double* partials,
                               int grid, hipStream_t s, int batch, long stride_y, long stride_dy) {
    if (batch < 1 || T < 1) return hipSuccess;
    const Walk w = make_walk(T, pieces_of(n, 4), 4, grid);
#define DQ_GO(F, BF, TINY)                                                                                                                          \
    hipLaunchKernelGGL((mx_objective_kernel<F, BF, TINY>), dim3(grid, batch), dim3(256), 0, s, Y, ldy, T, n, scale, dY, lddy, partials, stride_y, \
                       stride_dy, w)
#define DQ_TYPE(F, TINY) do { if (dy_is_bf16) DQ_GO(F, true, TINY); else DQ_GO(F, false, TINY); } while (0)
    if (format == DQ_MXFP4) { if (n < 4) DQ_TYPE(DQ_MXFP4, true); else DQ_TYPE(DQ_MXFP4, false); }
    else { if (n < 4) DQ_TYPE(DQ_MXFP8, true); else DQ_TYPE(DQ_MXFP8, false); }
#undef DQ_TYPE
#undef DQ_GO
    return hipGetLastError();
}

}  // namespace dq
