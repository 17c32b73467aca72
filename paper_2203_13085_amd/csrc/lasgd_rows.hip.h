// Row-wise operators of the replicas' forward and backward passes: device code of dropout and of root-mean-square norms.
//
// Bound by HBM: a handful of operations per element that is read or written once.  A dropout draw is ten rounds of two 32-bit
// products for eight elements.
#pragma once
#include "lasgd_memory.hip.h"

#include <type_traits>

namespace lasgd {


struct RowsAt {             // element (k, r, c) is at p + (k * rs + r * ss + c) elements
    char *p;
    int64_t rs, ss;
};

struct DropArgs {
    uint64_t seed, call;
    const uint64_t *counter;     // added to call, or NULL
    uint32_t below;              // an element is dropped if its 16 bits are below this (0: no dropout; 65536: all are)
    float scale;                 // of those that stay
};

// ---- Philox 4x32, ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC 2011) ------------
__device__ __forceinline__ uint4 philox(uint4 c, uint2 key)
{
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
        c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ key.x, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ key.y, (uint32_t)a);
        key.x += 0x9E3779B9u;
        key.y += 0xBB67AE85u;
    }
    return c;
}

// The mask of eight columns: one draw, 16 bits an element, the low half of a word first.  16 bits and not 32: the draws are what
// a dropout pass would otherwise wait for (p is taken to the nearest 1/65536 and the scale is that number's, so means stay exact).
// The counter names the place (replica, row, group of eight columns) and the call, so a mask does not depend on the launch shape, on the
// layout, on how many replicas or rows there are, or on what ran before.
struct Lots {
    uint32_t w[4];
};
__device__ __forceinline__ Lots draw_lots(const DropArgs &d, uint64_t call, uint32_t k, uint64_t group)
{
    const uint4 w = philox(make_uint4((uint32_t)group, (uint32_t)(group >> 32) | k << 16, (uint32_t)call, (uint32_t)(call >> 32)),
                           make_uint2((uint32_t)d.seed, (uint32_t)(d.seed >> 32)));
    return Lots{{w.x, w.y, w.z, w.w}};
}
__device__ __forceinline__ bool stays(const Lots &l, int j, uint32_t below)
{
    const uint32_t lot = j & 1 ? l.w[j >> 1] >> 16 : l.w[j >> 1] & 0xffffu;
    return lot >= below;
}
__device__ __forceinline__ uint64_t call_number(const DropArgs &d)
{
    return d.counter ? d.call + *as_global<uint64_t>(d.counter) : d.call;
}

// ---- eight elements ------------------------------------------------------------------------------------------------------
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float widen_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float widen_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Two to bf16, to nearest, ties to even.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t narrow2(float a, float b)
{
    bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}

template <bool BF16> __device__ __forceinline__ float load1(const char *p, int64_t i)
{
    if constexpr (BF16) return __uint_as_float((uint32_t)as_global<uint16_t>(p)[i] << 16);
    else return as_global<float>(p)[i];
}
template <bool BF16> __device__ __forceinline__ void store1(char *p, int64_t i, float v)
{
    if constexpr (BF16) as_global<uint16_t>(p)[i] = __builtin_bit_cast(uint16_t, (__bf16)v);
    else as_global<float>(p)[i] = v;
}

// The type of a 16-byte access to elements of ES bytes that are aligned to themselves only.
template <int ES> struct Loose;
template <> struct Loose<2> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Loose<4> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4))); };

// Eight elements as they are in memory.
template <bool BF16> struct Raw8 { u32x4 w[BF16 ? 1 : 2]; };

// How a call's rows are accessed.  LOOSE: n elements are there, eight or more at once, fewer one by one.  (Rows that do not start on 16 bytes: a norm of 1023
// fp32 columns took 53 us with single accesses throughout, 18 so.)  WIDE: aligned, and all eight are there.  STREAM: the same with the streaming hint, for calls
// that move more than the memory-side cache holds.
enum Access : int { LOOSE = 0, WIDE = 1, STREAM = 2 };
template <bool BF16, int VEC> __device__ __forceinline__ Raw8<BF16> load_raw(const char *p, int64_t at, uint32_t n)
{
    constexpr int ES = BF16 ? 2 : 4;
    Raw8<BF16> r;
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < 8 * ES / 16; ++i) {
            if constexpr (VEC == STREAM) r.w[i] = __builtin_nontemporal_load(as_global<u32x4>(p + at * ES + i * 16));
            else r.w[i] = *as_global<u32x4>(p + at * ES + i * 16);
        }
    } else if (n >= 8u) {
#pragma unroll
        for (int i = 0; i < 8 * ES / 16; ++i) r.w[i] = *as_global<typename Loose<ES>::type>(p + at * ES + i * 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8 * ES / 16; ++i) r.w[i] = u32x4{};
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if ((uint32_t)j < n) {
                if constexpr (BF16) r.w[0][j >> 1] |= (uint32_t)as_global<uint16_t>(p)[at + j] << (16 * (j & 1));
                else r.w[j >> 2][j & 3] = as_global<uint32_t>(p)[at + j];
            }
    }
    return r;
}
template <bool BF16> __device__ __forceinline__ void widen8(float (&v)[8], const Raw8<BF16> &r)
{
    if constexpr (BF16) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[2 * j] = widen_lo(r.w[0][j]), v[2 * j + 1] = widen_hi(r.w[0][j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(r.w[j >> 2][j & 3]);
    }
}
template <bool BF16, int VEC> __device__ __forceinline__ void load8(float (&v)[8], const char *p, int64_t at, uint32_t n)
{
    widen8<BF16>(v, load_raw<BF16, VEC>(p, at, n));
}
template <bool BF16, int VEC> __device__ __forceinline__ void store8(char *p, int64_t at, uint32_t n, const float (&v)[8])
{
    constexpr int ES = BF16 ? 2 : 4;
    if (VEC || n >= 8u) {
        Raw8<BF16> r;
        if constexpr (BF16) {
#pragma unroll
            for (int j = 0; j < 4; ++j) r.w[0][j] = narrow2(v[2 * j], v[2 * j + 1]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) r.w[j >> 2][j & 3] = __float_as_uint(v[j]);
        }
#pragma unroll
        for (int i = 0; i < 8 * ES / 16; ++i) {
            if constexpr (VEC == STREAM) __builtin_nontemporal_store(r.w[i], as_global<u32x4>(p + at * ES + i * 16));
            else if constexpr (VEC) *as_global<u32x4>(p + at * ES + i * 16) = r.w[i];
            else *as_global<typename Loose<ES>::type>(p + at * ES + i * 16) = r.w[i];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if ((uint32_t)j < n) store1<BF16>(p, at + j, v[j]);
    }
}

// ---- dropout ---------------------------------------------------------------------------------------------------------------
//     y = residual + m x / (1 - p),      a dropped element counts 0 whatever it holds
// 8 x 4096 x 2048 bf16, with a residual and back: 671 MB in 118 us, 5.7 TB/s (a copy of 1 GiB reaches 5.2).
// A thread has eight columns of kDropRows rows at a time; a workgroup is tx threads along a row (a power of two) and 256 / tx rows.
constexpr uint32_t kDropRows = 4;

struct DropoutArgs {
    RowsAt x, residual, y;       // residual.p NULL: none
    DropArgs drop;
    uint32_t cols, groups;       // groups of eight columns
    uint32_t tx_shift;           // log2 of tx
    uint64_t row0;               // of a replica, that the launch starts with
    uint32_t rows[64];
};

template <bool BF16, int VEC>
__global__ __launch_bounds__(256) void dropout_kernel(const DropoutArgs a)
{
    const uint32_t k = blockIdx.y, rows = a.rows[k];
    const uint32_t ty = 256u >> a.tx_shift;
    const uint64_t r0 = a.row0 + (uint64_t)blockIdx.x * (ty * kDropRows);
    if (r0 >= rows) return;
    const uint32_t tx = threadIdx.x & ((1u << a.tx_shift) - 1u);
    const uint64_t r1 = r0 + (threadIdx.x >> a.tx_shift);
    const uint64_t call = call_number(a.drop);
    for (uint32_t g = tx; g < a.groups; g += 1u << a.tx_shift) {
        const uint32_t c = g * 8u, n = a.cols - c;
        Raw8<BF16> x[kDropRows], res[kDropRows];
#pragma unroll
        for (uint32_t u = 0; u < kDropRows; ++u) {
            const uint64_t r = r1 + u * ty;
            if (r < rows) {
                x[u] = load_raw<BF16, VEC>(a.x.p, k * a.x.rs + (int64_t)r * a.x.ss + c, n);
                if (a.residual.p) res[u] = load_raw<BF16, VEC>(a.residual.p, k * a.residual.rs + (int64_t)r * a.residual.ss + c, n);
            }
        }
#pragma unroll
        for (uint32_t u = 0; u < kDropRows; ++u) {
            const uint64_t r = r1 + u * ty;
            if (r >= rows) break;
            const Lots lots = draw_lots(a.drop, call, k, r * a.groups + g);
            float y[8], z[8];
            widen8<BF16>(y, x[u]);
            if (a.residual.p) widen8<BF16>(z, res[u]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                y[j] = stays(lots, j, a.drop.below) ? y[j] * a.drop.scale : 0.f;
                if (a.residual.p) y[j] = z[j] + y[j];
            }
            store8<BF16, VEC>(a.y.p, k * a.y.rs + (int64_t)r * a.y.ss + c, n, y);
        }
    }
}

// ---- root-mean-square norm ----------------------------------------------------------------------------------------------------
//     h = residual + m x / (1 - p),   rho = (mean h^2 + eps)^(-1/2),   y = gain (h rho)
// 8 x 4096 x 2048 bf16 with a residual: 537 MB in 90 us, 5.9 TB/s; 8 x 2048 x 4096 in 8 bits 470 MB in 90.
// G threads hold a row, NV groups of eight columns each, so everything is read once; h is rounded where it is stored, and enters the norm
// as it was before.
//
// In 8 bits (OUT8): scale = max |y| / 448, at least the smallest normal number, and y / scale to e4m3, of whose values so few are that with a norm in fp32, whose
// roundings add up to some of its last places, 1 in 10^6 quotients would cross a border between two and end up an eighth off. So this form computes in 64 bits from
// the loaded values on, which the memory hides. The instruction that makes e4m3 takes fp32: a quotient within half a step of fp32 (2^-24) of a border comes to lie on it and
// goes to its even side, as in any conversion of an fp32 array (of uniform quotients 3 in 10^7 change sides so).
constexpr double kE4m3Max = 448.0;
constexpr double kLeastScale = 1.1754943508222875e-38;

struct NormRowsArgs {
    RowsAt x, residual, sum, y, scales;
    DropArgs drop;
    uint32_t cols, groups;
    float eps, inv_cols;
    uint64_t row0;               // of a replica, that the launch starts with
    uint32_t rows[64];
    const char *gain[64];
};

// Sum over the G threads of a row, the same in all of them.  lds: one a wave.
template <int G, class T> __device__ __forceinline__ T row_sum(T v, T *lds)
{
#pragma unroll
    for (int d = (G < 64 ? G : 64) / 2; d; d >>= 1) v += __shfl_xor(v, d, 64);
    if constexpr (G > 64) {
        __syncthreads();                 // the words of the sum before
        if ((threadIdx.x & 63u) == 0u) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = T(0);
#pragma unroll
        for (int w = 0; w < G / 64; ++w) v += lds[w];
    }
    return v;
}
// Two at once.
template <int G> __device__ __forceinline__ float2 row_sums(float2 v, float2 *lds)
{
#pragma unroll
    for (int d = (G < 64 ? G : 64) / 2; d; d >>= 1) v.x += __shfl_xor(v.x, d, 64), v.y += __shfl_xor(v.y, d, 64);
    if constexpr (G > 64) {
        __syncthreads();
        if ((threadIdx.x & 63u) == 0u) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < G / 64; ++w) v.x += lds[w].x, v.y += lds[w].y;
    }
    return v;
}
template <class T> __device__ __forceinline__ T larger(T a, T b) { return b > a || b != b ? b : a; }      // a NaN stays
template <int G, class T> __device__ __forceinline__ T row_max(T v, T *lds)
{
#pragma unroll
    for (int d = (G < 64 ? G : 64) / 2; d; d >>= 1) v = larger(v, __shfl_xor(v, d, 64));
    if constexpr (G > 64) {
        __syncthreads();
        if ((threadIdx.x & 63u) == 0u) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int w = 1; w < G / 64; ++w) v = larger(v, lds[w]);
    }
    return v;
}

constexpr int norm_threads(int G) { return G > 256 ? G : 256; }

__device__ __forceinline__ float reciprocal_root(float v) { return 1.f / __builtin_sqrtf(v); }
__device__ __forceinline__ double reciprocal_root(double v) { return 1.0 / __builtin_sqrt(v); }

template <bool BF16, int VEC, int G, int NV, bool OUT8>
__global__ __launch_bounds__(norm_threads(G)) void rms_norm_kernel(const NormRowsArgs a)
{
    typedef std::conditional_t<OUT8, double, float> T;
    __shared__ T lds[G > 64 ? G / 64 : 1];
    constexpr uint32_t R = norm_threads(G) / G;              // rows a workgroup
    const uint32_t k = blockIdx.y, rows = a.rows[k];
    const uint64_t r0 = a.row0 + (uint64_t)blockIdx.x * R, r = r0 + threadIdx.x / G;
    if (r0 >= rows) return;
    if (G <= 64 && r >= rows) return;                        // (with G > 64 a workgroup is one row)
    const uint32_t t = threadIdx.x % G;
    const uint64_t call = a.drop.below ? call_number(a.drop) : 0;
    const T stay = OUT8 ? a.drop.below < 65536u ? T(65536) / T(65536u - a.drop.below) : T(0) : T(a.drop.scale);
    const char *gain = a.gain[k];
    T h[NV][8];
    T sum = 0;
    {
        Raw8<BF16> x[NV], res[NV];               // all asked for before the first is looked at
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t g = t + i * G, c = g * 8u;
            x[i] = Raw8<BF16>{};
            if (g < a.groups) x[i] = load_raw<BF16, VEC>(a.x.p, k * a.x.rs + (int64_t)r * a.x.ss + c, a.cols - c);
        }
        if (a.residual.p) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t g = t + i * G, c = g * 8u;
                res[i] = Raw8<BF16>{};
                if (g < a.groups) res[i] = load_raw<BF16, VEC>(a.residual.p, k * a.residual.rs + (int64_t)r * a.residual.ss + c, a.cols - c);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t g = t + i * G, c = g * 8u;
            float v[8];
            widen8<BF16>(v, x[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[i][j] = v[j];
            if (a.drop.below) {
                const Lots lots = draw_lots(a.drop, call, k, r * a.groups + g);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] = stays(lots, j, a.drop.below) ? h[i][j] * stay : T(0);
            }
            if (a.residual.p) {
                widen8<BF16>(v, res[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] = T(v[j]) + h[i][j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = OUT8 ? T(__builtin_fma((double)h[i][j], (double)h[i][j], (double)sum))
                                                   : T(__builtin_fmaf((float)h[i][j], (float)h[i][j], (float)sum));
            if (a.sum.p && g < a.groups) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = (float)h[i][j];
                store8<BF16, VEC>(a.sum.p, k * a.sum.rs + (int64_t)r * a.sum.ss + c, a.cols - c, v);
            }
        }
    }
    sum = row_sum<G>(sum, lds);
    const T rho = reciprocal_root(OUT8 ? sum / T(a.cols) + T(a.eps) : T(__builtin_fmaf((float)sum, a.inv_cols, a.eps)));
    T most = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t g = t + i * G, c = g * 8u;
        if (g < a.groups) {
            float w[8];
            load8<BF16, VEC ? WIDE : LOOSE>(w, gain, c, a.cols - c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[i][j] = T(w[j]) * (h[i][j] * rho);
                if constexpr (OUT8) most = larger(most, h[i][j] < 0 ? -h[i][j] : h[i][j]);
            }
            if constexpr (!OUT8) store8<BF16, VEC>(a.y.p, k * a.y.rs + (int64_t)r * a.y.ss + c, a.cols - c, h[i]);
        }
    }
    if constexpr (OUT8) {
        most = row_max<G>(most, lds);
        double scale = most / kE4m3Max;
        if (scale < kLeastScale) scale = kLeastScale;
        const double inv = 1.0 / scale;
        if (t == 0u) as_global<float>(a.scales.p)[k * a.scales.rs + (int64_t)r * a.scales.ss] = (float)scale;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t g = t + i * G, c = g * 8u;
            if (g < a.groups) {
                uint32_t q[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    int w = 0;
                    w = __builtin_amdgcn_cvt_pk_fp8_f32((float)(h[i][4 * j] * inv), (float)(h[i][4 * j + 1] * inv), w, false);
                    w = __builtin_amdgcn_cvt_pk_fp8_f32((float)(h[i][4 * j + 2] * inv), (float)(h[i][4 * j + 3] * inv), w, true);
                    q[j] = (uint32_t)w;
                }
                char *y = a.y.p + (k * a.y.rs + (int64_t)r * a.y.ss + c);
                typedef uint32_t loose2 __attribute__((ext_vector_type(2), aligned(1)));
                if constexpr (VEC) *as_global<u32x2>(y) = u32x2{q[0], q[1]};
                else if (a.cols - c >= 8u) *as_global<loose2>(y) = u32x2{q[0], q[1]};
                else {
#pragma unroll
                    for (uint32_t j = 0; j < 8u; ++j)
                        if (c + j < a.cols) *as_global<uint8_t>(y + j) = (uint8_t)(q[j >> 2] >> (8u * (j & 3u)));
                }
            }
        }
    }
}

// The backward pass, with hhat = h rho:
//     dh = rho (gain dy - hhat mean(hhat gain dy)) + dsum,   dx = m dh / (1 - p),   dgain = sum over the rows of dy hhat
// 8 x 4096 x 2048 bf16 with all five arrays: 671 MB in 136 us, 4.9 TB/s, and 5 for the shares.
// rho is made again from h, which is read anyway.  h is the sum as it was stored: to make it again from x, the residual and the mask would read a fifth more. In
// bf16 that leaves dgain 0.0023 off (root mean square, relative), where one rounding of the result is 0.0017; dx and dresidual, with a dsum beside them, 0.0017.
// A workgroup takes rows one after the other and adds up its share of dgain
// in registers; the shares of a replica's workgroups go to the workspace and are added in their order by join_gain_kernel.
struct NormBackArgs {
    RowsAt h, dy, dsum, dresidual, dx;       // dsum, dresidual, dx: may be NULL
    DropArgs drop;
    uint32_t cols, groups;
    float eps, inv_cols;
    uint32_t parts;              // workgroups a replica
    float *part;                 // [K][parts][groups * 8]
    uint32_t rows[64];
    const char *gain[64];
};

template <bool BF16, int VEC, int G, int NV>
__global__ __launch_bounds__(norm_threads(G)) void rms_norm_backward_kernel(const NormBackArgs a)
{
    __shared__ float2 lds[G > 64 ? G / 64 : 1];
    constexpr bool AHEAD = G < 1024;             // the next row is on its way while this one is worked on; 1024 threads have no registers for it
    constexpr uint32_t R = norm_threads(G) / G;
    const uint32_t k = blockIdx.y, rows = a.rows[k];
    const uint32_t t = threadIdx.x % G, lane_row = threadIdx.x / G;
    const uint64_t call = a.drop.below ? call_number(a.drop) : 0;
    const char *gain = a.gain[k];
    float acc[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
    }
    struct Row {
        Raw8<BF16> h[NV], dy[NV], dsum[NV];
    };
    auto ask = [&](Row &row, uint64_t r) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t g = t + i * G, c = g * 8u;
            row.h[i] = row.dy[i] = row.dsum[i] = Raw8<BF16>{};
            if (g < a.groups && r < rows) {
                row.h[i] = load_raw<BF16, VEC>(a.h.p, k * a.h.rs + (int64_t)r * a.h.ss + c, a.cols - c);
                row.dy[i] = load_raw<BF16, VEC>(a.dy.p, k * a.dy.rs + (int64_t)r * a.dy.ss + c, a.cols - c);
                if (a.dsum.p) row.dsum[i] = load_raw<BF16, VEC>(a.dsum.p, k * a.dsum.rs + (int64_t)r * a.dsum.ss + c, a.cols - c);
            }
        }
    };
    const uint64_t on = (uint64_t)a.parts * R;
    Row row;
    ask(row, (uint64_t)blockIdx.x * R + lane_row);
    for (uint64_t r = (uint64_t)blockIdx.x * R + lane_row; r < rows; r += on) {
        Row next;
        if constexpr (AHEAD) ask(next, r + on);
        float sum = 0.f, dot = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t g = t + i * G, c = g * 8u;
            if (g < a.groups) {
                float w[8], h[8], d[8];
                load8<BF16, VEC ? WIDE : LOOSE>(w, gain, c, a.cols - c);
                widen8<BF16>(h, row.h[i]);
                widen8<BF16>(d, row.dy[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sum = __builtin_fmaf(h[j], h[j], sum);
                    dot = __builtin_fmaf(h[j], w[j] * d[j], dot);
                }
            }
        }
        const float2 both = row_sums<G>(make_float2(sum, dot), lds);
        sum = both.x, dot = both.y;
        const float rho = 1.f / __builtin_sqrtf(__builtin_fmaf(sum, a.inv_cols, a.eps));
        const float mean = dot * rho * a.inv_cols;           // of hhat gain dy
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t g = t + i * G, c = g * 8u;
            if (g < a.groups) {
                float w[8], h[8], d[8], more[8];
                load8<BF16, VEC ? WIDE : LOOSE>(w, gain, c, a.cols - c);
                widen8<BF16>(h, row.h[i]);
                widen8<BF16>(d, row.dy[i]);
                if (a.dsum.p) widen8<BF16>(more, row.dsum[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float hat = h[j] * rho;
                    acc[i][j] = __builtin_fmaf(d[j], hat, acc[i][j]);
                    d[j] = rho * __builtin_fmaf(-hat, mean, w[j] * d[j]);
                    if (a.dsum.p) d[j] += more[j];
                }
                if (a.dresidual.p) store8<BF16, VEC>(a.dresidual.p, k * a.dresidual.rs + (int64_t)r * a.dresidual.ss + c, a.cols - c, d);
                if (a.dx.p) {
                    if (a.drop.below) {
                        const Lots lots = draw_lots(a.drop, call, k, r * a.groups + g);
#pragma unroll
                        for (int j = 0; j < 8; ++j) d[j] = stays(lots, j, a.drop.below) ? d[j] * a.drop.scale : 0.f;
                    }
                    store8<BF16, VEC>(a.dx.p, k * a.dx.rs + (int64_t)r * a.dx.ss + c, a.cols - c, d);
                }
            }
        }
        if constexpr (AHEAD) row = next;
        else ask(row, r + on);
    }
    // the workgroup's rows, added in their order
    if constexpr (R > 1) {
        __shared__ float sums[R - 1][G * NV][9];
        if (lane_row) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
#pragma unroll
                for (int j = 0; j < 8; ++j) sums[lane_row - 1][i * G + t][j] = acc[i][j];
            }
        }
        __syncthreads();
        if (lane_row) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                for (uint32_t o = 0; o < R - 1u; ++o) acc[i][j] += sums[o][i * G + t][j];
            }
        }
    }
    const uint64_t part = (uint64_t)k * a.parts + blockIdx.x;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t g = t + i * G;
        if (g < a.groups) store8<false, WIDE>(reinterpret_cast<char *>(a.part), (int64_t)(part * a.groups + g) * 8, 8u, acc[i]);
    }
}

struct JoinArgs {
    const float *part;           // [K][shares][groups * 8]
    uint32_t shares, cols, groups;
    int32_t accumulate;
    char *grad[64];
};

// The shares of a column, added in their order: 16 threads, one share in 16 each, and then those.
template <bool BF16>
__global__ __launch_bounds__(256) void join_gain_kernel(const JoinArgs a)
{
    __shared__ float lds[16][17];
    const uint32_t k = blockIdx.y, x = threadIdx.x & 15u, y = threadIdx.x >> 4;
    const uint32_t c = blockIdx.x * 16u + x;
    float sum = 0.f;
    if (c < a.cols)
        for (uint32_t s = y; s < a.shares; s += 16u) sum += as_global<float>(a.part)[((uint64_t)k * a.shares + s) * (a.groups * 8u) + c];
    lds[y][x] = sum;
    __syncthreads();
    if (y == 0u && c < a.cols) {
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += lds[i][x];
        if (a.accumulate) sum += load1<BF16>(a.grad[k], c);
        store1<BF16>(a.grad[k], c, sum);
    }
}

} // namespace lasgd
