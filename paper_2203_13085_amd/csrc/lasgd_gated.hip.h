// Gated blocks of the replicas' forward and backward passes: device code.
//     g = x Wg^T,  u = x Wu^T,  a = f(g) u
//     dg = da u f'(g),  du = da f(g);   dx = dg Wg + du Wu,   dWg = dg^T x,  dWu = du^T x
// Each replica (blockIdx.y) has weights of its own, as many rows as it likes, and all are in one launch.
#pragma once
#include "lasgd_rows.hip.h"

namespace lasgd {

enum Act : int { ACT_SILU = 0, ACT_GELU = 1, ACT_GELU_TANH = 2, ACT_RELU = 3 };

struct ActPair {
    float f, slope;
};

// The activation and its slope, in 32 bits.
__device__ __forceinline__ ActPair activation(int act, float v)
{
    switch (act) {
    case ACT_SILU: {
        const float s = 1.f / (1.f + expf(-v));
        return {v * s, s * __builtin_fmaf(v, 1.f - s, 1.f)};
    }
    case ACT_GELU: {
        const float cdf = 0.5f * (1.f + erff(v * 0.70710678118654752f));
        return {v * cdf, __builtin_fmaf(v * 0.39894228040143268f, expf(-0.5f * v * v), cdf)};
    }
    case ACT_GELU_TANH: {
        constexpr float b = 0.79788456080286536f, c = 0.044715f;
        const float t = tanhf(b * __builtin_fmaf(c * v * v, v, v));
        return {0.5f * v * (1.f + t), 0.5f * (1.f + t) + 0.5f * v * (1.f - t * t) * b * __builtin_fmaf(3.f * c * v, v, 1.f)};
    }
    default: return {v > 0.f ? v : v == v ? 0.f : v, v > 0.f ? 1.f : 0.f};
    }
}

// ---- dg and du -----------------------------------------------------------------------------------------------------------
// Bound by HBM.  dg and du are rounded to the storage type here, as g and u were: the products that read them take that type.
struct GatesArgs {
    RowsAt g, u, da;
    char *dg, *du;               // [rows of all replicas][pitch]
    uint32_t wide, groups, pitch;
    int32_t act;
    uint32_t rows[64];
    uint32_t first[64];          // rows of the replicas before
};

template <bool BF16, bool VEC>
__global__ __launch_bounds__(256) void gates_backward_kernel(const GatesArgs a)
{
    const uint32_t k = blockIdx.y, rows = a.rows[k];
    for (uint64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (uint32_t g = threadIdx.x; g < a.groups; g += 256u) {
            const uint32_t c = g * 8u, n = a.wide - c;
            float gv[8], uv[8], dv[8];
            load8<BF16, VEC>(gv, a.g.p, k * a.g.rs + (int64_t)r * a.g.ss + c, n);
            load8<BF16, VEC>(uv, a.u.p, k * a.u.rs + (int64_t)r * a.u.ss + c, n);
            load8<BF16, VEC>(dv, a.da.p, k * a.da.rs + (int64_t)r * a.da.ss + c, n);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const ActPair f = activation(a.act, gv[j]);
                gv[j] = dv[j] * uv[j] * f.slope;
                uv[j] = dv[j] * f.f;
            }
            const int64_t at = (int64_t)(a.first[k] + r) * a.pitch + c;
            store8<BF16, true>(a.dg, at, 8u, gv);            // whole groups: the columns behind the last are the workspace's own
            store8<BF16, true>(a.du, at, 8u, uv);
        }
}

// ---- products -------------------------------------------------------------------------------------------------------------
// C[m][n] = sum over c of M[m][c] N[n][c], in one of three forms:
//   FWD  m: rows, n: hidden, c: model;   N twice (gate and up), joined by the activation where C is stored
//   DX   m: rows, n: model,  c: hidden;  both pairs (dg, gate) and (du, up) into one C
//   DW   m: hidden, n: model, c: rows;   one launch for both weights
enum Form : int { FWD = 0, DX = 1, DW = 2 };

struct ProductArgs {
    RowsAt x, g, u, a;           // FWD: a, and g and u unless NULL; DX: a is dx; DW: x
    const char *dg, *du;         // DX, DW: [rows of all replicas][pitch]
    uint32_t cols, wide, pitch;
    int32_t act, accumulate;
    uint32_t rows[64];
    uint32_t first[64];
    char *gate[64], *up[64];     // the weights; DW: their gradients
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---- any size, stride and alignment ------------------------------------------------------------------------------------------
// Tiles of 64 x 64, four waves of 32 x 32, 32 of the contraction at a time through LDS, where both sides lie [64][32] whatever they are in memory; what is
// outside is zero there.
constexpr uint32_t kTile = 64, kDeep = 32;

template <bool BF16> struct Elem { typedef float type; static constexpr uint32_t pitch = kDeep + 1; };
template <> struct Elem<true> { typedef uint16_t type; static constexpr uint32_t pitch = kDeep + 8; };

// One side's tile: element (i, c) of i < ni, c < nc is at p + i * stride + c (ALONG) or p + c * stride + i.
// Eight at a time along what is contiguous; VEC: these are aligned, and ni or nc counts whole eights.
template <bool BF16, bool ALONG, bool VEC>
__device__ __forceinline__ void stage(typename Elem<BF16>::type *lds, const char *p, int64_t stride, int64_t i0, int64_t ni, int64_t c0, int64_t nc)
{
    constexpr uint32_t P = Elem<BF16>::pitch;
    const uint32_t t = threadIdx.x;
    const uint32_t il = ALONG ? t >> 2 : (t & 7u) * 8u, cl = ALONG ? (t & 3u) * 8u : t >> 3;
    const int64_t i = i0 + il, c = c0 + cl;
    const int64_t left = ALONG ? (i < ni ? nc - c : 0) : (c < nc ? ni - i : 0);
    const uint32_t n = left >= 8 ? 8u : left > 0 ? (uint32_t)left : 0u;
    const int64_t at = ALONG ? i * stride + c : c * stride + i;
    float v[8];
    if (VEC && n) load8<BF16, VEC>(v, p, at, 8u);
    else load8<BF16, false>(v, p, at, VEC ? 0u : n);
#pragma unroll
    for (uint32_t j = 0; j < 8u; ++j) {
        const uint32_t w = ALONG ? il * P + cl + j : (il + j) * P + cl;
        if constexpr (BF16) lds[w] = (uint16_t)(__float_as_uint(v[j]) >> 16);          // exact: it was bf16
        else lds[w] = v[j];
    }
}

// acc += the tile's part of C: element (n = 4 * (lane / 16) + reg, m = lane % 16) of each 16 x 16.
template <bool BF16>
__device__ __forceinline__ void multiply(f32x4 (&acc)[2][2], const typename Elem<BF16>::type *m, const typename Elem<BF16>::type *n, uint32_t wm, uint32_t wn)
{
    constexpr uint32_t P = Elem<BF16>::pitch;
    const uint32_t lane = threadIdx.x & 63u, row = lane & 15u, quad = lane >> 4;
    if constexpr (BF16) {
        bf16x8 fm[2], fn[2];
#pragma unroll
        for (uint32_t i = 0; i < 2u; ++i) {
            fm[i] = *reinterpret_cast<const bf16x8 *>(m + (wm * 32u + i * 16u + row) * P + quad * 8u);
            fn[i] = *reinterpret_cast<const bf16x8 *>(n + (wn * 32u + i * 16u + row) * P + quad * 8u);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fn[j], fm[i], acc[i][j], 0, 0, 0);
        }
    } else {
#pragma unroll
        for (uint32_t c = 0; c < kDeep; c += 4u) {
            float fm[2], fn[2];
#pragma unroll
            for (uint32_t i = 0; i < 2u; ++i) {
                fm[i] = m[(wm * 32u + i * 16u + row) * P + c + quad];
                fn[i] = n[(wn * 32u + i * 16u + row) * P + c + quad];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fn[j], fm[i], acc[i][j], 0, 0, 0);
            }
        }
    }
}

template <bool BF16, int FORM, bool VM, bool VN>
__global__ __launch_bounds__(256) void product_kernel(const ProductArgs a)
{
    typedef typename Elem<BF16>::type T;
    constexpr uint32_t ES = BF16 ? 2u : 4u;
    __shared__ __attribute__((aligned(16))) T ldsm[kTile * Elem<BF16>::pitch], ldsn[(FORM == FWD ? 2 : 1) * kTile * Elem<BF16>::pitch];
    const uint32_t k = blockIdx.y;
    const int64_t rows = a.rows[k], cols = a.cols, wide = a.wide;
    const int64_t M = FORM == DW ? wide : rows, N = FORM == FWD ? wide : cols;
    const uint32_t tn = (uint32_t)((N + kTile - 1) / kTile);
    const int64_t m0 = (int64_t)(blockIdx.x / tn) * kTile, n0 = (int64_t)(blockIdx.x % tn) * kTile;
    if (m0 >= M) return;
    const uint32_t w = threadIdx.x >> 6, wm = w >> 1, wn = w & 1u;
    f32x4 acc[FORM == FWD ? 2 : 1][2][2] = {};
    const char *dg = a.dg + (uint64_t)a.first[k] * a.pitch * ES, *du = a.du + (uint64_t)a.first[k] * a.pitch * ES;
    const int64_t deep = FORM == FWD ? cols : FORM == DX ? wide : rows;
    for (int half = 0; half < (FORM == DX ? 2 : 1); ++half)
        for (int64_t c = 0; c < deep; c += kDeep) {
            if constexpr (FORM == FWD) {
                stage<BF16, true, VM>(ldsm, a.x.p + k * a.x.rs * ES, a.x.ss, m0, M, c, deep);
                stage<BF16, true, VN>(ldsn, a.gate[k], cols, n0, N, c, deep);
                stage<BF16, true, VN>(ldsn + kTile * Elem<BF16>::pitch, a.up[k], cols, n0, N, c, deep);
            } else if constexpr (FORM == DX) {
                stage<BF16, true, VM>(ldsm, half ? du : dg, a.pitch, m0, M, c, deep);
                stage<BF16, false, VN>(ldsn, half ? a.up[k] : a.gate[k], cols, n0, N, c, deep);
            } else {
                stage<BF16, false, VM>(ldsm, blockIdx.z ? du : dg, a.pitch, m0, M, c, deep);
                stage<BF16, false, VN>(ldsn, a.x.p + k * a.x.rs * ES, a.x.ss, n0, N, c, deep);
            }
            __syncthreads();
            multiply<BF16>(acc[0], ldsm, ldsn, wm, wn);
            if constexpr (FORM == FWD) multiply<BF16>(acc[1], ldsm, ldsn + kTile * Elem<BF16>::pitch, wm, wn);
            __syncthreads();
        }
    const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t m = m0 + wm * 32u + i * 16 + (lane & 15u), n1 = n0 + wn * 32u + j * 16 + (lane >> 4) * 4u;
            if (m >= M) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t n = n1 + e;
                if (n >= N) continue;
                if constexpr (FORM == FWD) {
                    const float g = acc[0][i][j][e], u = acc[1][i][j][e];
                    store1<BF16>(a.a.p, k * a.a.rs + m * a.a.ss + n, activation(a.act, g).f * u);
                    if (a.g.p) {
                        store1<BF16>(a.g.p, k * a.g.rs + m * a.g.ss + n, g);
                        store1<BF16>(a.u.p, k * a.u.rs + m * a.u.ss + n, u);
                    }
                } else if constexpr (FORM == DX) {
                    store1<BF16>(a.a.p, k * a.a.rs + m * a.a.ss + n, acc[0][i][j][e]);
                } else {
                    char *grad = blockIdx.z ? a.up[k] : a.gate[k];
                    float v = acc[0][i][j][e];
                    if (a.accumulate) v += load1<BF16>(grad, m * cols + n);
                    store1<BF16>(grad, m * cols + n, v);
                }
            }
        }
    }
}

} // namespace lasgd
