// Gated blocks of the replicas' forward and backward passes: device code.
//     g = x Wg^T,  u = x Wu^T,  a = f(g) u
//     dg = da u f'(g),  du = da f(g);   dx = dg Wg + du Wu,   dWg = dg^T x,  dWu = du^T x
// Each replica has weights of its own and as many rows as it likes, and all are in one launch.
#pragma once
#include "lasgd_rows.hip.h"

namespace lasgd {

enum Act : int { ACT_SILU = 0, ACT_GELU = 1, ACT_GELU_TANH = 2, ACT_RELU = 3 };

struct ActPair {
    float f, slope;
};

// 1 / (1 + exp(-v)).  BF16: by the two instructions for it, some roundings of 2^-24 (and of v's size, where the result is small) off, which the rounding to 8
// bits that follows hides.  (Forward product of K = 8, 2048 rows, 2048 x 5504: 804 us so, 819 with an exact division and exponential.)
template <bool BF16> __device__ __forceinline__ float sigmoid(float v)
{
    if constexpr (BF16) return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896341f * v));
    else return 1.f / (1.f + expf(-v));
}

// The activation and its slope, in 32 bits.
template <bool BF16> __device__ __forceinline__ ActPair activation(int act, float v)
{
    switch (act) {
    case ACT_SILU: {
        const float s = sigmoid<BF16>(v);
        return {v * s, s * __builtin_fmaf(v, 1.f - s, 1.f)};
    }
    case ACT_GELU: {
        const float cdf = 0.5f * erfcf(v * -0.70710678118654752f);             // 1 + erf would lose what is small
        return {v * cdf, __builtin_fmaf(v * 0.39894228040143268f, expf(-0.5f * v * v), cdf)};
    }
    case ACT_GELU_TANH: {
        constexpr float b = 0.79788456080286536f, c = 0.044715f;
        const float s = sigmoid<BF16>(2.f * b * __builtin_fmaf(c * v * v, v, v));             // (1 + tanh z) / 2
        const float t = s * (1.f - s);                                           // 0 long before v^3 is beyond fp32, from 1.3e13 on
        return {v * s, t == 0.f ? s : __builtin_fmaf(2.f * b * v * __builtin_fmaf(3.f * c * v, v, 1.f), t, s)};
    }
    default: return {v > 0.f ? v : v == v ? 0.f : v, v > 0.f ? 1.f : 0.f};
    }
}

// ---- dg and du -----------------------------------------------------------------------------------------------------------
// Bound by HBM: 900 MB (K = 8, 2048 rows, 5504 wide, bf16) in 148 us, 6.1 TB/s; 4 rows in 6.
//
// dg and du are rounded to the storage type here, as g and u were: the matrix instructions take that type, and 32 bits of g and u would double what is kept
// between the passes.  With bf16 the gradients end up 0.0031 off (root mean square, relative), where a single rounding of the result is 0.0017.
struct GatesArgs {
    RowsAt g, u, da;
    char *dg, *du;               // [rows of all replicas][pitch]
    uint32_t wide, groups, pitch;
    int32_t act;
    uint32_t rows[64];
    uint32_t first[64];          // rows of the replicas before
};

template <bool BF16, int VEC>
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
                const ActPair f = activation<BF16>(a.act, gv[j]);
                gv[j] = dv[j] * uv[j] * f.slope;
                uv[j] = dv[j] * f.f;
            }
            const int64_t at = (int64_t)(a.first[k] + r) * a.pitch + c;
            store8<BF16, WIDE>(a.dg, at, 8u, gv);            // whole groups: the columns behind the last are the workspace's own
            store8<BF16, WIDE>(a.du, at, 8u, uv);
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
    uint32_t tiles, tiles_m;     // product_kernel: of a replica, and of its rows
    int32_t wide_out;            // outputs take accesses of eight elements
    uint32_t rows[64];
    uint32_t first[64];
    char *gate[64], *up[64];     // the weights; DW: their gradients
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// A quotient: divisions are made by the vector unit, and what comes of one stays in vector registers, with all that is computed from it.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// Workgroups are dealt out to the eight XCDs in turn; each XCD gets tiles that follow each other, which share their sides in its L2.
__device__ __forceinline__ uint32_t xcd_order(uint32_t id, uint32_t total)
{
    const uint32_t x = id & 7u, per = total >> 3, more = total & 7u;
    return x * per + (x < more ? x : more) + (id >> 3);
}

// ---- a tile's sides in LDS ------------------------------------------------------------------------------------------------------------
//   - A side whose contraction is contiguous in memory (ALONG) lies in LDS as [row][LP pieces of 16 bytes], and is read 16 bytes a lane.  Piece p of row i is
//     at p ^ (i & 7), or p ^ (i / 2 & 3) where a step has four: eight rows' equal pieces are in eight different places of 128 bytes.
//   - A side whose rows are contiguous (ACROSS) lies as [contraction][T elements].  bf16: read by the transposing read, 16 lanes of which take 4 lines of 16
//     columns, and a lane gets one column of them; piece p of line c is at p ^ 2 (c & 3) ^ (c & 8) (where a line has sixteen), so that the 8 lines that half a wave reads
//     are in eight different places of 256 bytes.  fp32: read an element a lane; p ^ (c & 12): the four lines of a wave are in four different places.
template <bool BF16> struct Width {
    static constexpr uint32_t bytes = BF16 ? 2 : 4, piece = 16u / bytes, deep = 4u * piece;        // of an element; elements; a fragment's contraction
};
// Where piece p of a line is.
template <uint32_t LP> __device__ __forceinline__ uint32_t along_place(uint32_t row, uint32_t p) { return p ^ (LP == 8u ? row & 7u : row >> 1 & 3u); }
template <bool BF16, uint32_t T> __device__ __forceinline__ uint32_t across_place(uint32_t line, uint32_t p)
{
    static_assert(T >= 64u, "a line has all the places");
    return p ^ (BF16 ? (line & 3u) * 2u ^ (T >= 128u ? line & 8u : 0u) : line & 12u);
}

typedef __attribute__((address_space(3))) char lds_char;
typedef short s16x4 __attribute__((ext_vector_type(4)));

// What a lane has of 16 rows from row0 on and of the contraction from c0 on: row lane % 16, and of 32 (bf16: 16 bytes) or 16 (fp32) of the contraction
// the share of its quarter of the wave.  Both sides take it in the same order, which is all that counts.
template <bool BF16> struct Frag { typedef f32x4 type; };
template <> struct Frag<true> { typedef bf16x8 type; };
template <bool BF16, uint32_t LP, bool ALONG, uint32_t T>
__device__ __forceinline__ typename Frag<BF16>::type fragment(const lds_char *lds, uint32_t row0, uint32_t c0)
{
    const uint32_t lane = threadIdx.x & 63u, quad = lane >> 4, i = lane & 15u;
    if constexpr (ALONG) {
        const uint32_t row = row0 + i, piece = along_place<LP>(row, c0 / Width<BF16>::piece + quad);
        return *reinterpret_cast<const __attribute__((address_space(3))) typename Frag<BF16>::type *>(lds + row * (LP * 16u) + piece * 16u);
    } else if constexpr (BF16) {
        const uint32_t line = c0 + quad * 8u + (i >> 2), piece = across_place<true, T>(line, row0 / 8u + ((i & 3u) >> 1));
        const lds_char *at = lds + line * (T * 2u) + piece * 16u + (i & 1u) * 8u;            // four lines on: the same place in its line
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at);
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at + 4u * T * 2u));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
        const uint32_t line = c0 + quad * 4u, piece = across_place<false, T>(line, (row0 + i) / 4u);
        const lds_char *at = lds + line * (T * 4u) + piece * 16u + (i & 3u) * 4u;
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const __attribute__((address_space(3))) float *>(at + e * T * 4u);
        return v;
    }
}

// acc += what fragments of both sides make: element (n = 4 * (lane / 16) + reg, m = lane % 16) of each 16 x 16.
template <bool BF16, uint32_t FM, uint32_t FN>
__device__ __forceinline__ void products(f32x4 (&acc)[FM][FN], const typename Frag<BF16>::type (&m)[FM], const typename Frag<BF16>::type (&n)[FN])
{
    if constexpr (BF16) {
#pragma unroll
        for (uint32_t i = 0; i < FM; ++i) {
#pragma unroll
            for (uint32_t j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(n[j], m[i], acc[i][j], 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (uint32_t i = 0; i < FM; ++i) {
#pragma unroll
                for (uint32_t j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(n[j][e], m[i][e], acc[i][j], 0, 0, 0);
            }
        }
    }
}

// fp32: a sum of thousands of products in one accumulator loses more than the rest of the pass, so after every 512 of the contraction it is added to
// a second one and starts again: 4096 of them end up 23 + 3 roundings off (root of the count) in place of 64.  (That case: 5.8e-7 to 6.2e-7 off, relative, where it was 9.3e-7 and a library's products are 1.2e-6.)
constexpr uint32_t kFold = 512;
template <uint32_t FM, uint32_t FN> __device__ __forceinline__ void fold(f32x4 (&sum)[FM][FN], f32x4 (&acc)[FM][FN])
{
#pragma unroll
    for (uint32_t i = 0; i < FM; ++i) {
#pragma unroll
        for (uint32_t j = 0; j < FN; ++j) {
            sum[i][j] += acc[i][j];
            acc[i][j] = f32x4{};
        }
    }
}

// ---- any size, stride and alignment ------------------------------------------------------------------------------------------
// Tiles of T x T (FWD: half of the columns gate's, half up's), four waves, 32 of the contraction at a time; what is outside is zero in LDS.  The next 32 are asked for, in
// the widest accesses that the alignment allows, before these are multiplied, and go into the other of two buffers after that.  bf16, K = 8, 2048 rows,
// 2047 x 5503: forward 1918 us, dx 1829, weights 1343 (385 to 550 TFLOP/s; with tiles in the order of rows and replicas spread over all XCDs 2083, 3346, 2281);
// fp32, K = 4, 1023 rows, 1023 x 2815 488, 477, 447 (a chip at rest; behind others of their kind 8 % more).
constexpr uint32_t kDeep = 32;

// Eight elements of a side's tile next to each other in memory: element (i, c) of i < ni, c < nc is at p + i * stride + c (ALONG) or p + c * stride + i.  A thread has
// some of every 64 rows.  VEC: these are aligned, and ni or nc counts whole eights.
template <bool BF16, bool ALONG, bool VEC>
__device__ __forceinline__ Raw8<BF16> ask(const char *p, int64_t stride, int64_t i, int64_t ni, int64_t c, int64_t nc)
{
    const int64_t left = ALONG ? (i < ni ? nc - c : 0) : (c < nc ? ni - i : 0);
    const uint32_t n = left >= 8 ? 8u : left > 0 ? (uint32_t)left : 0u;
    const int64_t at = ALONG ? i * stride + c : c * stride + i;
    if (VEC && n) return load_raw<BF16, WIDE>(p, at, 8u);
    return load_raw<BF16, LOOSE>(p, at, VEC ? 0u : n);
}
template <bool ALONG> __device__ __forceinline__ uint32_t own_row() { return ALONG ? threadIdx.x >> 2 : (threadIdx.x & 7u) * 8u; }
template <bool ALONG> __device__ __forceinline__ uint32_t own_deep() { return ALONG ? (threadIdx.x & 3u) * 8u : threadIdx.x >> 3; }

// (fp32 with its second accumulator: two workgroups a CU, or the 128-tiles take 269 to 285 registers and a CU has one: that forward product 640 us.)
template <bool BF16, int FORM, bool VM, bool VN, uint32_t T>
__global__ __launch_bounds__(256, BF16 ? 1 : 2) void product_kernel(const ProductArgs a)
{
    constexpr uint32_t ES = Width<BF16>::bytes, LP = kDeep / Width<BF16>::piece, R = T / 64u, F = T / 32u, NT = FORM == FWD ? T / 2u : T, SIDE = T * LP * 16u;
    constexpr bool ALONG_M = FORM != DW, ALONG_N = FORM == FWD;
    __shared__ __attribute__((aligned(1024))) char mem[4u * SIDE];
    lds_char *lds = (lds_char *)mem;
    const uint32_t order = xcd_order(blockIdx.x, gridDim.x), k = uniform(order / a.tiles), tile = order - k * a.tiles;
    const int64_t rows = a.rows[k], cols = a.cols, wide = a.wide;
    const int64_t M = FORM == DW ? wide : rows, N = FORM == FWD ? wide : cols;
    const uint32_t tile_n = uniform(tile / a.tiles_m);                           // tiles next to each other have the same columns
    const int64_t m0 = (int64_t)(tile - tile_n * a.tiles_m) * T, n0 = (int64_t)tile_n * NT;
    if (m0 >= M) return;
    const uint32_t w = threadIdx.x >> 6, wm = w >> 1, wn = w & 1u;
    f32x4 acc[F][F] = {}, sum[F][F] = {};
    const char *dg = a.dg + (uint64_t)a.first[k] * a.pitch * ES, *du = a.du + (uint64_t)a.first[k] * a.pitch * ES;
    const char *x = a.x.p + k * a.x.rs * (int64_t)ES;
    const int64_t deep = FORM == FWD ? cols : FORM == DX ? wide : rows;
    Raw8<BF16> rm[R], rn[R];
    auto ask_both = [&](int half, int64_t c0) {
        const int64_t cm = c0 + own_deep<ALONG_M>(), cn = c0 + own_deep<ALONG_N>();
#pragma unroll
        for (uint32_t q = 0; q < R; ++q) {
            const uint32_t im = q * 64u + own_row<ALONG_M>(), in = q * 64u + own_row<ALONG_N>();
            if constexpr (FORM == FWD) {
                rm[q] = ask<BF16, true, VM>(x, a.x.ss, m0 + im, M, cm, deep);
                rn[q] = ask<BF16, true, VN>(in < T / 2u ? a.gate[k] : a.up[k], cols, n0 + in % (T / 2u), N, cn, deep);
            } else if constexpr (FORM == DX) {
                rm[q] = ask<BF16, true, VM>(half ? du : dg, a.pitch, m0 + im, M, cm, deep);
                rn[q] = ask<BF16, false, VN>(half ? a.up[k] : a.gate[k], cols, n0 + in, N, cn, deep);
            } else {
                rm[q] = ask<BF16, false, VM>(blockIdx.z ? du : dg, a.pitch, m0 + im, M, cm, deep);
                rn[q] = ask<BF16, false, VN>(x, a.x.ss, n0 + in, N, cn, deep);
            }
        }
    };
    auto put = [&](auto along, lds_char *to, const Raw8<BF16> &r, uint32_t q) {
        constexpr bool ALONG = decltype(along)::value;
        const uint32_t row = q * 64u + own_row<ALONG>(), c = own_deep<ALONG>();
#pragma unroll
        for (uint32_t i = 0; i < 8u / Width<BF16>::piece; ++i) {
            uint32_t at;
            if constexpr (ALONG) at = row * LP + along_place<LP>(row, c / Width<BF16>::piece + i);
            else at = c * (T / Width<BF16>::piece) + across_place<BF16, T>(c, row / Width<BF16>::piece + i);
            *reinterpret_cast<__attribute__((address_space(3))) u32x4 *>(to + at * 16u) = r.w[i];
        }
    };
    auto put_both = [&](uint32_t buffer) {
#pragma unroll
        for (uint32_t q = 0; q < R; ++q) {
            put(std::bool_constant<ALONG_M>{}, lds + buffer * 2u * SIDE, rm[q], q);
            put(std::bool_constant<ALONG_N>{}, lds + buffer * 2u * SIDE + SIDE, rn[q], q);
        }
    };
    // column of C that a wave's fragment j of the n side starts with (FWD: j < F / 2 gate's, then up's), and where it is among the tile's lines in LDS
    auto n_col = [&](uint32_t j) { return FORM == FWD ? wn * (T / 4u) + j % (F / 2u) * 16u : wn * (T / 2u) + j * 16u; };
    const int64_t steps1 = (deep + kDeep - 1) / kDeep, steps = FORM == DX ? 2 * steps1 : steps1;
    if (steps) {
        ask_both(0, 0);
        put_both(0u);
    }
    for (int64_t s = 0; s < steps; ++s) {
        __syncthreads();
        if (s + 1 < steps) ask_both(FORM == DX && s + 1 >= steps1, (FORM == DX && s + 1 >= steps1 ? s + 1 - steps1 : s + 1) * kDeep);
        const lds_char *side = lds + ((uint32_t)s & 1u) * 2u * SIDE;
#pragma unroll
        for (uint32_t c = 0; c < kDeep; c += Width<BF16>::deep) {
            typename Frag<BF16>::type m[F], n[F];
#pragma unroll
            for (uint32_t i = 0; i < F; ++i) {
                m[i] = fragment<BF16, LP, ALONG_M, T>(side, wm * (T / 2u) + i * 16u, c);
                n[i] = fragment<BF16, LP, ALONG_N, T>(side + SIDE, n_col(i) + (FORM == FWD && i >= F / 2u ? T / 2u : 0u), c);
            }
            products<BF16, F, F>(acc, m, n);
        }
        if (s + 1 < steps) put_both(((uint32_t)s + 1u) & 1u);
        if constexpr (!BF16) {
            if ((uint32_t)s % (kFold / kDeep) == kFold / kDeep - 1u) fold<F, F>(sum, acc);
        }
    }
    if constexpr (!BF16) {
        fold<F, F>(sum, acc);
#pragma unroll
        for (uint32_t i = 0; i < F; ++i) {
#pragma unroll
            for (uint32_t j = 0; j < F; ++j) acc[i][j] = sum[i][j];
        }
    }
    const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
    for (uint32_t i = 0; i < F; ++i) {
#pragma unroll
        for (uint32_t j = 0; j < (FORM == FWD ? F / 2u : F); ++j) {
            const int64_t m = m0 + wm * (T / 2u) + i * 16 + (lane & 15u), n1 = n0 + n_col(j) + (lane >> 4) * 4u;
            if (m >= M) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t n = n1 + e;
                if (n >= N) continue;
                if constexpr (FORM == FWD) {
                    const float g = acc[i][j][e], u = acc[i][j + F / 2u][e];
                    store1<BF16>(a.a.p, k * a.a.rs + m * a.a.ss + n, activation<BF16>(a.act, g).f * u);
                    if (a.g.p) {
                        store1<BF16>(a.g.p, k * a.g.rs + m * a.g.ss + n, g);
                        store1<BF16>(a.u.p, k * a.u.rs + m * a.u.ss + n, u);
                    }
                } else if constexpr (FORM == DX) {
                    store1<BF16>(a.a.p, k * a.a.rs + m * a.a.ss + n, acc[i][j][e]);
                } else {
                    char *grad = blockIdx.z ? a.up[k] : a.gate[k];
                    float v = acc[i][j][e];
                    if (a.accumulate) v += load1<BF16>(grad, m * cols + n);
                    store1<BF16>(grad, m * cols + n, v);
                }
            }
        }
    }
}

// ---- aligned ------------------------------------------------------------------------------------------------------------------------
// Bound by the matrix cores and what feeds them.  bf16, K = 8, 2048 rows, 2048 x 5504: forward 802 us (920 TFLOP/s), dx 675 (1095), weights 722 (1023), where a library's plain product
// of such sizes reaches 870 to 1070; of the forward pass, 526 are the products with LDS as it is, 500 the loads without the products, and 170 its three outputs.
// fp32, K = 4, 1024 rows, 1024 x 2816: 464, 412 and 435 us (102 to 115 TFLOP/s; a library 140 on 4096 x 4096 x 4096); the second accumulator takes 2 % of it.  A few rows: the weights' bytes, 361 MB in 59 to 70 us.
//
// A workgroup makes TM x TN of C, wave by wave, and takes the contraction a step (LP pieces of 16 bytes) at a time through NS
// buffers in LDS: while the waves multiply one, the next ones are on their way from memory straight into the others.
// What is outside is asked for beyond the end of a buffer resource, which gives zeros.

// A tile's place and how far what may be read reaches from there: T lines along, or a step's lines across.
struct Side {
    const char *p;               // of the tile's first element
    int64_t bytes;               // from there to the end of what is there
    int64_t stride;              // bytes from one line to the next
};

__device__ __forceinline__ uint32_t records(int64_t bytes) { return bytes <= 0 ? 0u : bytes > 0xfffffff0ll ? 0xfffffff0u : (uint32_t)bytes; }

// The next step of the contraction into LDS.  left: how much of it is still there (ALONG: beyond it the line goes on with something else).
template <bool BF16, uint32_t LP, bool ALONG, uint32_t T, uint32_t THREADS, bool HINT = false>
__device__ __forceinline__ void fetch(lds_char *lds, const Side &s, int64_t left)
{
    constexpr uint32_t PIECES = T * LP, LINE = ALONG ? LP : T / Width<BF16>::piece;
    static_assert(PIECES % 64u == 0, "whole waves");
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)s.p, 0, records(s.bytes), 0x00020000);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (uint32_t i = 0; i < (PIECES + THREADS - 1u) / THREADS; ++i) {
        if ((i + 1u) * THREADS > PIECES && i * THREADS + wave * 64u >= PIECES) break;
        const uint32_t at = i * THREADS + threadIdx.x, line = at / LINE;
        uint32_t piece;
        if constexpr (ALONG) piece = along_place<LP>(line, at % LINE);
        else piece = across_place<BF16, T>(line, at % LINE);
        uint32_t off = line * (uint32_t)s.stride + piece * 16u;
        if (ALONG && (int64_t)(piece * Width<BF16>::piece) >= left) off = 0xfffffff0u;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(lds + (i * THREADS + wave * 64u) * 16u), 16, off, 0, 0, HINT ? 2 : 0);
    }
}

// HINT: the weights are read with the streaming hint.
template <bool BF16, int FORM, uint32_t TM, uint32_t TN, uint32_t WM, uint32_t WN, uint32_t LP, uint32_t NS, bool HINT> struct Big {
    static constexpr uint32_t threads = 64u * WM * WN;
    static constexpr bool along_m = FORM != DW, along_n = FORM == FWD;
    static constexpr uint32_t FM = TM / WM / 16u, FN = TN / WN / 16u;           // fragments of a wave
    static constexpr uint32_t bytes = (TM + TN) * LP * 16u, n_at = TM * LP * 16u;            // of a buffer, and where the n side is in it
    static constexpr uint32_t step = LP * Width<BF16>::piece;                  // elements of the contraction
    static constexpr uint32_t cols_out = TN / WN / (FORM == FWD ? 2u : 1u);    // columns of C that a wave has
    static constexpr uint32_t part_rows = FM > 4u ? 64u : FM * 16u, part_pitch = TN / WN + 4u;     // of it, on its way out, in fp32
    static constexpr uint32_t out_bytes = WM * WN * part_rows * part_pitch * 4u;
    static constexpr uint32_t lds = NS * bytes > out_bytes ? NS * bytes : out_bytes;
    // loads a step of a wave: whole rounds, and one more of the first `more` waves where a side has less than a round
    static constexpr uint32_t sides[3] = {TM * LP, FORM == FWD ? TN / 2u * LP : TN * LP, FORM == FWD ? TN / 2u * LP : 0u};
    static constexpr uint32_t rounds = sides[0] / threads + sides[1] / threads + sides[2] / threads;
    static constexpr uint32_t more = sides[0] % threads / 64u;
    static_assert(sides[1] % threads == 0 && sides[2] % threads == 0 && sides[0] % 64u == 0, "whole waves");
    static_assert(lds <= 163840u && (NS - 2u) * (rounds + 1u) < 64u, "LDS; what the counter of loads holds");

    static __device__ __forceinline__ void fetch_both(lds_char *lds, const Side &m, const Side &n, const Side &n2, int64_t left)
    {
        fetch<BF16, LP, along_m, TM, threads>(lds, m, left);
        if constexpr (FORM == FWD) {
            fetch<BF16, LP, true, TN / 2u, threads, HINT>(lds + n_at, n, left);
            fetch<BF16, LP, true, TN / 2u, threads, HINT>(lds + n_at + TN / 2u * LP * 16u, n2, left);
        } else fetch<BF16, LP, along_n, TN, threads, HINT>(lds + n_at, n, left);
    }
    // row of the n side's fragment j: a wave of FWD has the same columns of gate and up
    static __device__ __forceinline__ uint32_t n_row(uint32_t wn, uint32_t j)
    {
        if constexpr (FORM == FWD) return (j >= FN / 2u ? TN / 2u + (j - FN / 2u) * 16u : j * 16u) + wn * (TN / WN / 2u);
        else return wn * (TN / WN) + j * 16u;
    }
    static __device__ __forceinline__ void multiply(f32x4 (&acc)[FM][FN], const lds_char *lds, uint32_t wm, uint32_t wn)
    {
#pragma unroll
        for (uint32_t c = 0; c < step; c += Width<BF16>::deep) {
            typename Frag<BF16>::type m[FM], n[FN];
#pragma unroll
            for (uint32_t j = 0; j < FN; ++j) n[j] = fragment<BF16, LP, along_n, TN>(lds + n_at, n_row(wn, j), c);
#pragma unroll
            for (uint32_t i = 0; i < FM; ++i) m[i] = fragment<BF16, LP, along_m, TM>(lds, wm * (TM / WM) + i * 16u, c);
            products<BF16, FM, FN>(acc, m, n);
            // The order of a fragment's worth: enough reads to begin with, then one after every FN products, four rows of fragments ahead.
            if constexpr (BF16 && FM > 4u) {
                constexpr int NB = along_n ? 1 : 2, MB = along_m ? 1 : 2;
                __builtin_amdgcn_sched_group_barrier(0x100, FN * NB + 4 * MB, 0);
#pragma unroll
                for (uint32_t i = 4; i < FM; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, FN, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, MB, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, 4 * FN, 0);
            }
        }
    }
    // The step in cur is there once no more than the loads of the NS - 2 steps behind it are on their way; and every wave is done with the step before.
    static __device__ __forceinline__ void arrive(uint32_t wave)
    {
        if (more && wave < more) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NS - 2u) * (rounds + 1u)) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NS - 2u) * rounds) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
    // cur is read while far is written: told apart by restrict, or every read would wait for all loads into LDS.  One place in the code for both, also for
    // the first loads, which nothing is multiplied beside, or they would not be told apart.
    static __device__ __forceinline__ void turn(f32x4 (&acc)[FM][FN], const lds_char *__restrict__ cur, lds_char *__restrict__ far, const Side &m,
                                                const Side &n, const Side &n2, int64_t left, bool ready, uint32_t wm, uint32_t wn)
    {
        fetch_both(far, m, n, n2, left);
        __builtin_amdgcn_sched_barrier(0);
        if (ready) multiply(acc, cur, wm, wn);
    }
};

// Eight elements or, where they may not be stored at once, as many as there are.
template <bool BF16> __device__ __forceinline__ void store_some(char *p, int64_t at, bool at_once, uint32_t there, const float (&v)[8])
{
    if (at_once) store8<BF16, WIDE>(p, at, 8u, v);
    else store8<BF16, LOOSE>(p, at, there, v);
}

struct TileMap {
    uint32_t first[65];          // tiles of the replicas before, and of all
    uint32_t replicas;
    uint32_t splits, per_split;  // workgroups that share a tile's contraction (DX), and the steps of each
    float *part;                 // more than one: what each of them has, [splits][rows of all replicas][cols]
    uint64_t part_stride;        // elements from one split to the next
};

template <bool BF16, int FORM, uint32_t TM, uint32_t TN, uint32_t WM, uint32_t WN, uint32_t LP, uint32_t NS, bool HINT>
__global__ __launch_bounds__((Big<BF16, FORM, TM, TN, WM, WN, LP, NS, HINT>::threads)) void big_product_kernel(const ProductArgs a, const TileMap map)
{
    using S = Big<BF16, FORM, TM, TN, WM, WN, LP, NS, HINT>;
    constexpr int ES = Width<BF16>::bytes;
    constexpr uint32_t STEP = S::step;
    __shared__ __attribute__((aligned(1024))) char lds_mem[S::lds];
    lds_char *lds = (lds_char *)lds_mem;
    const uint32_t order = xcd_order(blockIdx.x, gridDim.x);
    const uint32_t tiles = map.first[map.replicas];
    const uint32_t split = FORM == DX ? uniform(order / tiles) : 0u, id = FORM == DX ? order - split * tiles : order;
    uint32_t k = 0;
    for (uint32_t half = 32u; half; half >>= 1)
        if (k + half < map.replicas && map.first[k + half] <= id) k += half;
    uint32_t tile = id - map.first[k];
    const uint32_t rows = a.rows[k], cols = a.cols, wide = a.wide;
    const uint32_t M = FORM == DW ? wide : rows, N = FORM == FWD ? wide : cols;
    const uint32_t tm = (M + TM - 1u) / TM;
    const bool second = FORM == DW && tile >= tm * ((N + TN - 1u) / TN);         // DW: first all of the gate's gradient, then up's
    if (second) tile -= tm * ((N + TN - 1u) / TN);
    constexpr uint32_t NT = FORM == FWD ? TN / 2u : TN;                          // columns of C
    const uint32_t tile_n = uniform(tile / tm), tile_m = tile - tile_n * tm;
    const int64_t m0 = (int64_t)tile_m * TM, n0 = (int64_t)tile_n * NT;
    const uint32_t w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w / WN, wn = w % WN;
    const int64_t pitch = (int64_t)a.pitch * ES, width = (int64_t)cols * ES, xs = a.x.ss * ES;
    const uint64_t first = (uint64_t)a.first[k] * pitch;
    const char *x = a.x.p + k * a.x.rs * ES;
    Side m, n, n2;
    int64_t deep;
    if constexpr (FORM == FWD) {
        deep = cols;
        m = Side{x + m0 * xs, ((int64_t)rows - 1 - m0) * xs + width, xs};
        n = Side{a.gate[k] + n0 * width, (wide - n0) * width, width};
        n2 = Side{a.up[k] + n0 * width, (wide - n0) * width, width};
    } else if constexpr (FORM == DX) {
        deep = a.pitch;
        m = Side{a.dg + first + m0 * pitch, (rows - m0) * pitch, pitch};
        n = Side{a.gate[k] + n0 * ES, wide * width - n0 * ES, width};
        n2 = n;
    } else {
        deep = rows;
        m = Side{(second ? a.du : a.dg) + first + m0 * ES, rows * pitch - m0 * ES, pitch};
        n = Side{x + n0 * ES, ((int64_t)rows - 1) * xs + width - n0 * ES, xs};
        n2 = n;
    }
    const uint32_t steps1 = (uint32_t)((deep + STEP - 1) / STEP), all = FORM == DX ? 2u * steps1 : steps1;
    const uint32_t begin = FORM == DX ? split * map.per_split : 0u, end = FORM == DX && begin + map.per_split < all ? begin + map.per_split : all;
    const int64_t to_du = FORM == DX ? a.du - a.dg : 0, to_up = FORM == DX ? a.up[k] - a.gate[k] : 0;
    f32x4 acc[S::FM][S::FN] = {}, sum[S::FM][S::FN] = {};
    // The sides of the step that is asked for next.  DX goes through the first pair and then through the second; beyond the last step there is nothing to read.
    const int64_t on_m = S::along_m ? LP * 16 : STEP * m.stride, on_n = S::along_n ? LP * 16 : STEP * n.stride;
    const Side m_first = m, n_first = n;
    int64_t left = deep;
    auto move = [&](int64_t steps) {
        m.p += steps * on_m, m.bytes -= steps * on_m;
        n.p += steps * on_n, n.bytes -= steps * on_n;
        n2.p += steps * on_n, n2.bytes -= steps * on_n;
        left -= steps * STEP;
    };
    auto second_pair = [&] {
        m = m_first, n = n_first, left = deep;
        m.p += to_du, n.p += to_up;
    };
    if (FORM == DX && begin >= steps1) {
        second_pair();
        move(begin - steps1);
    } else move(begin);
    const uint32_t steps = end - begin;
    if (!steps) m.bytes = n.bytes = n2.bytes = 0;     // no rows at all: what is asked for in any case is zeros
    uint32_t into = 0u, cur = 0u;                     // buffers: of the step asked for next, and of the step that is multiplied next
    for (uint32_t t = 0; t < steps + NS - 1u; ++t) {              // asks for the t-th step, and multiplies the one NS - 1 before
        const bool ready = t >= NS - 1u;
        if (ready) S::arrive(w);
        S::turn(acc, lds + cur * S::bytes, lds + into * S::bytes, m, n, n2, left, ready, wm, wn);
        move(1);
        if (FORM == DX && begin + t + 1u == steps1) second_pair();
        if (t + 1u >= steps) m.bytes = n.bytes = n2.bytes = 0;
        into = into + 1u == NS ? 0u : into + 1u;
        if (ready) cur = cur + 1u == NS ? 0u : cur + 1u;
        if constexpr (!BF16) {
            if (t % (kFold / STEP) == 0u) fold<S::FM, S::FN>(sum, acc);
        }
    }
    if constexpr (!BF16) {
        fold<S::FM, S::FN>(sum, acc);
#pragma unroll
        for (uint32_t i = 0; i < S::FM; ++i) {
#pragma unroll
            for (uint32_t j = 0; j < S::FN; ++j) acc[i][j] = sum[i][j];
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // C through LDS, each wave in a part of its own, so that a lane has eight columns next to each other and the activation's code is there once.
    __syncthreads();
    float *mine = reinterpret_cast<float *>(lds_mem) + w * (S::part_rows * S::part_pitch);
    const uint32_t lane = threadIdx.x & 63u;
    constexpr uint32_t LANES = S::cols_out / 8u, ROWS = 64u / LANES;              // lanes a row, rows at a time
#pragma unroll
    for (uint32_t i0 = 0; i0 < S::FM; i0 += S::part_rows / 16u) {
#pragma unroll
        for (uint32_t i = 0; i < S::part_rows / 16u; ++i) {
#pragma unroll
            for (uint32_t j = 0; j < S::FN; ++j)
                *reinterpret_cast<f32x4 *>(mine + (i * 16u + (lane & 15u)) * S::part_pitch + j * 16u + (lane >> 4) * 4u) = acc[i0 + i][j];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int64_t row0 = m0 + wm * (TM / WM) + i0 * 16u, col = n0 + wn * S::cols_out + lane % LANES * 8u;
#pragma unroll 1
        for (uint32_t r = lane / LANES; r < S::part_rows; r += ROWS) {
            const int64_t row = row0 + r;
            if (row >= M || col >= N) break;
            const float *from = mine + r * S::part_pitch + lane % LANES * 8u;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = from[e];
            const uint32_t there = (uint32_t)(N - col < 8 ? N - col : 8);
            const bool at_once = a.wide_out && there == 8u;
            if constexpr (FORM == FWD) {
                float u[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = from[S::cols_out + e];
                if (a.g.p) {
                    store_some<BF16>(a.g.p, k * a.g.rs + row * a.g.ss + col, at_once, there, v);
                    store_some<BF16>(a.u.p, k * a.u.rs + row * a.u.ss + col, at_once, there, u);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = activation<BF16>(a.act, v[e]).f * u[e];
                store_some<BF16>(a.a.p, k * a.a.rs + row * a.a.ss + col, at_once, there, v);
            } else if constexpr (FORM == DX) {
                if (map.splits > 1u) store8<false, WIDE>((char *)(map.part + split * map.part_stride), (int64_t)(a.first[k] + row) * cols + col, 8u, v);
                else store_some<BF16>(a.a.p, k * a.a.rs + row * a.a.ss + col, at_once, there, v);
            } else {                                  // cols counts whole eights
                char *grad = second ? a.up[k] : a.gate[k];
                if (a.accumulate) {
                    float old[8];
                    load8<BF16, WIDE>(old, grad, row * cols + col, 8u);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += old[e];
                }
                store8<BF16, WIDE>(grad, row * cols + col, 8u, v);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// dx from the parts of a contraction that several workgroups shared, added in their order.
struct JoinRowsArgs {
    RowsAt a;
    const float *part;
    uint64_t part_stride;
    uint32_t splits, cols;       // cols counts whole eights
    int32_t wide_out;
    uint32_t rows[64];
    uint32_t first[64];
};
template <bool BF16>
__global__ __launch_bounds__(256) void join_rows_kernel(const JoinRowsArgs a)
{
    const uint32_t k = blockIdx.y, rows = a.rows[k], groups = a.cols / 8u;
    for (uint32_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (uint32_t g = threadIdx.x; g < groups; g += 256u) {
            float sum[8], v[8];
            const char *from = (const char *)a.part;
            const int64_t at = (int64_t)(a.first[k] + r) * a.cols + g * 8u;
            load8<false, WIDE>(sum, from, at, 8u);
#pragma unroll 4
            for (uint32_t s = 1; s < a.splits; ++s) {
                load8<false, WIDE>(v, from, at + (int64_t)(s * a.part_stride), 8u);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += v[e];
            }
            store_some<BF16>(a.a.p, k * a.a.rs + (int64_t)r * a.a.ss + g * 8u, a.wide_out, 8u, sum);
        }
}

// ---- bf16, aligned, a few rows ------------------------------------------------------------------------------------------------------
// DW, bound by the gradients' bytes: up to 32 rows are one step of the contraction.  A workgroup has 256 columns of the hidden side, 16 at a time, and 256 of
// the model's, 64 a wave, and both sides' rows in LDS as they are in memory.  C goes through LDS once more, so that a store writes whole lines of 128 bytes:
// with the streaming hint on halves of lines, 180 MB of gradients a weight (K = 8, 2048 x 5504) took 105 us in place of 68, on quarters 225.
constexpr uint32_t kFewRows = 32;
template <bool ACCUMULATE, int ACCESS>
__global__ __launch_bounds__(256) void few_rows_weights_kernel(const ProductArgs a)
{
    constexpr uint32_t T = 256;
    __shared__ __attribute__((aligned(1024))) char mem[2][kFewRows * T * 2u];
    __shared__ float out[4][16][68];
    lds_char *hidden = (lds_char *)mem[0], *model = (lds_char *)mem[1];
    const uint32_t k = blockIdx.y, rows = a.rows[k], cols = a.cols, wide = a.wide;
    const uint32_t tn = (cols + T - 1u) / T, d0 = blockIdx.x % tn * T, f0 = blockIdx.x / tn * T;
    const char *from = (blockIdx.z ? a.du : a.dg) + (uint64_t)a.first[k] * a.pitch * 2u, *x = a.x.p + k * a.x.rs * 2;
    char *grad = blockIdx.z ? a.up[k] : a.gate[k];
#pragma unroll
    for (uint32_t t = threadIdx.x; t < kFewRows * T / 8u; t += 256u) {
        const uint32_t line = t / (T / 8u), c = t % (T / 8u) * 8u, at = line * (T * 2u) + across_place<true, T>(line, c / 8u) * 16u;
        u32x4 h{}, m{};
        if (line < rows && f0 + c < a.pitch) h = *as_global<u32x4>(from + ((uint64_t)line * a.pitch + f0 + c) * 2u);
        if (line < rows && d0 + c < cols) m = *as_global<u32x4>(x + ((int64_t)line * a.x.ss + d0 + c) * 2);
        *reinterpret_cast<__attribute__((address_space(3))) u32x4 *>(hidden + at) = h;
        *reinterpret_cast<__attribute__((address_space(3))) u32x4 *>(model + at) = m;
    }
    __syncthreads();
    const uint32_t lane = threadIdx.x & 63u, w = threadIdx.x >> 6, col = d0 + w * 64u + (lane & 7u) * 8u;
    bf16x8 n[4];
#pragma unroll
    for (uint32_t j = 0; j < 4u; ++j) n[j] = fragment<true, 8, false, T>(model, w * 64u + j * 16u, 0);
#pragma unroll 2
    for (uint32_t i = 0; i < T; i += 16u) {
        if (f0 + i >= wide) break;
        const bf16x8 m = fragment<true, 8, false, T>(hidden, i, 0);
#pragma unroll
        for (uint32_t j = 0; j < 4u; ++j)
            *reinterpret_cast<f32x4 *>(&out[w][lane & 15u][j * 16u + (lane >> 4) * 4u]) = __builtin_amdgcn_mfma_f32_16x16x32_bf16(n[j], m, f32x4{}, 0, 0, 0);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (uint32_t r = lane >> 3; r < 16u; r += 8u) {
            if (f0 + i + r >= wide || col >= cols) continue;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = out[w][r][(lane & 7u) * 8u + e];
            const int64_t at = (int64_t)(f0 + i + r) * cols + col;
            if constexpr (ACCUMULATE) {
                float old[8];
                load8<true, ACCESS>(old, grad, at, 8u);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += old[e];
            }
            store8<true, ACCESS>(grad, at, 8u, v);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

} // namespace lasgd
