// Gradient norms and clipping: device code.
//
// Each replica (the paper's worker) has a norm of its own over its whole parameter list,
//     n_k = sqrt(sum_t sum_i g[k][t][i]^2),    c_k = min(1, max_norm / (n_k + 1e-6)),
// and its gradients count times c_k.  Squares and sums are in fp64 from the elements on: 1e30 or 1e-30 neither overflows nor
// vanishes in its square, and the sum is finite exactly when every element is.  Everything is added in an order that the launch shape fixes, so
// the same call on the same gradients gives the same bits.
//
// Bound by HBM: 2 flop per 2 or 4 bytes; the vector units do 64-bit additions ten times as fast as the elements arrive.
#pragma once
#include "lasgd_kernels.hip.h"

namespace lasgd {

constexpr uint32_t kNormThreads = 256;

struct NormArgs {
    double *part;           // [K][parts] a workgroup's sum of squares
    uint32_t parts;         // workgroups a replica
    uint64_t mask;          // replicas that take part
    uint32_t count;         // how many they are
    Clip *clip;             // [K] what comes of it, or NULL
    float *norms;           // [K] the caller's, or NULL
    float max_norm;
    int32_t skip_nonfinite;
};

__device__ __forceinline__ void add_squares(double &acc, float4 g)
{
    acc = __builtin_fma((double)g.x, (double)g.x, acc);
    acc = __builtin_fma((double)g.y, (double)g.y, acc);
    acc = __builtin_fma((double)g.z, (double)g.z, acc);
    acc = __builtin_fma((double)g.w, (double)g.w, acc);
}

// The sum over a workgroup, in thread 0.
__device__ __forceinline__ double block_sum(double acc)
{
    __shared__ double wave[kNormThreads / 64u];
#pragma unroll
    for (int d = 32; d; d >>= 1) acc += __shfl_down(acc, d, 64);
    if ((threadIdx.x & 63u) == 0u) wave[threadIdx.x >> 6] = acc;
    __syncthreads();
    if (threadIdx.x == 0u)
        for (uint32_t w = 1; w < kNormThreads / 64u; ++w) acc += wave[w];
    return acc;
}

// What comes of replica k's sum of squares.
__device__ __forceinline__ void finish_norm(const NormArgs &n, uint32_t k, double sum)
{
    const double norm = __builtin_sqrt(sum);
    if (n.norms) *as_global<float>(n.norms + k) = (float)norm;
    if (n.clip) {
        const double c = (double)n.max_norm / (norm + 1e-6);
        const bool finite = norm <= 1.7976931348623157e308;
        n.clip[k].c = c >= 1.0 ? 1.f : (float)c;               // a NaN stays one
        n.clip[k].skip = n.skip_nonfinite && !finite ? 1u : 0u;
    }
}

template <bool BF16>
__device__ __forceinline__ float4 grad_at(const char *g, uint32_t e, uint32_t n)
{
    if (n == 4u) return BF16 ? widen4(ld2<0>(reinterpret_cast<const uint16_t *>(g) + e)) : ld4<0>(reinterpret_cast<const float *>(g) + e);
    float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
    LASGD_FOR4(if (c < 3 && (uint32_t)c < n) comp(r, c) = BF16 ? bf16_widen(as_global<uint16_t>(g)[e + c]) : as_global<float>(g)[e + c];)
    return r;
}

// Sums of squares of one replica's gradients (blockIdx.y: of which), tile by tile.
template <bool BF16>
__global__ __launch_bounds__(256) void grad_norm_kernel(const ApplyArgs a, const NormArgs n)
{
    const uint32_t lane = threadIdx.x & 63u, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t k = n.count == a.K ? blockIdx.y : nth_bit(n.mask, blockIdx.y);
    double acc = 0.0;
    for (uint32_t tile = blockIdx.x * 4u + w; tile < a.ntiles; tile += n.parts * 4u) {
        const uint32_t tensor = tensor_of(a, tile);
        const Record rec = load_record(a, k, tensor);
        const Tile t = locate(a, rec, tile, tensor, 256u);
        const char *g = reinterpret_cast<const char *>(rec.g) + t.toff * (BF16 ? 2 : 4);
        const uint32_t e = lane * 4u;
        add_squares(acc, grad_at<BF16>(g, e, lane_elems<false>(e, t.count)));
    }
    acc = block_sum(acc);
    if (threadIdx.x == 0u) n.part[(size_t)k * n.parts + blockIdx.x] = acc;
}

// The same of one vector: the mean gradient, `nvec` groups of four elements.
__global__ __launch_bounds__(256) void flat_norm_kernel(const float *v, uint64_t nvec, const NormArgs n)
{
    double acc = 0.0;
    for (uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x; i < nvec; i += (uint64_t)n.parts * 256u) add_squares(acc, ld4<0>(v + i * 4u));
    acc = block_sum(acc);
    if (threadIdx.x == 0u) n.part[blockIdx.x] = acc;
}

// One workgroup a replica: the parts in order.
__global__ __launch_bounds__(256) void finish_norm_kernel(const NormArgs n, const uint32_t all)
{
    const uint32_t k = n.count == all ? blockIdx.x : nth_bit(n.mask, blockIdx.x);
    double acc = 0.0;
    for (uint32_t i = threadIdx.x; i < n.parts; i += 256u) acc += n.part[(size_t)k * n.parts + i];
    acc = block_sum(acc);
    if (threadIdx.x == 0u) finish_norm(n, k, acc);
}

// Clipping in place: gradients times c, rounded once to the storage type, where c is not 1.
template <bool BF16>
__global__ __launch_bounds__(64) void scale_grads_kernel(const ApplyArgs a, const NormArgs n)
{
    const uint32_t e = threadIdx.x * 4u;
    const uint32_t k = n.count == a.K ? blockIdx.y : nth_bit(n.mask, blockIdx.y);
    const LASGD_CONST_AS Clip *cl = as_const(n.clip) + k;
    const float scale = cl->c;
    if (cl->skip || scale == 1.f) return;
    for (uint32_t tile = blockIdx.x; tile < a.ntiles; tile += gridDim.x) {
        const uint32_t tensor = tensor_of(a, tile);
        const Record rec = load_record(a, k, tensor);
        const Tile t = locate(a, rec, tile, tensor, 256u);
        char *g = reinterpret_cast<char *>(rec.g) + t.toff * (BF16 ? 2 : 4);
        const uint32_t m = lane_elems<false>(e, t.count);
        float4 v = grad_at<BF16>(g, e, m);
        v = make_float4(v.x * scale, v.y * scale, v.z * scale, v.w * scale);
        if (m == 4u) {
            if constexpr (BF16) st2<0>(reinterpret_cast<uint16_t *>(g) + e, round4(v));
            else st4<0>(reinterpret_cast<float *>(g) + e, v);
        } else {
            LASGD_FOR4(if (c < 3 && (uint32_t)c < m) {
                if constexpr (BF16) as_global<uint16_t>(g)[e + c] = (uint16_t)bf16_round(compv(v, c));
                else as_global<float>(g)[e + c] = compv(v, c);
            })
        }
    }
}

} // namespace lasgd
