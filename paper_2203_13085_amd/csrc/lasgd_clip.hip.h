// Gradient norms and clipping: device code.
//
// Each replica (the paper's worker) has a norm of its own over its whole parameter list,
//     n_k = sqrt(sum_t sum_i g[k][t][i]^2),    c_k = min(1, max_norm / (n_k + 1e-6)), 1 where max_norm is infinite,
// and its gradients count times c_k.  Squares and sums are in fp64 from the elements on: 1e30 or 1e-30 neither overflows nor
// vanishes in its square, and the sum is finite exactly when every element is.  Everything is added in an order that the launch shape fixes, so
// the same call on the same gradients gives the same bits.
//
// Bound by HBM: 2 flop per 2 or 4 bytes; the vector units do 64-bit additions ten times as fast as the elements arrive.
#pragma once
#include "lasgd_kernels.hip.h"
#include "../../include/lasgd.h"

namespace lasgd {

constexpr uint32_t kNormThreads = 1024, kNormWaves = kNormThreads / 64u;
constexpr uint32_t kNormRun = 4u * kNormWaves;      // tiles a workgroup takes at a time, four a wave
static_assert(kNormRun == 1u << kBlockShift, "a run is a block of the lookup table: one entry says what is in it");
constexpr uint32_t kArriveStride = 32;          // words: 128 bytes

struct NormArgs {
    double *part;           // [K][stride] a workgroup's sum of squares
    uint32_t *arrived;      // [K][kArriveStride] how many of them are there
    uint32_t stride, parts; // workgroups a replica, at most and in this call
    uint64_t mask;          // replicas that take part
    uint32_t count;         // how many they are
    Clip *clip;             // [K] what comes of it, or NULL
    float *norms;           // [K] the caller's, or NULL
    float max_norm;
    int32_t skip_nonfinite;
    FastDiv by_runs;        // division by a replica's runs of tiles (scale_grads_kernel)
};

__device__ __forceinline__ void add_squares(double &acc, float4 g)
{
    acc = __builtin_fma((double)g.x, (double)g.x, acc);
    acc = __builtin_fma((double)g.y, (double)g.y, acc);
    acc = __builtin_fma((double)g.z, (double)g.z, acc);
    acc = __builtin_fma((double)g.w, (double)g.w, acc);
}

// Into two sums, as in a run of one tensor (fp32).
__device__ __forceinline__ void add_squares(double &a0, double &a1, float4 g)
{
    a0 = __builtin_fma((double)g.x, (double)g.x, a0);
    a1 = __builtin_fma((double)g.y, (double)g.y, a1);
    a0 = __builtin_fma((double)g.z, (double)g.z, a0);
    a1 = __builtin_fma((double)g.w, (double)g.w, a1);
}

// The sum over a wave, in its first lane.
__device__ __forceinline__ double wave_sum(double acc)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) acc += __shfl_down(acc, d, 64);
    return acc;
}

// The sum over a workgroup of W waves, in thread 0.
template <uint32_t W> __device__ __forceinline__ double block_sum(double acc)
{
    __shared__ double wave[W];
    acc = wave_sum(acc);
    if ((threadIdx.x & 63u) == 0u) wave[threadIdx.x >> 6] = acc;
    __syncthreads();
    if (threadIdx.x == 0u) {
#pragma unroll
        for (uint32_t w = 1; w < W; ++w) acc += wave[w];
    }
    return acc;
}

// What comes of replica k's sum of squares.
__device__ __forceinline__ Clip clip_of(const NormArgs &n, uint32_t k, double sum)
{
    const double norm = __builtin_sqrt(sum);
    if (n.norms) *as_global<float>(n.norms + k) = (float)norm;
    // no limit: nothing is scaled, whatever the norm is (the quotient would make a NaN of an infinite one)
    const double c = __builtin_isinf(n.max_norm) ? 1.0 : (double)n.max_norm / (norm + LASGD_CLIP_EPS);
    const bool finite = norm <= 1.7976931348623157e308;
    return Clip{c >= 1.0 ? 1.f : (float)c, n.skip_nonfinite && !finite ? 1u : 0u};          // a NaN stays one
}
__device__ __forceinline__ void finish_norm(const NormArgs &n, uint32_t k, double sum)
{
    const Clip c = clip_of(n, k, sum);
    if (n.clip) n.clip[k] = c;
}

template <bool BF16>
__device__ __forceinline__ float4 grad_at(const char *g, uint32_t e, uint32_t n)
{
    if (n == 4u) return BF16 ? widen4(ld2<0>(reinterpret_cast<const uint16_t *>(g) + e)) : ld4<0>(reinterpret_cast<const float *>(g) + e);
    float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
    LASGD_FOR4(if (c < 3 && (uint32_t)c < n) comp(r, c) = BF16 ? bf16_widen(as_global<uint16_t>(g)[e + c]) : as_global<float>(g)[e + c];)
    return r;
}

// A workgroup has added up its share of replica k.  The last of the replica's workgroups adds the shares, in their order whoever is last, and is the
// one to say what comes of the norm: a kernel of its own for that costs a short call 2-4 us.  The counter is back at zero
// for the next call on the stream.
//
// Shares and counter are only ever touched by atomics of device scope, which bypass the XCDs' own L2s, so no cache has to be written back
// or invalidated for them.  What is needed beyond is that a share is in memory before its arrival is counted: the store is waited
// for.  (Left to an acquire-release addition, every workgroup writes back and invalidates its L2: norms of ResNet-50 K = 32 bf16
// 1863 us in place of 242.)  Counters of different replicas lie on lines of their own, kArriveStride apart.
__device__ __forceinline__ void join_norm(const NormArgs &n, uint32_t k, uint32_t group, uint32_t groups, double acc)
{
    double *part = n.part + (size_t)k * n.stride;
    acc = block_sum<kNormWaves>(acc);
    if (threadIdx.x >= 64u) return;               // the first wave does the rest
    if (groups > 1u) {
        uint32_t before = 0;
        if (threadIdx.x == 0u) {
            __hip_atomic_store(part + group, acc, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            before = __hip_atomic_fetch_add(n.arrived + k * kArriveStride, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        if (__builtin_amdgcn_readfirstlane(before) + 1u != groups) return;
        acc = 0.0;
        for (uint32_t i = threadIdx.x; i < groups; i += 256u) {
            double share[4];                      // asked for together
#pragma unroll
            for (uint32_t u = 0; u < 4u; ++u) {
                const uint32_t j = i + u * 64u;
                share[u] = __hip_atomic_load(part + (j < groups ? j : i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
#pragma unroll
            for (uint32_t u = 0; u < 4u; ++u) acc += i + u * 64u < groups ? share[u] : 0.0;
        }
        acc = wave_sum(acc);
        if (threadIdx.x == 0u) __hip_atomic_store(n.arrived + k * kArriveStride, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (threadIdx.x == 0u) finish_norm(n, k, acc);
}

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

template <int NT> __device__ __forceinline__ u32x4_t ld_u4(const char *p)
{
    if constexpr (NT & 1) return __builtin_nontemporal_load(as_global<u32x4_t>(p));
    else return *as_global<u32x4_t>(p);
}
template <int NT> __device__ __forceinline__ void st_u4(char *p, u32x4_t v)
{
    if constexpr (NT & 2) __builtin_nontemporal_store(v, as_global<u32x4_t>(p));
    else *as_global<u32x4_t>(p) = v;
}
template <bool BF16> __device__ __forceinline__ void add_squares(double &a0, double &a1, u32x4_t v)
{
    if constexpr (BF16) {
        add_squares(a0, widen4(make_uint2(v.x, v.y)));
        add_squares(a1, widen4(make_uint2(v.z, v.w)));
    } else
        add_squares(a0, a1, make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w)));
}

// A workgroup's runs are blocks of the lookup table, 64 tiles.  A run inside one tensor, as nearly all of a long list are,
// takes one lookup: its address, or NULL where several tensors meet in it or the list ends.
template <bool BF16>
__device__ __forceinline__ char *whole_run(const ApplyArgs &a, uint32_t k, uint32_t first, uint32_t entry)
{
    if (entry & kMoreInBlock) return nullptr;
    const Record rec = load_record(a, k, entry);
    const uint32_t off = (first - rec.arow) * 256u;                  // a tensor's first row in the arenas is its first tile
    return rec.numel - off >= kNormRun * 256u ? reinterpret_cast<char *>(rec.g) + (uint64_t)off * (BF16 ? 2u : 4u) : nullptr;
}

// Any run, tile by tile: four of a wave's tiles from `tile` on, every W-th one.  With sixteen waves a lane has the elements that it has in a run of one
// tensor in fp32.
struct FourTiles {
    char *g[4];             // the tensor's gradient from the tile on
    uint32_t n[4];          // how many of the lane's four elements there are
    float4 v[4];
};
// starts: at most 64 tensors start in a block; each lane holds one's first tile, and how many of them are not beyond a tile says whose it is.
__device__ __forceinline__ uint32_t later_starts(const ApplyArgs &a, uint32_t t0)
{
    const uint32_t t = t0 + 1u + (threadIdx.x & 63u);
    return t < a.n_tensors ? as_global<uint32_t>(a.tile0)[t] : 0xffffffffu;
}
template <bool BF16, uint32_t W>
__device__ __forceinline__ void load_four(FourTiles &f, const ApplyArgs &a, uint32_t k, uint32_t t0, uint32_t starts, uint32_t tile, uint32_t end)
{
    const uint32_t e = (threadIdx.x & 63u) * 4u;
#pragma unroll
    for (uint32_t u = 0; u < 4u; ++u, tile += W) {
        f.n[u] = 0;
        if (tile < end) {
            const Record rec = load_record(a, k, t0 + (uint32_t)__popcll(__ballot(starts <= tile)));
            const uint32_t off = (tile - rec.arow) * 256u;
            f.g[u] = reinterpret_cast<char *>(rec.g) + (uint64_t)off * (BF16 ? 2u : 4u);
            f.n[u] = lane_elems<false>(e, rec.numel - off);
        }
        f.v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (f.n[u]) f.v[u] = grad_at<BF16>(f.g[u], e, f.n[u]);
    }
}

// Sums of squares of one replica's gradients (blockIdx.y: of which).
//
// Few and large workgroups that go on: a share and its arrival are an atomic each at the memory all XCDs see, and arrivals at one
// counter come one after the other, 10 ns each.  norm_groups in the host code holds their number and what it measured.
template <bool BF16, int NT>
__global__ __launch_bounds__(kNormThreads) void grad_norm_kernel(const ApplyArgs a, const NormArgs n)
{
    constexpr uint32_t ROUNDS = kNormRun * 256u * (BF16 ? 2u : 4u) / (kNormThreads * 16u);          // of 16 bytes a thread
    const uint32_t w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t k = n.count == a.K ? blockIdx.y : nth_bit(n.mask, blockIdx.y);
    const uint32_t runs = (a.ntiles + kNormRun - 1u) / kNormRun;
    double a0 = 0.0, a1 = 0.0;
    for (uint32_t b = blockIdx.x; b < runs; b += n.parts) {
        const uint32_t first = b * kNormRun, entry = as_const(a.blocks)[first >> kBlockShift];
        if (const char *p = whole_run<BF16>(a, k, first, entry)) {
            u32x4_t v[ROUNDS];
#pragma unroll
            for (uint32_t u = 0; u < ROUNDS; ++u) v[u] = ld_u4<NT>(p + threadIdx.x * 16u + u * kNormThreads * 16u);
#pragma unroll
            for (uint32_t u = 0; u < ROUNDS; ++u) add_squares<BF16>(a0, a1, v[u]);
            continue;
        }
        const uint32_t t0 = entry & ~kMoreInBlock, starts = later_starts(a, t0);
        const uint32_t end = first + kNormRun < a.ntiles ? first + kNormRun : a.ntiles;
        FourTiles f;
        load_four<BF16, kNormWaves>(f, a, k, t0, starts, first + w, end);
#pragma unroll
        for (uint32_t u = 0; u < 4u; ++u) add_squares(a0, a1, f.v[u]);
    }
    join_norm(n, k, blockIdx.x, n.parts, a0 + a1);
}

// The mean gradient of all replicas (mean_grad_tile) and its norm in one pass.  A wave's tiles stay on its XCD, where the step looks for them.
template <bool BF16, int NT>
__global__ __launch_bounds__(kNormThreads) void mean_grad_norm_kernel(const ApplyArgs a, const NormArgs n)
{
    const uint32_t lane = threadIdx.x & 63u, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    double acc = 0.0;
    for (uint32_t tile = w * n.parts + blockIdx.x; tile < a.ntiles; tile += kNormWaves * n.parts) {
        const uint32_t tensor = tensor_of(a, tile);
        const Tile t = locate(a, load_record(a, 0, tensor), tile, tensor, 256u);
        // the lanes beyond a tensor's end have a mean of zero
        if (t.count == 256u) add_squares(acc, mean_grad_tile<BF16, NT, true>(a, t, tensor, lane));
        else add_squares(acc, mean_grad_tile<BF16, NT, false>(a, t, tensor, lane));
    }
    join_norm(n, 0u, blockIdx.x, n.parts, acc);
}

__device__ __forceinline__ float4 times(float4 v, float c) { return make_float4(v.x * c, v.y * c, v.z * c, v.w * c); }

template <bool BF16>
__device__ __forceinline__ void store_grad(char *g, uint32_t e, uint32_t n, float4 v)
{
    if (n == 4u) {
        if constexpr (BF16) st2<0>(reinterpret_cast<uint16_t *>(g) + e, round4(v));
        else st4<0>(reinterpret_cast<float *>(g) + e, v);
    } else {
        LASGD_FOR4(if (c < 3 && (uint32_t)c < n) {
            if constexpr (BF16) as_global<uint16_t>(g)[e + c] = (uint16_t)bf16_round(compv(v, c));
            else as_global<float>(g)[e + c] = compv(v, c);
        })
    }
}

// Clipping in place: gradients times c, rounded once to the storage type, where c is not 1.  How many replicas that is is known here alone, so the
// workgroups share out the runs of those that are scaled.  us of a call with four of eight
// replicas scaled, workgroups for each replica / this: ResNet-50 list 322 / 297 (the norms alone 122), ResNet-18 162 / 138; bf16, 20 of 32, ResNet-50 757 / 660.
template <bool BF16, int NT>
__global__ __launch_bounds__(kNormThreads) void scale_grads_kernel(const ApplyArgs a, const NormArgs n)
{
    constexpr uint32_t ROUNDS = kNormRun * 256u * (BF16 ? 2u : 4u) / (kNormThreads * 16u);
    const uint32_t lane = threadIdx.x & 63u, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), e = lane * 4u;
    bool scale = false;
    if ((n.mask >> lane) & 1ull) {
        const Clip mine = n.clip[lane];
        scale = !mine.skip && mine.c != 1.f;
    }
    const uint64_t scaled = __ballot(scale);
    const uint32_t runs = (a.ntiles + kNormRun - 1u) / kNormRun, items = (uint32_t)__popcll(scaled) * runs;
    for (uint32_t i = blockIdx.x; i < items; i += n.parts) {
        const uint32_t j = fast_div(i, n.by_runs), k = nth_bit(scaled, j);
        const Clip cl = load_clip(n.clip, k);
        const uint32_t first = (i - j * runs) * kNormRun, entry = as_const(a.blocks)[first >> kBlockShift];
        if (char *p = whole_run<BF16>(a, k, first, entry)) {
            u32x4_t v[ROUNDS];
#pragma unroll
            for (uint32_t u = 0; u < ROUNDS; ++u) v[u] = ld_u4<NT>(p + threadIdx.x * 16u + u * kNormThreads * 16u);
#pragma unroll
            for (uint32_t u = 0; u < ROUNDS; ++u) {
                if constexpr (BF16) {
                    const uint2 lo = round4(times(widen4(make_uint2(v[u].x, v[u].y)), cl.c)), hi = round4(times(widen4(make_uint2(v[u].z, v[u].w)), cl.c));
                    v[u] = u32x4_t{lo.x, lo.y, hi.x, hi.y};
                } else {
                    const float4 t = times(make_float4(__uint_as_float(v[u].x), __uint_as_float(v[u].y), __uint_as_float(v[u].z), __uint_as_float(v[u].w)), cl.c);
                    v[u] = u32x4_t{__float_as_uint(t.x), __float_as_uint(t.y), __float_as_uint(t.z), __float_as_uint(t.w)};
                }
                st_u4<NT>(p + threadIdx.x * 16u + u * kNormThreads * 16u, v[u]);
            }
            continue;
        }
        const uint32_t t0 = entry & ~kMoreInBlock, starts = later_starts(a, t0);
        const uint32_t end = first + kNormRun < a.ntiles ? first + kNormRun : a.ntiles;
        FourTiles f;
        load_four<BF16, kNormWaves>(f, a, k, t0, starts, first + w, end);
#pragma unroll
        for (uint32_t u = 0; u < 4u; ++u) store_grad<BF16>(f.g[u], e, f.n[u], times(f.v[u], cl.c));
    }
}

// ---- short lists ---------------------------------------------------------------
// Norm and what follows in one launch of workgroups of sixteen waves, bound by latency: 4.5 us a step of the list of 5,453 elements in six tensors, K = 3,
// in two launches 6.2 to 8.1.  one_launch in the host code holds the lines.
//
// fp32 sums come to the same bits as grad_norm_kernel's, in which a list of two blocks has two workgroups: a clipped step is to be
// clipping in place and a step, whichever of them takes one launch.  Each block's sum is made in the same order, and then they are added.
constexpr uint32_t kSmallWaves = 16, kSmallBlocks = 2;           // at most
static_assert(kSmallWaves == kNormWaves, "a lane's elements of a block are those it has in grad_norm_kernel");

// What comes of a replica's sums of squares, wave[block][its waves], in all threads; `says`: this workgroup is the one to write the norm.
__device__ __forceinline__ Clip small_clip(const NormArgs &n, uint32_t k, const double (*wave)[kSmallWaves], uint32_t blocks, bool says)
{
    __shared__ Clip shared;
    __syncthreads();
    if (threadIdx.x == 0u) {
        double sum = 0.0;
        for (uint32_t b = 0; b < blocks; ++b) {
            double acc = wave[b][0];
#pragma unroll
            for (uint32_t w = 1; w < kSmallWaves; ++w) acc += wave[b][w];
            sum += acc;
        }
        NormArgs m = n;
        if (!says) m.norms = nullptr;
        shared = clip_of(m, k, sum);
    }
    __syncthreads();
    return shared;
}

// The same of all of replica k: always in one order, so that every workgroup that takes it gets the same bits.  A block's sums leave the registers before the next
// one's gradients come: kept until all are there, 64 replicas of 128 tiles take 10.9 us a step in place of 10.4.
template <bool BF16>
__device__ __forceinline__ Clip whole_clip(const ApplyArgs &a, const NormArgs &n, uint32_t k, uint32_t w, bool says)
{
    constexpr uint32_t kBlock = 1u << kBlockShift;
    __shared__ double wave[kSmallBlocks][kSmallWaves];
    for (uint32_t first = 0; first < a.ntiles; first += kBlock) {
        const uint32_t b = first >> kBlockShift, t0 = as_const(a.blocks)[b] & ~kMoreInBlock;
        FourTiles f;
        load_four<BF16, kSmallWaves>(f, a, k, t0, later_starts(a, t0), first + w, first + kBlock < a.ntiles ? first + kBlock : a.ntiles);
        double a0 = 0.0, a1 = 0.0;
#pragma unroll
        for (uint32_t u = 0; u < 4u; ++u) add_squares(a0, a1, f.v[u]);
        const double sum = wave_sum(a0 + a1);
        if ((threadIdx.x & 63u) == 0u) wave[b][w] = sum;
    }
    return small_clip(n, k, wave, (a.ntiles + kBlock - 1u) / kBlock, says);
}

// Clipping in place, lists of one block: a workgroup a replica, whose gradients wait in registers for the norm.
template <bool BF16>
__global__ __launch_bounds__(1024) void small_scale_kernel(const ApplyArgs a, const NormArgs n)
{
    const uint32_t w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), e = (threadIdx.x & 63u) * 4u;
    const uint32_t k = n.count == a.K ? blockIdx.x : nth_bit(n.mask, blockIdx.x);
    FourTiles f;
    load_four<BF16, kSmallWaves>(f, a, k, 0u, later_starts(a, 0u), w, a.ntiles);
    double a0 = 0.0, a1 = 0.0;
#pragma unroll
    for (uint32_t u = 0; u < 4u; ++u) add_squares(a0, a1, f.v[u]);
    __shared__ double wave[1][kSmallWaves];
    const double sum = wave_sum(a0 + a1);
    if ((threadIdx.x & 63u) == 0u) wave[0][w] = sum;
    const Clip cl = small_clip(n, k, wave, 1u, true);
    if (cl.skip || cl.c == 1.f) return;
#pragma unroll
    for (uint32_t u = 0; u < 4u; ++u) store_grad<BF16>(f.g[u], e, f.n[u], times(f.v[u], cl.c));
}

// A local step of the replicas in the mask.  Sixteen tiles of a replica to a workgroup (blockIdx.y: which), one a wave; each workgroup takes the norm
// of the whole replica by itself rather than wait for the others: gradients are only read here.  A wave asks for its tile's gradients, model and
// momentum first.  bf16: one_launch sees to it that the models are in the master copies.
template <bool BF16>
__global__ __launch_bounds__(1024) void small_step_kernel(const ApplyArgs a, const ExtArgs xa, const NormArgs n)
{
    constexpr uint32_t ESZ = BF16 ? 2u : 4u;
    const uint32_t w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), e = (threadIdx.x & 63u) * 4u;
    const uint32_t k = replica_at<true>(a, &xa, blockIdx.x), tile = blockIdx.y * kSmallWaves + w;
    float4 g = make_float4(0.f, 0.f, 0.f, 0.f), x = g, v = g;
    char *xu = nullptr;
    float *vp = nullptr, *xm = nullptr, wd = 0.f;
    uint32_t m = 0;
    if (tile < a.ntiles) {
        const uint32_t tensor = tensor_of(a, tile);
        const Record rec = load_record(a, k, tensor);
        const Tile t = locate(a, rec, tile, tensor, 256u);
        const size_t ao = (size_t)k * a.npad + t.aoff;
        m = lane_elems<false>(e, t.count);
        wd = t.wd;
        xu = reinterpret_cast<char *>(rec.x) + t.toff * ESZ;
        vp = a.v + ao;
        xm = BF16 ? a.x32 + ao : reinterpret_cast<float *>(xu);
        if (m) {
            g = grad_at<BF16>(reinterpret_cast<const char *>(rec.g) + t.toff * ESZ, e, m);
            x = grad_at<false>(reinterpret_cast<const char *>(xm), e, m);
            v = ld4<0>(vp + e);                          // the arenas are padded to whole rows
        }
    }
    const Clip cl = whole_clip<BF16>(a, n, k, w, blockIdx.y == 0u);
    if (cl.skip || !m) return;
    const float neg_lr = xa.neg_lr_k[k];
    LASGD_FOR4(step_elem(comp(x, c), comp(v, c), cl.c * compv(g, c), wd, a.mu, neg_lr, a.nesterov);)
    store_grad<false>(reinterpret_cast<char *>(vp), e, m, v);
    store_grad<false>(reinterpret_cast<char *>(xm), e, m, x);
    if constexpr (BF16) store_grad<true>(xu, e, m, x);
}

// The same with the global update, of the replicas in the masks.
template <bool BF16>
__global__ __launch_bounds__(1024) void small_update_kernel(const ApplyArgs a, const ExtArgs xa, const NormArgs n)
{
    const uint32_t lane = threadIdx.x & 63u, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t k = replica_at<true>(a, &xa, blockIdx.x), tile = blockIdx.y * kSmallWaves + w;
    const bool in_step = (xa.step_mask >> k) & 1ull, in_merge = (xa.merge_mask >> k) & 1ull;
    Clip cl{1.f, 0u};
    if (in_step) cl = whole_clip<BF16>(a, n, k, w, blockIdx.y == 0u);
    if (tile >= a.ntiles) return;
    const uint32_t tensor = tensor_of(a, tile);
    const Record rec = load_record(a, k, tensor);
    const Tile t = locate(a, rec, tile, tensor, 256u);
    const float4 zt[1] = {ld4<0>(a.z + t.aoff + lane * 4u)};
    char *xu = reinterpret_cast<char *>(rec.x) + t.toff * (BF16 ? 2u : 4u);
    const char *gu = reinterpret_cast<const char *>(rec.g) + t.toff * (BF16 ? 2u : 4u);
    const size_t ao = (size_t)k * a.npad + t.aoff;
    float *xm = BF16 ? a.x32 + ao : nullptr;
    const float nlr = xa.neg_lr_k[k];
#define LASGD_SMALL(OPX) apply_tile<1, OPX, BF16, 0, false, true, false, false, true>(a, xu, gu, xm, xm, a.v + ao, a.s + ao, zt, t.wd, t.count, lane, nlr, xa.alpha, cl)
    if (!in_merge) LASGD_SMALL(OP_STEP);
    else if (in_step) LASGD_SMALL(OP_STEP_MERGE);
    else LASGD_SMALL(OP_MERGE);
#undef LASGD_SMALL
}

} // namespace lasgd
