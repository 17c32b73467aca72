// Host side of the operators of the replicas' forward and backward passes: checks, launch shapes.  Declared in include/lasgd.h.
#include "lasgd_context.h"
#include "lasgd_gated.hip.h"

#include <cmath>
#include <cstring>

using namespace lasgd;

namespace {

constexpr int64_t kMaxRows = 0x7fffffff;             // of all replicas together
constexpr int64_t kMaxGroups = 1ll << 48;            // of eight columns, a replica's, where a mask's counter names them
constexpr int64_t kMaxTiles = 0x7fffffff;            // of a gated block's products, what their kernels count
constexpr uint64_t kMaxThreads = 0xffffffff;         // of a launch, along x

// What a call's rows come to.
struct Rows {
    uint32_t n[64], first[64];
    uint32_t most = 0, total = 0, replicas = 0;      // replicas: with any rows
};

#define CHECK(cond, st, ...) do { if (!(cond)) return refuse(c, st, __VA_ARGS__); } while (0)
#define TRY(call) do { const lasgd_status st_ = (call); if (st_ != LASGD_OK) return st_; } while (0)

lasgd_status check_call(lasgd_ctx *c, const ContextView &v, const int64_t *rows, Rows &r)
{
    CHECK(rows, LASGD_ERR_INVALID, "NULL rows");
    int64_t total = 0;
    for (int32_t k = 0; k < v.K; ++k) {
        CHECK(rows[k] >= 0, LASGD_ERR_INVALID, "rows[%d] = %lld", k, (long long)rows[k]);
        CHECK(rows[k] <= kMaxRows - total, LASGD_ERR_UNSUPPORTED, "more than %lld rows", (long long)kMaxRows);
        r.first[k] = (uint32_t)total;
        r.n[k] = (uint32_t)rows[k];
        total += rows[k];
        if (r.n[k] > r.most) r.most = r.n[k];
        r.replicas += rows[k] > 0;
    }
    r.total = (uint32_t)total;
    return LASGD_OK;
}

lasgd_status check_device(lasgd_ctx *c, const ContextView &v)
{
    int dev = -1;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        return refuse(c, LASGD_ERR_HIP, "hipGetDevice failed: %s", hipGetErrorString(e));
    }
    CHECK(dev == v.device, LASGD_ERR_INVALID, "the context is on device %d, the current device is %d", v.device, dev);
    return LASGD_OK;
}

// An activation of `cols` columns.  vec comes out false if accesses of eight elements would not be aligned (es bytes an element).  A stride that
// nothing is multiplied with does not count.
lasgd_status check_rows(lasgd_ctx *c, const ContextView &v, const Rows &r, const char *name, const lasgd_rows *a, int64_t cols, int es, bool output,
                        RowsAt &at, bool &vec)
{
    CHECK(a && (a->data || !r.most), LASGD_ERR_INVALID, "NULL %s", name);
    at = RowsAt{(char *)a->data, v.K > 1 ? a->replica_stride : 0, r.most > 1 ? a->row_stride : 0};
    CHECK((uintptr_t)a->data % es == 0, LASGD_ERR_INVALID, "%s is not aligned to its elements", name);
    CHECK(at.rs >= 0 && at.ss >= 0, LASGD_ERR_INVALID, "%s has a negative stride", name);
    const __int128 end = (__int128)at.rs * (v.K - 1) + (__int128)at.ss * (r.most ? r.most - 1 : 0) + cols;
    CHECK(end * es < (__int128)1 << 47, LASGD_ERR_INVALID, "%s reaches beyond the address space", name);
    if (output) {
        CHECK(r.most <= 1 || at.ss >= cols, LASGD_ERR_INVALID, "the rows of %s overlap: stride %lld, %lld columns", name, (long long)at.ss, (long long)cols);
        if (r.replicas > 1) {
            const bool apart = at.rs >= (int64_t)(r.most - 1) * at.ss + cols;
            const bool turned = at.rs >= cols && (r.most <= 1 || at.ss >= (v.K - 1) * at.rs + cols);
            CHECK(apart || turned, LASGD_ERR_INVALID, "the replicas of %s overlap: stride %lld", name, (long long)at.rs);
        }
    }
    const int wide = es == 1 ? 8 : 16;
    if (cols % 8 || (uintptr_t)a->data % wide || at.rs * es % wide || at.ss * es % wide) vec = false;
    return LASGD_OK;
}

lasgd_status check_drop(lasgd_ctx *c, const lasgd_drop *d, DropArgs &a)
{
    a = DropArgs{};
    if (!d) return LASGD_OK;
    CHECK(d->p >= 0.f && d->p <= 1.f, LASGD_ERR_INVALID, "p = %g is no probability", (double)d->p);
    if (d->p == 0.f) return LASGD_OK;
    a.below = (uint32_t)std::lrint((double)d->p * 65536.0);
    a.scale = a.below < 65536u ? (float)(65536.0 / (65536.0 - a.below)) : 0.f;
    a.seed = d->seed;
    a.call = d->call;
    a.counter = d->counter;
    CHECK((uintptr_t)d->counter % 8 == 0, LASGD_ERR_INVALID, "the counter is not 8-byte aligned");
    return LASGD_OK;
}

lasgd_status check_groups(lasgd_ctx *c, const Rows &r, int64_t cols)
{
    CHECK((__int128)r.most * ((cols + 7) / 8) < kMaxGroups, LASGD_ERR_UNSUPPORTED, "a mask of more than 2^48 groups of eight columns");
    return LASGD_OK;
}

lasgd_status check_tensor(lasgd_ctx *c, const ContextView &v, const char *name, int32_t t)
{
    CHECK(t >= 0 && t < v.n_tensors, LASGD_ERR_INVALID, "%s = %d outside 0..%d", name, t, v.n_tensors - 1);
    return LASGD_OK;
}

lasgd_status check_workspace(lasgd_ctx *c, const void *p, int64_t have, int64_t need)
{
    if (!need) return LASGD_OK;
    CHECK(p, LASGD_ERR_INVALID, "NULL workspace");
    CHECK((uintptr_t)p % 16 == 0, LASGD_ERR_INVALID, "the workspace is not 16-byte aligned");
    CHECK(have >= need, LASGD_ERR_INVALID, "a workspace of %lld bytes, %lld are needed", (long long)have, (long long)need);
    return LASGD_OK;
}

lasgd_status launched(lasgd_ctx *c)
{
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return refuse(c, LASGD_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
    return LASGD_OK;
}

template <class T> void copy_rows(T &a, const Rows &r, int32_t K) { memcpy(a.rows, r.n, K * sizeof(uint32_t)); }

uint64_t round_up16(uint64_t n) { return (n + 15) / 16 * 16; }

uint32_t ceil_div(uint64_t a, uint64_t b) { return (uint32_t)((a + b - 1) / b); }

// f(std::integral_constant<bool, ...>...) for two flags.
template <class F> void two_flags(bool a, bool b, F f)
{
    if (a) {
        if (b) f(std::true_type{}, std::true_type{});
        else f(std::true_type{}, std::false_type{});
    } else {
        if (b) f(std::false_type{}, std::true_type{});
        else f(std::false_type{}, std::false_type{});
    }
}

// launch(first row, workgroups) for all rows of a call whose workgroups take `each` of them, in as few launches as hold them.
template <class F> void in_launches(const Rows &r, uint32_t each, uint32_t threads, F launch)
{
    const uint64_t all = ceil_div(r.most, each), most = kMaxThreads / threads;
    for (uint64_t at = 0; at < all; at += most) launch(at * each, (uint32_t)(all - at < most ? all - at : most));
}

constexpr int64_t kBeyondCache = 256ll << 20;        // the memory-side cache

// f(storage is bf16, Access) for a call whose accesses are aligned or not, and that moves so many bytes.  The hint beyond the memory-side
// cache: dropout of 8 x 4096 x 2048 bf16, forward and backward, 79 us without and 67 with it (the median of the two); a norm with an
// 8-bit output of 8 x 2048 x 4096 86 and 79; a norm's backward pass 139 and 137.  Below, what is written is still there for the next call.
template <class F> void row_access(bool bf16, bool vec, int64_t bytes, F f)
{
    auto storage = [&](auto v) {
        if (bf16) f(std::true_type{}, v);
        else f(std::false_type{}, v);
    };
    if (!vec) storage(std::integral_constant<int, LOOSE>{});
    else if (bytes < kBeyondCache) storage(std::integral_constant<int, WIDE>{});
    else storage(std::integral_constant<int, STREAM>{});
}

// Threads that share a row of a norm, and groups of eight columns that each of them holds.
template <int G_, int NV_> struct NormShape { static constexpr int G = G_, NV = NV_; };
template <class F> void norm_shape(uint32_t groups, F f)
{
    if (groups <= 16u) f(NormShape<16, 1>{});
    else if (groups <= 64u) f(NormShape<64, 1>{});
    else if (groups <= 128u) f(NormShape<64, 2>{});
    else if (groups <= 256u) f(NormShape<64, 4>{});
    else if (groups <= 512u) f(NormShape<256, 2>{});
    else if (groups <= 1024u) f(NormShape<256, 4>{});
    else f(NormShape<1024, 2>{});
}

// The backward pass holds more of a row's data a thread, so more threads share it: 2048 bf16 columns with 64 threads 156 us (238 registers, two waves a SIMD),
// with 256 139.
template <class F> void norm_back_shape(uint32_t groups, F f)
{
    if (groups <= 16u) f(NormShape<16, 1>{});
    else if (groups <= 64u) f(NormShape<64, 1>{});
    else if (groups <= 256u) f(NormShape<256, 1>{});
    else if (groups <= 512u) f(NormShape<256, 2>{});
    else if (groups <= 1024u) f(NormShape<1024, 1>{});
    else f(NormShape<1024, 2>{});
}

// Workgroups a replica of a norm's backward pass, each of which leaves a share of the gain's gradient: 1024 in all, four a CU.  (8 x 4096 x 2048 bf16, with the
// shares' sum: 1024 144 us, 1280 145, 2048 163.)
struct Shares {
    uint32_t parts;
    int64_t bytes;
};
Shares norm_shares(int32_t K, const Rows &r, uint32_t groups)
{
    Shares s{};
    norm_back_shape(groups, [&](auto shape) {
        constexpr uint32_t R = norm_threads(shape.G) / shape.G;
        const uint32_t want = 1024u / (r.replicas ? r.replicas : 1u), have = ceil_div(r.most, R);
        s.parts = have < want ? have : want;
    });
    s.bytes = (int64_t)K * s.parts * groups * 8 * sizeof(float);
    return s;
}

lasgd_status check_norm(lasgd_ctx *c, ContextView &v, int32_t gain, const int64_t *rows, Rows &r, int64_t &cols)
{
    v = view_of(c);
    TRY(check_call(c, v, rows, r));
    TRY(check_tensor(c, v, "gain", gain));
    cols = v.numel[gain];
    CHECK(cols <= LASGD_NORM_MAX_COLS, LASGD_ERR_UNSUPPORTED, "%lld columns, LASGD_NORM_MAX_COLS is %d", (long long)cols, LASGD_NORM_MAX_COLS);
    return LASGD_OK;
}

lasgd_status check_eps(lasgd_ctx *c, float eps)
{
    CHECK(std::isfinite(eps) && eps >= 0.f, LASGD_ERR_INVALID, "eps must be finite and >= 0");
    return LASGD_OK;
}

} // namespace

extern "C" lasgd_status lasgd_dropout(lasgd_ctx *c, const int64_t *rows, int64_t cols, const lasgd_rows *x, const lasgd_rows *residual,
                                      const lasgd_rows *y, const lasgd_drop *drop, void *stream)
{
    if (!c) return LASGD_ERR_INVALID;
    const ContextView v = view_of(c);
    const int es = v.bf16 ? 2 : 4;
    Rows r;
    DropoutArgs a{};
    bool vec = true;
    TRY(check_call(c, v, rows, r));
    CHECK(cols >= 1 && cols <= kMaxRows, LASGD_ERR_INVALID, "cols = %lld", (long long)cols);
    CHECK(drop, LASGD_ERR_INVALID, "NULL drop");
    TRY(check_drop(c, drop, a.drop));
    if (!a.drop.below) a.drop.scale = 1.f;
    TRY(check_groups(c, r, cols));
    TRY(check_rows(c, v, r, "x", x, cols, es, false, a.x, vec));
    if (residual) TRY(check_rows(c, v, r, "residual", residual, cols, es, false, a.residual, vec));
    TRY(check_rows(c, v, r, "y", y, cols, es, true, a.y, vec));
    TRY(check_device(c, v));
    if (!r.most) return LASGD_OK;
    a.cols = (uint32_t)cols;
    a.groups = ceil_div(cols, 8);
    while (a.tx_shift < 8u && (1u << a.tx_shift) < a.groups) ++a.tx_shift;
    copy_rows(a, r, v.K);
    row_access(v.bf16, vec, (int64_t)r.total * cols * es * (residual ? 3 : 2), [&](auto bf16, auto wide) {
        in_launches(r, (256u >> a.tx_shift) * kDropRows, 256, [&](uint64_t row0, uint32_t blocks) {
            a.row0 = row0;
            hipLaunchKernelGGL((dropout_kernel<bf16, wide>), dim3(blocks, v.K), dim3(256), 0, (hipStream_t)stream, a);
        });
    });
    return launched(c);
}

extern "C" lasgd_status lasgd_rms_norm(lasgd_ctx *c, int32_t gain, const int64_t *rows, const lasgd_rows *x, const lasgd_rows *residual,
                                       const lasgd_rows *sum, const lasgd_rows *y, const lasgd_rows *scales, float eps, const lasgd_drop *drop, void *stream)
{
    if (!c) return LASGD_ERR_INVALID;
    ContextView v;
    Rows r;
    int64_t cols;
    NormRowsArgs a{};
    bool vec = true, ignored = true;
    TRY(check_norm(c, v, gain, rows, r, cols));
    const int es = v.bf16 ? 2 : 4;
    TRY(check_eps(c, eps));
    TRY(check_drop(c, drop, a.drop));
    TRY(check_groups(c, r, cols));
    TRY(check_rows(c, v, r, "x", x, cols, es, false, a.x, vec));
    if (residual) TRY(check_rows(c, v, r, "residual", residual, cols, es, false, a.residual, vec));
    if (sum) TRY(check_rows(c, v, r, "sum", sum, cols, es, true, a.sum, vec));
    TRY(check_rows(c, v, r, "y", y, cols, scales ? 1 : es, true, a.y, vec));
    if (scales) TRY(check_rows(c, v, r, "scales", scales, 1, 4, true, a.scales, ignored));
    CHECK(v.all_bound, LASGD_ERR_STATE, "not every replica is bound");
    TRY(check_device(c, v));
    if (!r.most) return LASGD_OK;
    a.cols = (uint32_t)cols;
    a.groups = ceil_div(cols, 8);
    a.eps = eps;
    a.inv_cols = (float)(1.0 / (double)cols);
    copy_rows(a, r, v.K);
    for (int32_t k = 0; k < v.K; ++k) a.gain[k] = (const char *)v.params[(size_t)k * v.n_tensors + gain];
    norm_shape(a.groups, [&](auto shape) {
        constexpr int G = decltype(shape)::G, NV = decltype(shape)::NV, T = norm_threads(G);
        const int64_t bytes = (int64_t)r.total * cols * (es * (1 + !!residual + !!sum) + (scales ? 1 : es));
        row_access(v.bf16, vec, bytes, [&](auto bf16, auto wide) {
            in_launches(r, T / G, T, [&](uint64_t row0, uint32_t blocks) {
                a.row0 = row0;
                if (scales) hipLaunchKernelGGL((rms_norm_kernel<bf16, wide, G, NV, true>), dim3(blocks, v.K), dim3(T), 0, (hipStream_t)stream, a);
                else hipLaunchKernelGGL((rms_norm_kernel<bf16, wide, G, NV, false>), dim3(blocks, v.K), dim3(T), 0, (hipStream_t)stream, a);
            });
        });
    });
    return launched(c);
}

extern "C" lasgd_status lasgd_rms_norm_backward_bytes(lasgd_ctx *c, int32_t gain, const int64_t *rows, int64_t *bytes)
{
    if (!c) return LASGD_ERR_INVALID;
    ContextView v;
    Rows r;
    int64_t cols;
    CHECK(bytes, LASGD_ERR_INVALID, "NULL bytes");
    TRY(check_norm(c, v, gain, rows, r, cols));
    *bytes = norm_shares(v.K, r, ceil_div(cols, 8)).bytes;
    return LASGD_OK;
}

extern "C" lasgd_status lasgd_rms_norm_backward(lasgd_ctx *c, int32_t gain, const int64_t *rows, const lasgd_rows *h, const lasgd_rows *dy,
                                                const lasgd_rows *dsum, const lasgd_rows *dresidual, const lasgd_rows *dx, float eps,
                                                const lasgd_drop *drop, int32_t accumulate, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (!c) return LASGD_ERR_INVALID;
    ContextView v;
    Rows r;
    int64_t cols;
    NormBackArgs a{};
    bool vec = true;
    TRY(check_norm(c, v, gain, rows, r, cols));
    const int es = v.bf16 ? 2 : 4;
    TRY(check_eps(c, eps));
    TRY(check_drop(c, drop, a.drop));
    TRY(check_groups(c, r, cols));
    TRY(check_rows(c, v, r, "h", h, cols, es, false, a.h, vec));
    TRY(check_rows(c, v, r, "dy", dy, cols, es, false, a.dy, vec));
    if (dsum) TRY(check_rows(c, v, r, "dsum", dsum, cols, es, false, a.dsum, vec));
    if (dresidual) TRY(check_rows(c, v, r, "dresidual", dresidual, cols, es, true, a.dresidual, vec));
    if (dx) TRY(check_rows(c, v, r, "dx", dx, cols, es, true, a.dx, vec));
    a.groups = ceil_div(cols, 8);
    const Shares s = norm_shares(v.K, r, a.groups);
    TRY(check_workspace(c, workspace, workspace_bytes, s.bytes));
    CHECK(v.all_bound, LASGD_ERR_STATE, "not every replica is bound");
    TRY(check_device(c, v));
    if (!r.most && accumulate) return LASGD_OK;
    a.cols = (uint32_t)cols;
    a.eps = eps;
    a.inv_cols = (float)(1.0 / (double)cols);
    a.parts = s.parts;
    a.part = (float *)workspace;
    copy_rows(a, r, v.K);
    JoinArgs j{(const float *)workspace, s.parts, (uint32_t)cols, a.groups, accumulate, {}};
    for (int32_t k = 0; k < v.K; ++k) {
        a.gain[k] = (const char *)v.params[(size_t)k * v.n_tensors + gain];
        j.grad[k] = (char *)v.grads[(size_t)k * v.n_tensors + gain];
    }
    if (r.most) {
        norm_back_shape(a.groups, [&](auto shape) {
            constexpr int G = decltype(shape)::G, NV = decltype(shape)::NV, T = norm_threads(G);
            const int64_t bytes = (int64_t)r.total * cols * es * (2 + !!dsum + !!dresidual + !!dx);
            row_access(v.bf16, vec, bytes, [&](auto bf16, auto wide) {
                hipLaunchKernelGGL((rms_norm_backward_kernel<bf16, wide, G, NV>), dim3(s.parts, v.K), dim3(T), 0, (hipStream_t)stream, a);
            });
        });
        TRY(launched(c));
    }
    const dim3 grid(ceil_div(cols, 16), v.K);
    if (v.bf16) hipLaunchKernelGGL((join_gain_kernel<true>), grid, dim3(256), 0, (hipStream_t)stream, j);
    else hipLaunchKernelGGL((join_gain_kernel<false>), grid, dim3(256), 0, (hipStream_t)stream, j);
    return launched(c);
}

// ---- gated blocks ------------------------------------------------------------------------------------------------------------
namespace {

struct Gated {
    ContextView v;
    Rows r;
    int64_t wide, pitch;
    int es;
    bool few_tiles;                                  // no launch comes near kMaxThreads
};

lasgd_status check_gated(lasgd_ctx *c, Gated &d, int32_t gate, int32_t up, const int64_t *rows, int64_t cols)
{
    d.v = view_of(c);
    d.es = d.v.bf16 ? 2 : 4;
    TRY(check_call(c, d.v, rows, d.r));
    TRY(check_tensor(c, d.v, "gate", gate));
    TRY(check_tensor(c, d.v, "up", up));
    CHECK(cols >= 1, LASGD_ERR_INVALID, "cols = %lld", (long long)cols);
    const int64_t n = d.v.numel[gate], per = gate == up ? 2 * cols : cols;
    CHECK(n % per == 0, LASGD_ERR_INVALID, "tensor %d has %lld elements, no multiple of %lld", gate, (long long)n, (long long)per);
    CHECK(gate == up || d.v.numel[up] == n, LASGD_ERR_INVALID, "gate has %lld elements, up %lld", (long long)n, (long long)d.v.numel[up]);
    d.wide = n / per;
    d.pitch = (d.wide + 7) / 8 * 8;
    // a launch's workgroups: no tile is smaller than 16 rows of 32 columns, nor those of the weights' gradients than 32 x 32 (shares of dx are for few tiles)
    const __int128 tiles_w = (d.wide + 31) / 32, tiles_c = (cols + 31) / 32, tiles_r = ((int64_t)d.r.most / 16 + 1) * d.v.K;
    const auto each_below = [&](int64_t most) { return tiles_r * tiles_w <= most && tiles_r * tiles_c <= most && 2 * tiles_w * tiles_c * d.v.K <= most; };
    CHECK(each_below(kMaxTiles), LASGD_ERR_UNSUPPORTED, "more tiles than a launch counts");
    d.few_tiles = each_below(1 << 16);               // of 512 threads, and 64 shares of a contraction: 2^31
    return LASGD_OK;
}

lasgd_status check_act(lasgd_ctx *c, lasgd_activation act)
{
    CHECK((int)act >= LASGD_SILU && (int)act <= LASGD_RELU, LASGD_ERR_INVALID, "unknown activation %d", (int)act);
    return LASGD_OK;
}

ProductArgs product_args(const Gated &d, int64_t cols, lasgd_activation act)
{
    ProductArgs a{};
    a.cols = (uint32_t)cols;
    a.wide = (uint32_t)d.wide;
    a.pitch = (uint32_t)d.pitch;
    a.act = (int32_t)act;
    copy_rows(a, d.r, d.v.K);
    memcpy(a.first, d.r.first, d.v.K * sizeof(uint32_t));
    return a;
}

void weights(ProductArgs &a, const Gated &d, void *const *of, int32_t gate, int32_t up, int64_t cols)
{
    for (int32_t k = 0; k < d.v.K; ++k) {
        a.gate[k] = (char *)of[(size_t)k * d.v.n_tensors + gate];
        a.up[k] = (char *)of[(size_t)k * d.v.n_tensors + up] + (gate == up ? d.wide * cols * d.es : 0);
    }
}

// Whether a product's sides can go straight from memory into LDS: 16-byte pieces, a tile's lines within 32 bits of bytes.
bool streams(const Gated &d, int64_t cols, const RowsAt &x, bool vx)
{
    constexpr int64_t most = (1ll << 31) / 256 / 4;          // elements from one line to the next
    return vx && cols <= most && d.pitch <= most && x.ss <= most;
}

// Tiles of all replicas.
template <int FORM> uint64_t tiles_of(const Gated &d, int64_t cols, uint32_t tm, uint32_t tn)
{
    uint64_t rows = 0;
    for (int32_t k = 0; k < d.v.K; ++k) rows += ceil_div(FORM == DW ? d.wide : d.r.n[k], tm);
    return rows * ceil_div(FORM == FWD ? d.wide : cols, tn) * (FORM == DW ? 2 : 1);
}

constexpr uint32_t kCus = 256;

// The launches below: `go` false only says whether the product's launch has no more threads than it may.
constexpr const char *kTooManyThreads = "a product of 2^32 threads or more";
constexpr bool fits(uint64_t blocks, uint32_t threads) { return blocks <= kMaxThreads / threads; }

template <int FORM> bool launch_loose(const Gated &d, const ProductArgs &a, bool vm, bool vn, hipStream_t st, bool go)
{
    auto launch = [&](auto tile) {
        constexpr uint32_t T = decltype(tile)::value;
        const uint64_t M = FORM == DW ? d.wide : d.r.most, N = FORM == FWD ? a.wide : a.cols;
        ProductArgs b = a;
        b.tiles_m = ceil_div(M, T);
        b.tiles = b.tiles_m * ceil_div(N, FORM == FWD ? T / 2 : T);
        if (!go || !fits((uint64_t)b.tiles * d.v.K, 256)) return fits((uint64_t)b.tiles * d.v.K, 256);
        const dim3 grid(b.tiles * d.v.K, 1, FORM == DW ? 2 : 1);
        // dg and du lie in the workspace, aligned; an aligned x has whole eights of columns, and so have the weights
        two_flags(vm, vn, [&](auto m, auto n) {
            if constexpr (FORM == FWD ? !m || n : m) {
                if (d.v.bf16) hipLaunchKernelGGL((product_kernel<true, FORM, m, n, T>), grid, dim3(256), 0, st, b);
                else hipLaunchKernelGGL((product_kernel<false, FORM, m, n, T>), grid, dim3(256), 0, st, b);
            }
        });
        return true;
    };
    // us forward / dx / weights, tiles of 128 and of 64, behind others of their kind (a chip at rest clocks higher: fp32 488 / 477 / 447): bf16, K = 8, 2048 rows,
    // 2047 x 5503 1942 / 1828 / 1348 and 3487 / 3170 / 2158; fp32, K = 4, 1023 rows, 1023 x 2815 528 / 510 / 486 and 549 / 537 / 544; K = 8, 700 rows, 1535 x 1901
    // 756 / 896 / 680 and 739 / 772 / 736 (of dx there are 576 tiles of 128 in 512 places: a second round for 64); K = 3, up to 333 rows, 515 x 1030 61 / 188 / 60 and 46 / 75 / 38.
    if (tiles_of<FORM>(d, a.cols, 128, FORM == FWD ? 64 : 128) >= 2 * kCus) return launch(std::integral_constant<uint32_t, 128>{});
    return launch(std::integral_constant<uint32_t, 64>{});
}

// Rows of a tile of a gated block's products.  Large tiles read their sides less often, small ones fill the chip and waste less of few rows.  us forward / dx (with the
// sum of its shares) / weights, tiles of 128 and of 256: bf16, K = 8, 2048 rows, 2048 x 5504 985 / 849 / 900 and 802 / 675 / 722; K = 2, 512 rows, 1024 x 2816 24 / 39 / 22
// and 37 / 53 / 22; K = 16, up to 192 rows, 512 x 1408 31 / 30 / 22 and 32 / 35 / 24; fp32, K = 4, 1024 rows, 1024 x 2816 449 / 416 / 429 and 536 / 410 / 517: fp32, whose
// products take sixteen times as long beside the same reads, has none of 256.
// Of 64, K = 8, 48 rows, 2048 x 5504 66 / 94, of 256 151 / 98; of 16 with 4 rows 59 / 64.
template <int FORM> uint32_t tile_rows(const Gated &d, int64_t cols)
{
    if (FORM != DW && d.r.most <= 16u) return 16u;
    if (FORM != DW && d.r.most <= 64u) return 64u;
    return d.v.bf16 && tiles_of<FORM>(d, cols, 256, FORM == FWD ? 128 : 256) >= 2 * kCus ? 256u : 128u;
}

// Workgroups that share a tile of dx, in units of the contraction that every step divides: a contraction of 2 wide, and often few tiles.  us alone / shared, with the
// sum of the shares: K = 8, 4 rows, 2048 x 5504 179 / 64; 48 rows 185 / 85; K = 2, 512 rows, 1024 x 2816 58 / 39; K = 16, up to 192 rows, 512 x 1408 32 / 30.
constexpr uint32_t kUnit = 64;
struct Split {
    uint32_t count;
    int64_t deep;                // of the contraction, each
};
Split dx_split(const Gated &d, int64_t cols)
{
    if (!d.r.most) return {1, 2 * d.pitch};
    const uint32_t tm = tile_rows<DX>(d, cols), tn = tm == 128u ? 128u : 256u;
    const uint64_t tiles = tiles_of<DX>(d, cols, tm, tn), units = 2 * (uint64_t)ceil_div(d.pitch, kUnit);
    const uint64_t want = (tm == 256u ? 2 * kCus : 4 * kCus) / tiles, most = units / 4;
    uint64_t n = want < most ? want : most;
    n = n < 1 ? 1 : n > 64 ? 64 : n;
    const uint32_t per = ceil_div(units, n);
    return {ceil_div(units, per), (int64_t)per * kUnit};
}

template <int FORM, uint32_t TM, uint32_t TN, uint32_t WM, uint32_t WN, uint32_t LP, uint32_t NS, bool HINT = false>
bool launch_big(const Gated &d, const ProductArgs &a, const Split &split, float *part, hipStream_t st, bool go)
{
    static_assert(kUnit % (LP * 8u) == 0, "whole steps");
    constexpr uint32_t NT = FORM == FWD ? TN / 2u : TN;
    TileMap map{};
    map.replicas = (uint32_t)d.v.K;
    map.splits = split.count;
    map.per_split = (uint32_t)(split.deep / (LP * 16 / d.es));
    map.part = part;
    map.part_stride = (uint64_t)d.r.total * a.cols;
    uint32_t total = 0;
    for (int32_t k = 0; k < d.v.K; ++k) {
        map.first[k] = total;
        const uint32_t tm = ceil_div(FORM == DW ? a.wide : d.r.n[k], TM);
        total += tm * ceil_div(FORM == FWD ? a.wide : a.cols, NT) * (FORM == DW ? 2u : 1u);
    }
    map.first[d.v.K] = total;
    if (!go || !fits((uint64_t)total * split.count, 64u * WM * WN)) return fits((uint64_t)total * split.count, 64u * WM * WN);
    const dim3 grid(total * split.count), threads(64u * WM * WN);
    if (d.v.bf16) hipLaunchKernelGGL((big_product_kernel<true, FORM, TM, TN, WM, WN, LP, NS, HINT>), grid, threads, 0, st, a, map);
    else if constexpr (TM < 256u) hipLaunchKernelGGL((big_product_kernel<false, FORM, TM, TN, WM, WN, LP, NS, HINT>), grid, threads, 0, st, a, map);
    return true;
}

template <int FORM> bool launch_form(const Gated &d, const ProductArgs &a, bool big, bool vm, bool vn, const Split &split, float *part, hipStream_t st, bool go)
{
    const bool few = FORM == DW && d.v.bf16 && d.r.most <= kFewRows;
    // The tiles find the end of DW's rows of x by their address alone.  Rows that overlap do not end there: what is behind them counts 0 times, but an infinity
    // among it would still make a NaN of every sum.
    if (FORM == DW && !few && a.x.ss < (int64_t)a.cols) big = false;
    if (!big) return launch_loose<FORM>(d, a, vm, vn, st, go);
    if constexpr (FORM == DW) {
        if (few) {
            const uint64_t blocks = (uint64_t)ceil_div(a.wide, 256) * ceil_div(a.cols, 256);
            if (!go || !fits(blocks, 256)) return fits(blocks, 256);
            const dim3 grid((uint32_t)blocks, d.v.K, 2);
            two_flags(a.accumulate, 4 * (uint64_t)d.v.K * a.wide * a.cols >= kBeyondCache, [&](auto add, auto stream) {
                hipLaunchKernelGGL((few_rows_weights_kernel<add, stream ? STREAM : WIDE>), grid, dim3(256), 0, st, a);
            });
            return true;
        }
    }
    const uint32_t tm = tile_rows<FORM>(d, a.cols);
    if constexpr (FORM != DW) {
        // The hint on weights beyond the cache.  us, bf16, 2048 x 5504, without / with it: K = 4, 1 row (180 MB) forward 28 / 34; K = 8 (361 MB), 4 rows, forward 75 / 70,
        // backward 67 / 58; 48 rows 128 / 66 and 115 / 84.
        const bool hint = 2 * (uint64_t)d.es * d.v.K * a.wide * a.cols >= kBeyondCache;
        constexpr uint32_t TN = FORM == FWD ? 128 : 256;
        if (tm == 16u) return hint ? launch_big<FORM, 16, TN, 1, 4, 8, 2, true>(d, a, split, part, st, go) : launch_big<FORM, 16, TN, 1, 4, 8, 2>(d, a, split, part, st, go);
        if (tm == 64u) return hint ? launch_big<FORM, 64, TN, 1, 4, 8, 2, true>(d, a, split, part, st, go) : launch_big<FORM, 64, TN, 1, 4, 8, 2>(d, a, split, part, st, go);
    }
    if (tm == 128u) return launch_big<FORM, 128, 128, 2, 2, 8, 2>(d, a, split, part, st, go);
    return launch_big<FORM, 256, 256, 2, 4, 8, 2>(d, a, split, part, st, go);
}

int64_t gates_bytes(const Gated &d) { return (int64_t)round_up16((uint64_t)d.r.total * d.pitch * d.es); }          // dg, and du again
int64_t gated_bytes(const Gated &d, int64_t cols)
{
    const uint32_t splits = dx_split(d, cols).count;
    return 2 * gates_bytes(d) + (splits > 1 ? (int64_t)splits * d.r.total * cols * (int64_t)sizeof(float) : 0);
}

} // namespace

extern "C" lasgd_status lasgd_gated(lasgd_ctx *c, int32_t gate, int32_t up, const int64_t *rows, int64_t cols, const lasgd_rows *x, const lasgd_rows *g,
                                    const lasgd_rows *u, const lasgd_rows *a, lasgd_activation activation, void *stream)
{
    if (!c) return LASGD_ERR_INVALID;
    Gated d;
    TRY(check_gated(c, d, gate, up, rows, cols));
    TRY(check_act(c, activation));
    ProductArgs p = product_args(d, cols, activation);
    bool vx = true, vo = true;
    TRY(check_rows(c, d.v, d.r, "x", x, cols, d.es, false, p.x, vx));
    CHECK(!g == !u, LASGD_ERR_INVALID, "g and u are given together or not at all");
    if (g) {
        TRY(check_rows(c, d.v, d.r, "g", g, d.wide, d.es, true, p.g, vo));
        TRY(check_rows(c, d.v, d.r, "u", u, d.wide, d.es, true, p.u, vo));
    }
    TRY(check_rows(c, d.v, d.r, "a", a, d.wide, d.es, true, p.a, vo));
    CHECK(d.v.all_bound, LASGD_ERR_STATE, "not every replica is bound");
    TRY(check_device(c, d.v));
    if (!d.r.most) return LASGD_OK;
    weights(p, d, d.v.params, gate, up, cols);
    p.wide_out = vo;
    const auto product = [&](bool go) { return launch_form<FWD>(d, p, streams(d, cols, p.x, vx), vx, cols % 8 == 0, Split{1, 0}, nullptr, (hipStream_t)stream, go); };
    CHECK(d.few_tiles || product(false), LASGD_ERR_UNSUPPORTED, "%s", kTooManyThreads);
    product(true);
    return launched(c);
}

extern "C" lasgd_status lasgd_gated_backward_bytes(lasgd_ctx *c, int32_t gate, int32_t up, const int64_t *rows, int64_t cols, int64_t *bytes)
{
    if (!c) return LASGD_ERR_INVALID;
    Gated d;
    CHECK(bytes, LASGD_ERR_INVALID, "NULL bytes");
    TRY(check_gated(c, d, gate, up, rows, cols));
    *bytes = gated_bytes(d, cols);
    return LASGD_OK;
}

extern "C" lasgd_status lasgd_gated_backward(lasgd_ctx *c, int32_t gate, int32_t up, const int64_t *rows, int64_t cols, const lasgd_rows *x,
                                             const lasgd_rows *g, const lasgd_rows *u, const lasgd_rows *da, const lasgd_rows *dx,
                                             lasgd_activation activation, int32_t accumulate, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (!c) return LASGD_ERR_INVALID;
    Gated d;
    TRY(check_gated(c, d, gate, up, rows, cols));
    TRY(check_act(c, activation));
    ProductArgs p = product_args(d, cols, activation);
    GatesArgs e{};
    RowsAt out{};
    bool vx = true, vg = true, vo = true;
    TRY(check_rows(c, d.v, d.r, "x", x, cols, d.es, false, p.x, vx));
    TRY(check_rows(c, d.v, d.r, "g", g, d.wide, d.es, false, e.g, vg));
    TRY(check_rows(c, d.v, d.r, "u", u, d.wide, d.es, false, e.u, vg));
    TRY(check_rows(c, d.v, d.r, "da", da, d.wide, d.es, false, e.da, vg));
    if (dx) TRY(check_rows(c, d.v, d.r, "dx", dx, cols, d.es, true, out, vo));
    const int64_t need = gated_bytes(d, cols);
    TRY(check_workspace(c, workspace, workspace_bytes, need));
    CHECK(d.v.all_bound, LASGD_ERR_STATE, "not every replica is bound");
    TRY(check_device(c, d.v));
    if (!d.r.most && accumulate) return LASGD_OK;
    const hipStream_t st = (hipStream_t)stream;
    e.dg = (char *)workspace;
    e.du = e.dg + gates_bytes(d);
    p.dg = e.dg;
    p.du = e.du;
    const bool big = streams(d, cols, p.x, vx);
    ProductArgs q = p;
    q.a = out;
    weights(q, d, d.v.params, gate, up, cols);
    q.wide_out = vo;
    const Split split = big ? dx_split(d, cols) : Split{1, 0};
    float *part = (float *)(e.du + gates_bytes(d));
    p.accumulate = accumulate;
    if (d.r.most <= 1) p.x.ss = cols;                        // no second row: any stride, and with this one the rows end where x does
    weights(p, d, d.v.grads, gate, up, cols);
    const auto rows_product = [&](bool go) { return launch_form<DX>(d, q, big, true, cols % 8 == 0, split, part, st, go); };
    const auto weights_product = [&](bool go) { return launch_form<DW>(d, p, big, true, vx, Split{1, 0}, nullptr, st, go); };
    CHECK(d.few_tiles || ((!dx || rows_product(false)) && weights_product(false)), LASGD_ERR_UNSUPPORTED, "%s", kTooManyThreads);
    if (d.r.most) {
        e.wide = (uint32_t)d.wide;
        e.groups = ceil_div(d.wide, 8);
        e.pitch = (uint32_t)d.pitch;
        e.act = (int32_t)activation;
        copy_rows(e, d.r, d.v.K);
        memcpy(e.first, d.r.first, d.v.K * sizeof(uint32_t));
        const dim3 grid(d.r.most < 4096u ? d.r.most : 4096u, d.v.K);
        row_access(d.v.bf16, vg, 5 * (int64_t)d.r.total * d.pitch * d.es, [&](auto bf16, auto wide) {
            hipLaunchKernelGGL((gates_backward_kernel<bf16, wide>), grid, dim3(256), 0, st, e);
        });
        TRY(launched(c));
    }
    if (dx && d.r.most) {
        rows_product(true);
        TRY(launched(c));
        if (split.count > 1) {
            JoinRowsArgs j{out, part, (uint64_t)d.r.total * cols, split.count, (uint32_t)cols, vo, {}, {}};
            copy_rows(j, d.r, d.v.K);
            memcpy(j.first, d.r.first, d.v.K * sizeof(uint32_t));
            const dim3 grid(d.r.most < 4096u ? d.r.most : 4096u, d.v.K);
            if (d.v.bf16) hipLaunchKernelGGL((join_rows_kernel<true>), grid, dim3(256), 0, st, j);
            else hipLaunchKernelGGL((join_rows_kernel<false>), grid, dim3(256), 0, st, j);
            TRY(launched(c));
        }
    }
    weights_product(true);
    return launched(c);
}
