// What the layers' entry points would launch, on the CPU: the library's host side with a device that only writes down what it is
// asked for.  Prints the status and, for each launch, its workgroups along x, threads a workgroup and first row.
#include "../../paper_2203_13085_amd/csrc/lasgd.hip"
#include "../../paper_2203_13085_amd/csrc/lasgd_rows.hip.h"

#include <cstddef>
#include <cstdlib>

struct Launch {
    dim3 grid, block;
    uint64_t row0;
};
static std::vector<Launch> launches;
static size_t row0_at = 0;
static struct {
    dim3 grid, block;
    size_t bytes;
    hipStream_t stream;
} asked;

extern "C" {
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t bytes, hipStream_t st)
{
    asked = {grid, block, bytes, st};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *bytes, hipStream_t *st)
{
    *grid = asked.grid, *block = asked.block, *bytes = asked.bytes, *st = asked.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *, dim3 grid, dim3 block, void **args, size_t, hipStream_t)
{
    uint64_t row0 = 0;
    if (row0_at) memcpy(&row0, (const char *)args[0] + row0_at, sizeof row0);
    launches.push_back({grid, block, row0});
    return hipSuccess;
}
}

// call, storage, columns, hidden columns, x's address, rows of each replica
int main(int argc, char **argv)
{
    if (argc < 7) return 2;
    const std::string what = argv[1];
    const int64_t cols = atoll(argv[3]), wide = atoll(argv[4]), es = !strcmp(argv[2], "bf16") ? 2 : 4;
    void *const at = (void *)(uintptr_t)atoll(argv[5]);
    std::vector<int64_t> rows;
    int64_t most = 0;
    for (int i = 6; i < argc; ++i) {
        rows.push_back(atoll(argv[i]));
        if (rows.back() > most) most = rows.back();
    }
    lasgd_ctx c;
    c.K = (int32_t)rows.size();
    c.storage = es == 2 ? LASGD_BF16 : LASGD_F32;
    c.numel = {cols, wide * cols, wide * cols};
    c.n_tensors = 3;
    c.device = 0;
    c.h_xptr.assign(3 * rows.size(), (void *)4096);
    c.h_gptr.assign(3 * rows.size(), (void *)4096);
    c.n_bound = c.K;
    const lasgd_rows x = {at, most * cols, cols}, h = {(void *)4096, most * wide, wide}, scales = {(void *)4096, most, 1};
    const lasgd_drop drop = {0.5f, 1, 2, nullptr};
    void *const work = (void *)4096;
    int64_t need = 0;
    lasgd_status st = LASGD_ERR_INVALID;
    if (what == "dropout") {
        row0_at = offsetof(DropoutArgs, row0);
        st = lasgd_dropout(&c, rows.data(), cols, &x, nullptr, &x, &drop, nullptr);
    } else if (what == "norm" || what == "norm8") {
        row0_at = offsetof(NormRowsArgs, row0);
        st = lasgd_rms_norm(&c, 0, rows.data(), &x, nullptr, nullptr, &x, what == "norm8" ? &scales : nullptr, 1e-6f, nullptr, nullptr);
    } else if (what == "norm_back") {
        if (lasgd_rms_norm_backward_bytes(&c, 0, rows.data(), &need)) return 3;
        st = lasgd_rms_norm_backward(&c, 0, rows.data(), &x, &x, nullptr, nullptr, &x, 1e-6f, nullptr, 1, work, need, nullptr);
    } else if (what == "gated") {
        st = lasgd_gated(&c, 1, 2, rows.data(), cols, &x, nullptr, nullptr, &h, LASGD_SILU, nullptr);
    } else if (what == "gated_back" || what == "gated_back_weights") {
        if (lasgd_gated_backward_bytes(&c, 1, 2, rows.data(), cols, &need)) return 3;
        st = lasgd_gated_backward(&c, 1, 2, rows.data(), cols, &x, &h, &h, &h, what == "gated_back" ? &x : nullptr, LASGD_SILU, 1, work, need, nullptr);
    }
    printf("%d\n", (int)st);
    for (const Launch &l : launches) printf("%u %u %llu\n", l.grid.x, l.block.x, (unsigned long long)l.row0);
    return 0;
}
