"""CPU checks of gradient norms and clipping: the argument structure, refusals before any device call, the host's rules, and the
generated code of the kernels."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2203_13085_amd import binding as B
from paper_2203_13085_amd import build as build_mod

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_clip_structure_matches_the_header():
    text = open(os.path.join(ROOT, "include", "lasgd.h")).read()
    body = re.search(r"typedef struct \{([^{}]*)\} lasgd_clip;", text, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    assert re.findall(r"(\w+)\s*;", body) == [f for f, _ in B.Clip._fields_]
    assert ctypes.sizeof(B.Clip) == 16
    eps = float(re.search(r"#define LASGD_CLIP_EPS (\S+)", text).group(1))
    kernels = open(os.path.join(ROOT, "paper_2203_13085_amd", "csrc", "lasgd_clip.hip.h")).read()
    assert eps == 1e-6 and "LASGD_CLIP_EPS" in kernels


def test_calls_without_a_context_are_refused():
    L = B.load()
    clip = B.Clip(1.0, 0, None)
    ref, lrs = ctypes.byref(clip), (ctypes.c_float * 2)(0.1, 0.1)
    assert L.lasgd_grad_norms(None, 1, 64) == B.ERR_INVALID
    assert L.lasgd_clip_grads(None, 1, ref) == B.ERR_INVALID
    assert L.lasgd_local_step_clip(None, lrs, 1, ref) == B.ERR_INVALID
    assert L.lasgd_step_merge_clip(None, lrs, 1, 1, 1, ref) == B.ERR_INVALID
    assert L.lasgd_sgd_ar_step_clip(None, 0.1, ref) == B.ERR_INVALID


RULES = r'''
#include "%s/paper_2203_13085_amd/csrc/lasgd.hip"
#include <cstdlib>
int main(int argc, char **argv)
{
    const std::string what = argv[1];
    const uint64_t a = strtoull(argv[2], nullptr, 10), b = strtoull(argv[3], nullptr, 10);
    const bool bf16 = !strcmp(argv[4], "bf16");
    lasgd_ctx c;
    c.storage = bf16 ? LASGD_BF16 : LASGD_F32;
    if (what == "groups") {            // every number of replicas: one workgroup at least, no more than there is room for, and runs for all of them
        for (uint32_t k = 1; k <= 64; ++k) {
            const uint32_t n = norm_groups(bf16, (uint32_t)a, k), runs = (uint32_t)((a + kNormRun - 1) / kNormRun);
            if (n < 1 || n > kNormParts || n > runs || (n < runs && n < 256u / 64u)) return printf("replicas %%u: %%u\n", k, n), 1;
        }
        const uint32_t m = mean_norm_groups((uint32_t)a);
        if (m < 8 || m %% 8 || m > kMeanParts || m > kNormParts) return printf("mean: %%u\n", m), 1;
        printf("ok\n");
    } else if (what == "batch") {      // a = elements a replica, b = replicas
        c.packed = a;
        printf("%%u\n", norm_batch(&c, (uint32_t)b));
    } else if (what == "take") {       // a = mask, b = how many at a time: the parts are disjoint, in order, and make up the mask
        uint64_t left = a, sum = 0, last = 0;
        while (left) {
            const uint64_t t = take_replicas(left, (uint32_t)b);
            if (!t || (t & sum) || (t & ~a) || (last && (t & -t) < last) || (uint32_t)__builtin_popcountll(t) > b || (left && (uint32_t)__builtin_popcountll(t) != b)) return printf("part %%llx\n", (unsigned long long)t), 1;
            sum |= t;
            last = t;
        }
        printf(sum == a ? "ok\n" : "lost\n");
    } else return 2;
    return 0;
}
'''


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("clip_rules")
    hipcc, rocm = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), os.environ.get("ROCM_PATH", "/opt/rocm")
    src, obj, exe = str(d / "rules.cpp"), str(d / "rules.o"), str(d / "rules")
    with open(src, "w") as f:
        f.write(RULES % ROOT)
    subprocess.check_call([hipcc, "--offload-arch=gfx950", "--cuda-host-only", "-O0", "-std=c++17", "-x", "hip", "-c", "-o", obj, src],
                          stderr=subprocess.DEVNULL)
    name = re.search(r" U (__hip_fatbin\S*)", subprocess.check_output(["nm", obj], text=True)).group(1)       # the kernels' image, which nothing asks for
    (d / "image.c").write_text(f"const char {name}[4096] __attribute__((aligned(4096))) = {{0}};\n")
    subprocess.check_call(["g++", "-no-pie", "-o", exe, obj, "-x", "c", str(d / "image.c"), "-x", "none", f"-L{rocm}/lib", "-lamdhip64", f"-Wl,-rpath,{rocm}/lib"])

    def f(*args):
        r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True)
        assert r.returncode == 0, r.stdout
        return r.stdout.split()
    return f


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("tiles", [1, 2, 48, 63, 64, 65, 128, 4096, 99_867, 8_384_512])
def test_workgroups_of_the_norms(ask, tiles, storage):
    assert ask("groups", tiles, 0, storage) == ["ok"]


@pytest.mark.parametrize("n,K,storage,batch", [
    (25_600_000, 8, "f32", 8),                   # fp32: always all at once
    (1 << 30, 3, "f32", 3),
    (25_600_000, 32, "bf16", 8),                 # 1638 MB: four batches
    (25_600_000, 8, "bf16", 8),                  # 410 MB: one
    (29_959_168, 7, "bf16", 7), (29_959_424, 7, "bf16", 4),          # 400 MiB, and a row more
    (1 << 30, 3, "bf16", 1),                     # a replica alone is beyond the batch
    (256, 64, "bf16", 64)])
def test_batches(ask, n, K, storage, batch):
    assert ask("batch", n, K, storage) == [str(batch)]


@pytest.mark.parametrize("mask,count", [(1, 1), (0xFF, 3), (0xFFFFFFFFFFFFFFFF, 5), (0x8000000000000001, 1), (0xA5A5A5A5A5A5A5A5, 7), (0xFFFFFFFFFFFFFFFF, 64)])
def test_batches_take_every_replica_once(ask, mask, count):
    assert ask("take", mask, count, "f32") == ["ok"]


# ---- generated code -------------------------------------------------------------------------------------------------------
KERNELS = r'''
#include "%s/paper_2203_13085_amd/csrc/lasgd_clip.hip.h"
namespace lasgd {
template __global__ void grad_norm_kernel<false, 1>(const ApplyArgs, const NormArgs);
template __global__ void grad_norm_kernel<true, 1>(const ApplyArgs, const NormArgs);
template __global__ void scale_grads_kernel<false, 3>(const ApplyArgs, const NormArgs);
template __global__ void scale_grads_kernel<true, 3>(const ApplyArgs, const NormArgs);
template __global__ void mean_grad_norm_kernel<false, 3>(const ApplyArgs, const NormArgs);
template __global__ void small_step_kernel<false>(const ApplyArgs, const ExtArgs, const NormArgs);
template __global__ void small_update_kernel<true>(const ApplyArgs, const ExtArgs, const NormArgs);
template __global__ void apply_clip_kernel<OP_STEP, false, 3>(const ApplyArgs, const Clip *);
template __global__ void apply_clip_kernel<OP_STEP_MERGE, true, 3>(const ApplyArgs, const Clip *);
template __global__ void apply_clip_ext_kernel<OP_STEP, true, 3>(const ApplyArgs, const ExtArgs, const Clip *);
}
'''


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    d = tmp_path_factory.mktemp("clip_isa")
    src, out = str(d / "kernels.hip"), str(d / "kernels.s")
    with open(src, "w") as f:
        f.write(KERNELS % ROOT)
    flags = [f for f in build_mod.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.check_call([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + flags + ["--cuda-device-only", "-S", "-o", out, src], stderr=subprocess.DEVNULL)
    return open(out).read()


def _kernels(asm, name):
    return [asm[m.start():asm.index(".end_amdhsa_kernel", m.start())] for m in re.finditer(r"\n_ZN5lasgd\d+%s\S*:" % name, asm)]


@pytest.mark.parametrize("name,vgprs", [("grad_norm_kernel", 64), ("scale_grads_kernel", 64), ("mean_grad_norm_kernel", 128), ("small_step_kernel", 128),
                                        ("small_update_kernel", 128), ("apply_clip_kernel", 64), ("apply_clip_ext_kernel", 64)])
def test_kernels_stay_in_registers(asm, name, vgprs):
    """No scratch, 128-bit GLOBAL accesses, room for the waves that the launch counts on (1024 threads: 128 registers)."""
    bodies = _kernels(asm, name)
    assert bodies
    for body in bodies:
        assert re.search(r"\.amdhsa_private_segment_fixed_size 0\b", body)
        assert not re.search(r"\b(scratch|flat)_(load|store)", body)
        assert re.search(r"global_load_dwordx4", body)
        assert int(re.search(r"\.amdhsa_next_free_vgpr (\d+)", body).group(1)) <= vgprs


def test_norms_leave_the_caches_alone(asm):
    """Shares and counters go by atomics of device scope; an acquire or a release there would write back or invalidate the XCD's L2 once a
    workgroup, which made the norms six times as long."""
    for body in _kernels(asm, "grad_norm_kernel") + _kernels(asm, "mean_grad_norm_kernel"):
        assert not re.search(r"buffer_(wbl2|inv)", body)
        join = re.search(r"global_store_dwordx2 [^\n]* sc1\n(.*?)global_atomic_add", body, flags=re.S).group(1)
        assert "s_waitcnt vmcnt(0)" in join and "s_barrier" not in join              # the share is in memory before its arrival counts
        assert re.search(r"v_fma_f64", body)
    assert not re.search(r"v_pk_(add|mul|fma)_f32", asm)
