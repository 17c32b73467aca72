"""CPU checks of the layers' entry points: the argument structures, every refusal before any device call, the host's rules, and the generated code."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2203_13085_amd import binding as B
from paper_2203_13085_amd import build as build_mod

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _fields(text, name):
    body = re.search(r"typedef struct \{([^{}]*)\} %s;" % name, text, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    return [f for line in re.findall(r"([^;]+);", body) for f in re.findall(r"(\w+)\s*(?:,|$)", line.strip())]


def test_structures_match_the_header():
    text = open(os.path.join(ROOT, "include", "lasgd.h")).read()
    assert _fields(text, "lasgd_rows") == [f for f, _ in B.Rows._fields_] and ctypes.sizeof(B.Rows) == 24
    assert _fields(text, "lasgd_drop") == [f for f, _ in B.Drop._fields_] and ctypes.sizeof(B.Drop) == 32
    for name, value in (("SILU", B.SILU), ("GELU", B.GELU), ("GELU_TANH", B.GELU_TANH), ("RELU", B.RELU)):
        assert re.search(r"LASGD_%s = %d\b" % (name, value), text)


def test_calls_without_a_context_are_refused():
    L = B.load()
    n, r, d, out = (ctypes.c_int64 * 1)(1), ctypes.byref(B.Rows(64, 0, 0)), ctypes.byref(B.Drop(0.0, 0, 0, None)), ctypes.c_int64(0)
    assert L.lasgd_dropout(None, n, 8, r, None, r, d, None) == B.ERR_INVALID
    assert L.lasgd_rms_norm(None, 0, n, r, None, None, r, None, 1e-6, d, None) == B.ERR_INVALID
    assert L.lasgd_rms_norm_backward(None, 0, n, r, r, None, None, r, 1e-6, d, 1, None, 0, None) == B.ERR_INVALID
    assert L.lasgd_rms_norm_backward_bytes(None, 0, n, ctypes.byref(out)) == B.ERR_INVALID
    assert L.lasgd_gated(None, 0, 0, n, 8, r, None, None, r, 0, None) == B.ERR_INVALID
    assert L.lasgd_gated_backward(None, 0, 0, n, 8, r, r, r, r, r, 0, 1, None, 0, None) == B.ERR_INVALID
    assert L.lasgd_gated_backward_bytes(None, 0, 0, n, 8, ctypes.byref(out)) == B.ERR_INVALID


# A context without a device: tensors of 8, 8 x 16, 8 x 16, 2 x 4 x 8 (as one) and 20000 elements, three replicas. A call that is not refused
# gets as far as asking for the current device, and ends with HIP here.
CALLS = r'''
#include "%s/paper_2203_13085_amd/csrc/lasgd.hip"
#include <cstdlib>
#include <functional>
#include <map>
static int64_t rows[3] = {4, 0, 2};
static lasgd_rows ok8 = {(void *)4096, 64, 8}, ok16 = {(void *)8192, 128, 16}, wide = {(void *)65536, 200000, 20000};
static lasgd_drop half = {0.5f, 1, 2, nullptr}, none = {0.f, 0, 0, nullptr};
static void *const ws = (void *)(1 << 20);
int main(int argc, char **argv)
{
    lasgd_ctx c;
    c.K = 3;
    c.all = 7;
    c.storage = !strcmp(argv[2], "bf16") ? LASGD_BF16 : LASGD_F32;
    c.numel = {8, 128, 128, 64, 20000, 100};
    c.n_tensors = 6;
    c.h_xptr.assign(18, (void *)4096);
    c.h_gptr.assign(18, (void *)4096);
    c.n_bound = argc > 3 ? 2 : 3;
    const auto drop = [&](const int64_t *r, int64_t cols, const lasgd_rows *x, const lasgd_rows *res, const lasgd_rows *y, const lasgd_drop *d) {
        return lasgd_dropout(&c, r, cols, x, res, y, d, nullptr); };
    const auto norm = [&](int32_t t, const int64_t *r, const lasgd_rows *x, const lasgd_rows *y, const lasgd_rows *sc, float eps, const lasgd_drop *d) {
        return lasgd_rms_norm(&c, t, r, x, nullptr, nullptr, y, sc, eps, d, nullptr); };
    const auto back = [&](int32_t t, const lasgd_rows *h, const lasgd_rows *dx, void *w, int64_t n) {
        return lasgd_rms_norm_backward(&c, t, rows, h, &ok8, nullptr, nullptr, dx, 1e-6f, &none, 1, w, n, nullptr); };
    const auto gated = [&](int32_t g, int32_t u, int64_t cols, const lasgd_rows *x, const lasgd_rows *gg, const lasgd_rows *uu, const lasgd_rows *a, int act) {
        return lasgd_gated(&c, g, u, rows, cols, x, gg, uu, a, (lasgd_activation)act, nullptr); };
    const auto gback = [&](const lasgd_rows *x, const lasgd_rows *da, const lasgd_rows *dx, void *w, int64_t n) {
        return lasgd_gated_backward(&c, 1, 2, rows, 16, x, &ok8, &ok8, da, dx, LASGD_SILU, 1, w, n, nullptr); };
    int64_t nb = 0, ng = 0;
    if (lasgd_rms_norm_backward_bytes(&c, 0, rows, &nb) || lasgd_gated_backward_bytes(&c, 1, 2, rows, 16, &ng) || nb <= 0 || ng <= 0) return 3;
    int64_t negative[3] = {1, -1, 1}, many[3] = {1, 0x7fffffff, 0}, zero[3] = {0, 0, 0}, one[3] = {0, 9, 0}, huge[3] = {0x7ffffff0, 0, 0};
    const lasgd_rows null = {nullptr, 64, 8}, odd = {(void *)4097, 64, 8}, minus = {(void *)4096, -64, 8}, minus2 = {(void *)4096, 64, -8}, over = {(void *)4096, 64, 7},
                     same = {(void *)4096, 31, 8}, far = {(void *)4096, 1ll << 46, 8}, turned = {(void *)4096, 8, 24}, turned2 = {(void *)4096, 8, 23}, shared = {(void *)4096, 0, 8},
                     broad = {(void *)4096, 0, 0}, scales = {(void *)512, 4, 1}, scales2 = {(void *)512, 3, 1}, scales3 = {(void *)514, 4, 1};
    lasgd_drop d = half;
    const std::string what = argv[1];
    std::map<std::string, std::function<int()>> f = {
        {"drop", [&] { return drop(rows, 8, &ok8, &ok8, &ok8, &half); }},
        {"drop none", [&] { return drop(rows, 8, &ok8, nullptr, &ok8, &none); }},
        {"drop turned", [&] { return drop(rows, 8, &ok8, nullptr, &turned, &half); }},
        {"drop shared input", [&] { return drop(rows, 8, &shared, &broad, &ok8, &half); }},
        {"drop no rows", [&] { return drop(zero, 8, &null, nullptr, &null, &half); }},
        {"drop one replica", [&] { return drop(one, 8, &ok8, nullptr, &shared, &half); }},
        {"drop rows NULL", [&] { return drop(nullptr, 8, &ok8, nullptr, &ok8, &half); }},
        {"drop rows negative", [&] { return drop(negative, 8, &ok8, nullptr, &ok8, &half); }},
        {"drop rows many", [&] { return drop(many, 8, &shared, nullptr, &ok8, &half); }},
        {"drop cols 0", [&] { return drop(rows, 0, &ok8, nullptr, &ok8, &half); }},
        {"drop x NULL", [&] { return drop(rows, 8, nullptr, nullptr, &ok8, &half); }},
        {"drop y NULL", [&] { return drop(rows, 8, &ok8, nullptr, nullptr, &half); }},
        {"drop data NULL", [&] { return drop(rows, 8, &null, nullptr, &ok8, &half); }},
        {"drop drop NULL", [&] { return drop(rows, 8, &ok8, nullptr, &ok8, nullptr); }},
        {"drop misaligned", [&] { return drop(rows, 8, &odd, nullptr, &ok8, &half); }},
        {"drop minus", [&] { return drop(rows, 8, &minus, nullptr, &ok8, &half); }},
        {"drop minus2", [&] { return drop(rows, 8, &ok8, &minus2, &ok8, &half); }},
        {"drop rows overlap", [&] { return drop(rows, 8, &ok8, nullptr, &over, &half); }},
        {"drop replicas overlap", [&] { return drop(rows, 8, &ok8, nullptr, &same, &half); }},
        {"drop replicas overlap turned", [&] { return drop(rows, 8, &ok8, nullptr, &turned2, &half); }},
        {"drop output shared", [&] { return drop(rows, 8, &ok8, nullptr, &shared, &half); }},
        {"drop far", [&] { return drop(rows, 8, &far, nullptr, &ok8, &half); }},
        {"drop p negative", [&] { d.p = -0.1f; return drop(rows, 8, &ok8, nullptr, &ok8, &d); }},
        {"drop p above", [&] { d.p = 1.1f; return drop(rows, 8, &ok8, nullptr, &ok8, &d); }},
        {"drop p NaN", [&] { d.p = NAN; return drop(rows, 8, &ok8, nullptr, &ok8, &d); }},
        {"drop counter", [&] { d.counter = (const uint64_t *)4; return drop(rows, 8, &ok8, nullptr, &ok8, &d); }},
        {"drop groups", [&] { return drop(huge, 0x7fffffff, &broad, nullptr, &broad, &half); }},
        {"norm", [&] { return norm(0, rows, &ok8, &ok8, nullptr, 1e-6f, &half); }},
        {"norm no drop", [&] { return norm(0, rows, &ok8, &ok8, nullptr, 0.f, nullptr); }},
        {"norm 8 bits", [&] { return norm(0, rows, &ok8, &ok8, &scales, 1e-6f, &none); }},
        {"norm 8 bits odd", [&] { return norm(0, rows, &ok8, &odd, &scales, 1e-6f, &none); }},
        {"norm tensor", [&] { return norm(6, rows, &ok8, &ok8, nullptr, 1e-6f, &none); }},
        {"norm tensor negative", [&] { return norm(-1, rows, &ok8, &ok8, nullptr, 1e-6f, &none); }},
        {"norm long", [&] { return norm(4, rows, &wide, &wide, nullptr, 1e-6f, &none); }},
        {"norm eps", [&] { return norm(0, rows, &ok8, &ok8, nullptr, -1.f, &none); }},
        {"norm eps NaN", [&] { return norm(0, rows, &ok8, &ok8, nullptr, NAN, &none); }},
        {"norm scales overlap", [&] { return norm(0, rows, &ok8, &ok8, &scales2, 1e-6f, &none); }},
        {"norm scales misaligned", [&] { return norm(0, rows, &ok8, &ok8, &scales3, 1e-6f, &none); }},
        {"norm y NULL", [&] { return norm(0, rows, &ok8, nullptr, nullptr, 1e-6f, &none); }},
        {"back", [&] { return back(0, &ok8, &ok8, ws, nb); }},
        {"back not wanted", [&] { return back(0, &ok8, nullptr, ws, nb); }},
        {"back workspace", [&] { return back(0, &ok8, &ok8, ws, nb - 1); }},
        {"back workspace NULL", [&] { return back(0, &ok8, &ok8, nullptr, nb); }},
        {"back workspace misaligned", [&] { return back(0, &ok8, &ok8, (char *)ws + 8, nb); }},
        {"back h NULL", [&] { return back(0, nullptr, &ok8, ws, nb); }},
        {"back dx overlap", [&] { return back(0, &ok8, &same, ws, nb); }},
        {"gated", [&] { return gated(1, 2, 16, &ok16, &ok8, &ok8, &ok8, 0); }},
        {"gated packed", [&] { return gated(3, 3, 8, &ok8, nullptr, nullptr, &ok8, 3); }},
        {"gated tensor", [&] { return gated(1, 9, 16, &ok16, nullptr, nullptr, &ok8, 0); }},
        {"gated unlike", [&] { return gated(1, 3, 16, &ok16, nullptr, nullptr, &ok8, 0); }},
        {"gated cols", [&] { return gated(1, 2, 17, &ok16, nullptr, nullptr, &ok8, 0); }},
        {"gated packed cols", [&] { return gated(5, 5, 20, &ok16, nullptr, nullptr, &ok8, 0); }},
        {"gated cols 0", [&] { return gated(1, 2, 0, &ok16, nullptr, nullptr, &ok8, 0); }},
        {"gated g alone", [&] { return gated(1, 2, 16, &ok16, &ok8, nullptr, &ok8, 0); }},
        {"gated act", [&] { return gated(1, 2, 16, &ok16, nullptr, nullptr, &ok8, 4); }},
        {"gated act negative", [&] { return gated(1, 2, 16, &ok16, nullptr, nullptr, &ok8, -1); }},
        {"gated a overlap", [&] { return gated(1, 2, 16, &ok16, nullptr, nullptr, &over, 0); }},
        {"gback", [&] { return gback(&ok16, &ok8, &ok16, ws, ng); }},
        {"gback not wanted", [&] { return gback(&ok16, &ok8, nullptr, ws, ng); }},
        {"gback workspace", [&] { return gback(&ok16, &ok8, &ok16, ws, ng - 1); }},
        {"gback da NULL", [&] { return gback(&ok16, nullptr, &ok16, ws, ng); }},
        {"gback dx overlap", [&] { return gback(&ok16, &ok8, &ok8, ws, ng); }},
        {"bytes NULL", [&] { return lasgd_gated_backward_bytes(&c, 1, 2, rows, 16, nullptr); }},
        {"bytes NULL norm", [&] { return lasgd_rms_norm_backward_bytes(&c, 0, rows, nullptr); }},
    };
    if (what == "list") { for (auto &e : f) printf("%%s\n", e.first.c_str()); return 0; }
    const int st = f.at(what)();
    printf("%%d %%s\n", st, lasgd_last_error(&c));
    return 0;
}
'''
PASSES = {"drop", "drop none", "drop turned", "drop shared input", "drop no rows", "drop one replica", "norm", "norm no drop", "norm 8 bits", "back",
          "back not wanted", "gated", "gated packed", "gback", "gback not wanted"}
UNSUPPORTED = {"drop rows many", "drop groups", "norm long"}


def _host_object(src, obj):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.check_call([hipcc, "--offload-arch=gfx950", "--cuda-host-only", "-O0", "-std=c++17", "-x", "hip", "-c", "-o", obj, src], stderr=subprocess.DEVNULL)
    return re.search(r" U (__hip_fatbin\S*)", subprocess.check_output(["nm", obj], text=True)).group(1)       # the kernels' image, which nothing asks for


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    d, rocm = tmp_path_factory.mktemp("layers"), os.environ.get("ROCM_PATH", "/opt/rocm")
    (d / "calls.cpp").write_text(CALLS % ROOT)
    images = [_host_object(str(d / "calls.cpp"), str(d / "calls.o")), _host_object(build_mod.LAYERS_SRC, str(d / "layers.o"))]
    (d / "image.c").write_text("".join(f"const char {n}[4096] __attribute__((aligned(4096))) = {{0}};\n" for n in sorted(set(images))))
    subprocess.check_call(["g++", "-no-pie", "-o", str(d / "calls"), str(d / "calls.o"), str(d / "layers.o"), "-x", "c", str(d / "image.c"), "-x", "none",
                           f"-L{rocm}/lib", "-lamdhip64", f"-Wl,-rpath,{rocm}/lib"])
    return str(d / "calls")


def _call(exe, *args):
    env = dict(os.environ, HIP_VISIBLE_DEVICES="", ROCR_VISIBLE_DEVICES="")
    r = subprocess.run([exe, *args], capture_output=True, text=True, env=env)
    assert r.returncode == 0, (args, r.returncode, r.stderr)
    return r.stdout


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_refusals_come_before_any_device_call(exe, storage):
    names = _call(exe, "list", storage).split("\n")[:-1]
    assert len(names) >= 60 and PASSES | UNSUPPORTED <= set(names)
    for name in names:
        st, text = _call(exe, name, storage).strip("\n").split(" ", 1)
        if name in PASSES or name == "norm 8 bits odd":
            assert int(st) == B.ERR_HIP and "hipGetDevice" in text, (name, st, text)
        else:
            assert int(st) == (B.ERR_UNSUPPORTED if name in UNSUPPORTED else B.ERR_INVALID) and text, (name, st, text)


def test_unbound_replicas_are_refused(exe):
    for name in ("norm", "back", "gated", "gback"):
        assert _call(exe, name, "f32", "unbound").startswith(f"{B.ERR_STATE} ")
    assert _call(exe, "drop", "f32", "unbound").startswith(f"{B.ERR_HIP} ")       # needs no parameters


# ---- generated code -------------------------------------------------------------------------------------------------------
KERNELS = r'''
#include "%s/paper_2203_13085_amd/csrc/lasgd_gated.hip.h"
namespace lasgd {
template __global__ void dropout_kernel<true, STREAM>(const DropoutArgs);
template __global__ void rms_norm_kernel<true, WIDE, 64, 4, false>(const NormRowsArgs);
template __global__ void rms_norm_kernel<false, WIDE, 1024, 2, true>(const NormRowsArgs);
template __global__ void rms_norm_backward_kernel<true, WIDE, 256, 1>(const NormBackArgs);
template __global__ void rms_norm_backward_kernel<false, WIDE, 1024, 2>(const NormBackArgs);
template __global__ void gates_backward_kernel<true, WIDE>(const GatesArgs);
template __global__ void product_kernel<true, FWD, false, false, 128>(const ProductArgs);
template __global__ void product_kernel<false, DW, true, false, 128>(const ProductArgs);
template __global__ void big_product_kernel<true, FWD, 256, 256, 2, 4, 8, 2, false>(const ProductArgs, const TileMap);
template __global__ void big_product_kernel<true, DX, 256, 256, 2, 4, 8, 2, false>(const ProductArgs, const TileMap);
template __global__ void big_product_kernel<true, DW, 256, 256, 2, 4, 8, 2, false>(const ProductArgs, const TileMap);
template __global__ void big_product_kernel<false, DX, 128, 128, 2, 2, 8, 2, false>(const ProductArgs, const TileMap);
template __global__ void big_product_kernel<true, DX, 16, 256, 1, 4, 8, 2, true>(const ProductArgs, const TileMap);
template __global__ void few_rows_weights_kernel<true, STREAM>(const ProductArgs);
}
'''


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    d = tmp_path_factory.mktemp("layers_isa")
    src, out = str(d / "kernels.hip"), str(d / "kernels.s")
    with open(src, "w") as f:
        f.write(KERNELS % ROOT)
    flags = [f for f in build_mod.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.check_call([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + flags + ["--cuda-device-only", "-S", "-o", out, src], stderr=subprocess.DEVNULL)
    text = open(out).read()
    return {m.group(1): text[m.start():text.index(".end_amdhsa_kernel", m.start())] for m in re.finditer(r"\n(_ZN5lasgd\S*):", text)}


def test_kernels_stay_in_registers(asm):
    assert len(asm) == 14
    for name, body in asm.items():
        assert re.search(r"\.amdhsa_private_segment_fixed_size 0\b", body), name
        assert not re.search(r"\b(scratch|flat)_(load|store)", body), name
        assert not re.search(r"v_pk_(add|mul|fma)_f32", body), name


def test_tiles_go_straight_into_lds_and_nothing_waits_for_them_there(asm):
    """From the barrier that says a step is there to its last product, no wait for loads: those under way belong to later steps. (A compiler that takes them for
    what is being read waits for all of them, and a tile takes twice as long.)"""
    big = {n: b for n, b in asm.items() if "big_product" in n}
    assert len(big) == 5
    for name, body in big.items():
        assert re.search(r"buffer_load_dwordx4 [^\n]* lds", body)
        loop = body[body.rindex("s_barrier", 0, body.index("v_mfma")):body.rindex("v_mfma")]
        loop = re.sub(r";;#ASMSTART.*?;;#ASMEND", "", loop, flags=re.S)               # the waits that are written out
        assert len(re.findall("v_mfma", loop)) >= 7, name
        assert not re.search(r"vmcnt", loop), name
        assert re.search("ds_read_b64_tr_b16" if re.search("ILb1ELi[12]E", name) else "ds_read_b128", loop), name


@pytest.mark.parametrize("name,vgprs", [("dropout_kernel", 96), ("rms_norm_kernelILb1E", 72), ("rms_norm_backward_kernelILb1E", 102)])
def test_row_kernels_leave_room_for_waves(asm, name, vgprs):
    """At least five waves a SIMD of a norm's backward pass and of dropout, seven of a norm."""
    bodies = [b for n, b in asm.items() if name in n]
    assert bodies
    for body in bodies:
        assert int(re.search(r"\.amdhsa_next_free_vgpr (\d+)", body).group(1)) <= vgprs
