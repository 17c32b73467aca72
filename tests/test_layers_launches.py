"""The layers' launches, on the CPU: a launch has fewer than 2^32 threads along x. Dropout and norms of more rows than one holds take several, which
cover every row once; a gated block of more tiles is refused before anything is launched."""
import os
import re
import subprocess

import pytest

from paper_2203_13085_amd import binding as B
from paper_2203_13085_amd import build as build_mod
from tests.test_layers_host import _host_object

HERE = os.path.dirname(os.path.abspath(__file__))
MOST = 2 ** 32 - 1


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d, rocm = tmp_path_factory.mktemp("launches"), os.environ.get("ROCM_PATH", "/opt/rocm")
    images = [_host_object(os.path.join(HERE, "dispatch", "launches.cpp"), str(d / "calls.o")), _host_object(build_mod.LAYERS_SRC, str(d / "layers.o"))]
    (d / "image.c").write_text("".join(f"const char {n}[4096] __attribute__((aligned(4096))) = {{0}};\n" for n in sorted(set(images))))
    subprocess.check_call(["g++", "-no-pie", "-o", str(d / "calls"), str(d / "calls.o"), str(d / "layers.o"), "-x", "c", str(d / "image.c"), "-x", "none",
                           f"-L{rocm}/lib", "-lamdhip64", f"-Wl,-rpath,{rocm}/lib"])

    def f(what, storage, cols, wide, at, rows):
        """(status, [(workgroups, threads, first row), ...])"""
        env = dict(os.environ, HIP_VISIBLE_DEVICES="", ROCR_VISIBLE_DEVICES="")
        out = subprocess.check_output([str(d / "calls"), what, storage, *map(str, (cols, wide, at)), *map(str, rows)], text=True, env=env).split("\n")
        return int(out[0]), [tuple(map(int, line.split())) for line in out[1:] if line]
    return f


@pytest.mark.parametrize("what,storage,cols,each,rows", [
    ("norm", "bf16", 8, 16, [2 ** 28 + 5]), ("norm", "f32", 1, 16, [2 ** 28 - 16]), ("norm", "bf16", 7, 16, [2 ** 28 - 15]), ("norm8", "bf16", 128, 16, [5, 2 ** 28 + 3]),
    ("norm", "bf16", 136, 4, [2 ** 26 + 1]), ("norm", "bf16", 2056, 1, [2 ** 24 - 1]), ("norm", "bf16", 2056, 1, [2 ** 24]), ("norm8", "bf16", 16384, 1, [3, 2 ** 22]),
    ("norm", "bf16", 8, 16, [2 ** 31 - 1]), ("norm", "f32", 16384, 1, [7, 2 ** 22 - 1]), ("dropout", "bf16", 2041, 4, [2 ** 26 - 4]), ("dropout", "bf16", 2041, 4, [2 ** 26 + 1]),
    ("dropout", "bf16", 8, 1024, [2 ** 31 - 1]), ("norm", "bf16", 8, 16, [300, 0, 17])])
def test_every_row_is_in_one_launch(ask, what, storage, cols, each, rows):
    st, launches = ask(what, storage, cols, 8, 4096, rows)
    assert st == B.OK
    at = 0
    for blocks, threads, row0 in launches:
        assert 0 < blocks * threads <= MOST and row0 == at
        at += blocks * each
    assert at - each < max(rows) <= at
    threads = launches[0][1]
    assert len(launches) == -(-(-(-max(rows) // each)) // (MOST // threads))            # and no more than it takes


# rows, columns, hidden columns, address of x: either side of a product's line
LINES = [
    ("gated", "bf16", 7, 8, 4098, [(2 ** 18 - 1) * 128] + [0] * 63, True),               # 64 times the tiles of the replica with all the rows
    ("gated", "bf16", 7, 8, 4098, [(2 ** 18 - 1) * 128 + 1] + [0] * 63, False),
    ("gated", "f32", 8, 8, 4096, [2 ** 30], True),                                       # aligned: 2^23 tiles of its own
    ("gated", "f32", 8, 8, 4096, [2 ** 31 - 1], False),                                  # 2^24
    ("gated", "f32", 8, 8, 4096, [2 ** 31 - 129], True),
    ("gated", "bf16", 8, 8, 4096, [2 ** 31 - 257], True),                                # of 256: 2^23 - 1
    ("gated", "bf16", 8, 8, 4096, [2 ** 31 - 256], True),
    ("gated", "bf16", 8, 8, 4096, [2 ** 31 - 255], False),
    ("gated_back", "bf16", 8, 8, 4096, [2 ** 31 - 255], False),                          # dx; the weights' product has two tiles
    ("gated_back_weights", "bf16", 8, 8, 4096, [2 ** 31 - 255], True),
    ("gated_back_weights", "f32", 8, 2 ** 30, 4096, [1], True),                          # 2^23 tiles of each weight's
    ("gated_back_weights", "f32", 8, 2 ** 30 - 127, 4096, [1], True),
    ("gated_back_weights", "f32", 8, 2 ** 30, 4096, [1, 1], False),
    ("gated_back_weights", "f32", 8, 2 ** 30 - 128, 4096, [1, 1], True),
    ("gated_back", "f32", 8, 2 ** 30, 4096, [1, 1], False),
]


@pytest.mark.parametrize("what,storage,cols,wide,at,rows,goes", LINES)
def test_a_product_beyond_a_launch_is_refused_before_the_first(ask, what, storage, cols, wide, at, rows, goes):
    st, launches = ask(what, storage, cols, wide, at, rows)
    if goes:
        assert st == B.OK and launches and all(0 < blocks * threads <= MOST for blocks, threads, _ in launches)
    else:
        assert st == B.ERR_UNSUPPORTED and not launches


def test_every_product_kernel_can_be_reached(tmp_path):
    """Aligned sides imply each other (an aligned x whole eights of columns; dg and du always are), so no kernel is there for the rest."""
    obj = str(tmp_path / "layers.o")
    _host_object(build_mod.LAYERS_SRC, obj)
    names = set(re.findall(r"__device_stub__product_kernel<(.*?)>\(", subprocess.check_output(["nm", "-C", obj], text=True)))
    forms = [(0, a, b) for a, b in (("true", "true"), ("false", "true"), ("false", "false"))] + [(f, "true", b) for f in (1, 2) for b in ("true", "false")]
    assert names == {f"{t}, {f}, {a}, {b}, {tile}u" for t in ("true", "false") for f, a, b in forms for tile in (64, 128)}


def test_two_workgroups_of_the_large_fp32_tile_fit_on_a_cu(tmp_path):
    """Registers and LDS of the unaligned product, whose second accumulator is a quarter of them."""
    src, out = str(tmp_path / "kernels.hip"), str(tmp_path / "kernels.s")
    root = os.path.dirname(HERE)
    with open(src, "w") as f:
        f.write(f'#include "{root}/paper_2203_13085_amd/csrc/lasgd_gated.hip.h"\nnamespace lasgd {{\n' + "".join(
            f"template __global__ void product_kernel<false, {form}, {m}, false, 128>(const ProductArgs);\n" for form, m in (("FWD", "false"), ("DX", "true"), ("DW", "true"))) + "}\n")
    flags = [f for f in build_mod.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.check_call([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + flags + ["--cuda-device-only", "-S", "-o", out, src], stderr=subprocess.DEVNULL)
    text = open(out).read()
    vgprs, lds = ([int(v) for v in re.findall(r"\.amdhsa_%s (\d+)" % name, text)] for name in ("next_free_vgpr", "group_segment_fixed_size"))
    assert len(vgprs) == len(lds) == 3 and max(vgprs) <= 256 and max(lds) <= 80 << 10
    assert re.findall(r"\.amdhsa_private_segment_fixed_size (\d+)", text) == ["0"] * 3
