"""What the compiler cannot look after inside asm blocks, and scratch memory, in the built kernels of the layer, the loss and AdamW; and that the sizes
of the GPU tests reach every kernel.  Needs no GPU."""
import ctypes as C
import os
import re
import subprocess

import pytest

from paper_2011_06295_amd import binding as B, build
from test_kernel_resources import LLVM, _code_objects, _metadata
from test_text_machine_code import _before, _named, _states, _to_lds, _written

LIB = B.raw_library()


@pytest.fixture(scope="module")
def images():
    with open(build.LIB, "rb") as f:
        return [elf for elf in _code_objects(f.read()) if any(name in elf for name in (b"linear_tile_kernel", b"linear_dot_kernel", b"loss_row_kernel", b"adamw_kernel"))]


@pytest.fixture(scope="module")
def product_code(images, tmp_path_factory):
    """Instructions (name, operands) of the kernels that load straight to LDS, one list a kernel."""
    kernels, path = {}, tmp_path_factory.mktemp("code") / "object"
    for elf in images:
        if b"linear_tile_kernel" not in elf:
            continue
        path.write_bytes(elf)
        listing = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn", str(path)], stdout=subprocess.PIPE, text=True, check=True).stdout
        for line in listing.splitlines():
            if m := re.match(r"[0-9a-f]+ <(\S+)>:", line):
                code = kernels.setdefault(m[1], [])
            elif m := re.match(r"\t(\S+) *(.*?) *//", line):
                code.append((m[1], m[2]))
    kernels = {name: code for name, code in kernels.items() if "linear_tile_kernel" in name or "linear_row_kernel" in name}
    assert len(kernels) == 3 * (6 + 5 + 4 + 4) + 2 * 3 - 3          # row kernels, tiles of rows, of turned operands; the largest of 16-bit types alone
    return kernels


def test_loads_to_lds_come_late_enough(product_code):
    """A wait state after m0 is written, five after a vector instruction writes a scalar that they read."""
    loads, early = 0, []
    for kernel, code in product_code.items():
        for at, instruction in enumerate(code):
            if not _to_lds(*instruction):
                continue
            loads += 1
            early += [(kernel, i) for i in _before(code, at, 1) if i[1].startswith("m0,")]
            early += [(kernel, i) for i in _before(code, at, 5) if i[0].startswith("v_") and {r for r in _written(*i) if r[0] == "s"} & _named(instruction[1])]
    assert loads > 0 and not early, early[:4]


def test_products_are_written_and_read_late_enough(product_code):
    """Two wait states between another vector instruction's write and the product that reads it, 18 between a product and what reads or writes its sums."""
    early = []
    for kernel, code in product_code.items():
        if "linear_tile_kernel" not in kernel:
            continue          # (builtins: the compiler's own)
        for at, (name, operands) in enumerate(code):
            if not name.startswith("v_mfma"):
                if name.startswith("v_accvgpr"):
                    mine = {r for r in _named(operands) if r[0] == "a"}
                    early += [(kernel, i, code[at]) for i in _before(code, at, 18) if i[0].startswith("v_mfma") and _written(*i) & mine]
                continue
            early += [(kernel, i, code[at]) for i in _before(code, at, 2) if i[0].startswith("v_") and not i[0].startswith("v_mfma") and _written(*i) & _named(operands)]
    assert not early, early[:4]


def test_no_kernel_uses_scratch(images, tmp_path):
    """(Loads to LDS are waited for by number: a spilled register would be one more.)"""
    kernels = [k for elf in images for k in _metadata(elf, tmp_path / "object") if ".name" in k]
    assert len(kernels) > 150
    used = {k[".name"]: (k[".private_segment_fixed_size"], k[".vgpr_spill_count"]) for k in kernels if k[".private_segment_fixed_size"] != "0" or k[".vgpr_spill_count"] != "0"}
    assert not used, used


@pytest.mark.parametrize("dtype", [B.SC_F32, B.SC_F16, B.SC_BF16])
def test_every_kernel_has_a_layer_and_gradients_in_the_tests(dtype):
    from test_gpu_train import GRADIENTS, LARGE_GRADIENTS, LARGE_LAYERS, LAYERS
    layer, gradient = LIB["_ZN2sc13linear_kernelEiiii"], LIB["_ZN2sc18linear_grad_kernelEiiiii"]          # sc::linear_kernel, sc::linear_grad_kernel
    layer.argtypes, gradient.argtypes = [C.c_int] * 4, [C.c_int] * 5
    reached = {layer(dtype, M, N, K) for M, K, N in LAYERS + LARGE_LAYERS}
    of_x, of_w = set(), set()
    for M, K, N in GRADIENTS + LARGE_GRADIENTS:
        for act in (B.SC_ACT_NONE, B.SC_ACT_GELU):
            kernel = gradient(dtype, M, N, K, act)
            (of_x if kernel < 1000 else of_w).add(kernel if kernel < 1000 else kernel % 1000)
            if kernel >= 1000:
                of_x.add(kernel // 1000)
    print(sorted(reached), sorted(of_x), sorted(of_w))
    largest = set() if dtype == B.SC_F32 else {7}
    assert reached == {0, 1, 2, 3, 4, 5, 6, 8, 9, 10, 100, 101, 103} | largest
    assert of_x >= {5, 6, 8, 101, 102} | largest and of_w >= {5, 6, 8, 10} | largest
