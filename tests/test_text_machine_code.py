"""What the compiler cannot look after inside asm blocks, in the built kernels of the text model's operators.  Needs no GPU."""
import os
import re
import subprocess

import pytest

from paper_2011_06295_amd import build
from test_kernel_resources import LLVM, _code_objects, _metadata


@pytest.fixture(scope="module")
def product_code(tmp_path_factory):
    """Instructions (name, operands) of the kernels that multiply 8-bit integers, one list a kernel."""
    with open(build.LIB, "rb") as f:
        images = [elf for elf in _code_objects(f.read()) if b"row_product_kernel" in elf]
    assert len(images) == 1
    path = tmp_path_factory.mktemp("code") / "object"
    path.write_bytes(images[0])
    listing = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn", str(path)], stdout=subprocess.PIPE, text=True, check=True).stdout
    kernels = {}
    for line in listing.splitlines():
        if m := re.match(r"[0-9a-f]+ <(\S+)>:", line):
            code = kernels.setdefault(m[1], [])
        elif m := re.match(r"\t(\S+) *(.*?) *//", line):
            code.append((m[1], m[2]))
    return {name: code for name, code in kernels.items() if "product_kernel" in name}


def _to_lds(name, operands):
    return name.startswith("buffer_load") and operands.endswith(" lds")


def _written(name, operands):
    """(file, number) of the registers that an instruction's first operand names."""
    first = operands.split(",")[0].strip()
    if m := re.fullmatch(r"([sva])\[(\d+):(\d+)\]", first):
        return {(m[1], i) for i in range(int(m[2]), int(m[3]) + 1)}
    m = re.fullmatch(r"([sva])(\d+)", first)
    return {(m[1], int(m[2]))} if m else set()


def _named(operands):
    """(file, number) of all registers that the operands name."""
    found = {(f, int(n)) for f, n in re.findall(r"\b([sva])(\d+)\b", operands)}
    for f, a, b in re.findall(r"\b([sva])\[(\d+):(\d+)\]", operands):
        found |= {(f, i) for i in range(int(a), int(b) + 1)}
    return found


def _states(name, operands):
    return int(operands, 0) + 1 if name == "s_nop" else 1


def _before(code, at, states):
    """The instructions that lie fewer than `states` wait states before code[at]."""
    passed = 0
    while at > 0 and passed < states:
        at -= 1
        yield code[at]
        passed += _states(*code[at])


def test_a_load_to_lds_comes_a_wait_state_after_the_write_of_m0(product_code):
    loads, early = 0, {}
    for kernel, code in product_code.items():
        for at, instruction in enumerate(code):
            if not _to_lds(*instruction):
                continue
            loads += 1
            if any(operands.startswith("m0,") for _, operands in _before(code, at, 1)):
                early[kernel] = early.get(kernel, 0) + 1
    assert loads > 0 and not early, early


def test_no_vector_instruction_writes_a_load_s_scalars_right_before_it(product_code):
    """Scalars that a vector instruction wrote reach a load from memory five wait states later."""
    early = [(kernel, code[at], i) for kernel, code in product_code.items() for at in range(len(code)) if _to_lds(*code[at])
             for i in _before(code, at, 5) if i[0].startswith("v_") and {r for r in _written(*i) if r[0] == "s"} & _named(code[at][1])]
    assert not early, early[:4]


def test_no_vector_instruction_writes_a_product_s_operands_right_before_it(product_code):
    """Registers that another vector instruction wrote reach the matrix unit two wait states later."""
    early = [(kernel, code[at], i) for kernel, code in product_code.items() for at in range(len(code)) if code[at][0].startswith("v_mfma")
             for i in _before(code, at, 2) if i[0].startswith("v_") and not i[0].startswith("v_mfma") and _written(*i) & _named(code[at][1])]
    assert not early, early[:4]


def test_no_kernel_of_the_text_operators_uses_scratch(tmp_path):
    """(Their loads to LDS are waited for by number: a spilled register would be one more.)"""
    with open(build.LIB, "rb") as f:
        images = [elf for elf in _code_objects(f.read()) if b"row_product_kernel" in elf or b"embed_rows_kernel" in elf]
    kernels = [k for elf in images for k in _metadata(elf, tmp_path / "object") if ".name" in k]
    assert len(images) == 2 and len(kernels) > 60
    used = {k[".name"]: (k[".private_segment_fixed_size"], k[".vgpr_spill_count"]) for k in kernels if k[".private_segment_fixed_size"] != "0" or k[".vgpr_spill_count"] != "0"}
    assert not used, used
