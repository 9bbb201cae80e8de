"""What the router's and the products' sources assume of their machine code (CPU only).

The router's sorting networks are written as single instructions in inline assembly, between which the compiler puts the exchanges
across lanes (DPP): such an exchange may read a register two wait states after the instruction that wrote it at the earliest, and
the compiler has to see to that across the inline assembly.  Next to matrix products, whose results arrive many cycles later, no
instruction may stand in inline assembly at all."""
import os
import re

import paper_2606_01007_amd as tacg
from test_device_code import _registers, _tool, code_objects  # noqa: F401

CSRC = os.path.join(os.path.dirname(tacg.__file__), "csrc")


def _too_early(listing, kernel):
    """Exchanges of `kernel`s that read a register written less than two wait states before, and how many there are."""
    found, n, name, before = [], 0, None, []
    for line in listing.splitlines():
        m = re.match(r"^[0-9a-f]+ <(\S+)>:", line)
        if m:
            name, before = m.group(1), []
            continue
        ins = line.split("//")[0].strip()
        if not ins or name is None or kernel not in name:
            continue
        op, _, rest = ins.partition(" ")
        if "_dpp" in op:
            n += 1
            source = _registers(rest.split(",")[1])
            states = 0
            for earlier in reversed(before):
                eop, _, erest = earlier.partition(" ")
                if eop == "s_nop":
                    states += int(erest, 0) + 1
                elif states < 2 and eop.startswith("v_") and _registers(erest.split(",")[0]) & source:
                    found.append((name, earlier, ins))
                    break
                else:
                    states += 1
                if states >= 2:
                    break
        before = (before + [ins])[-4:]
    return found, n


def test_exchanges_wait_for_what_they_read(code_objects):  # noqa: F811
    found, n = [], 0
    for path in code_objects:
        f, c = _too_early(_tool("llvm-objdump", "-d", "--no-show-raw-insn", path), "route_main")
        found += f
        n += c
    assert n > 1000
    assert not found, f"{len(found)}, the first: {found[:3]}"


def test_the_check_sees_an_early_exchange():
    head = "0000000000001000 <route_main>:\n\tv_max_f32_e32 v3, v1, v2\n"
    late = "\tv_mov_b32_dpp v4, v3 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n"
    assert _too_early(head + late, "route_main")[0]
    assert _too_early(head + "\ts_nop 0\n" + late, "route_main")[0]
    assert not _too_early(head + "\ts_nop 1\n" + late, "route_main")[0]
    assert not _too_early(head + "\tv_add_f32_e32 v5, v1, v1\n\tv_add_f32_e32 v6, v1, v1\n" + late, "route_main")[0]


def test_no_instruction_in_inline_assembly_next_to_the_matrix_products():
    text = open(os.path.join(CSRC, "q4_kernels.h")).read()
    assert "mfma" in text
    for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(\s*\"([^\"]*)\"", text):
        assert m.group(1) == "", m.group(0)
