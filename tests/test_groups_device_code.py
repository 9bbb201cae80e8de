"""The exchanges across lanes of the router limited to groups, as test_moe_device_code checks those of the router (CPU only): they too read
what single instructions in inline assembly wrote."""
from test_device_code import _tool, code_objects  # noqa: F401
from test_moe_device_code import _too_early


def test_exchanges_of_the_groups_wait_for_what_they_read(code_objects):  # noqa: F811
    found, n = [], 0
    for path in code_objects:
        f, c = _too_early(_tool("llvm-objdump", "-d", "--no-show-raw-insn", path), "route_grouped")
        found += f
        n += c
    assert n > 1000
    assert not found, f"{len(found)}, the first: {found[:3]}"
