"""Registers of the kernels over a paged cache, from the metadata of every code object in the built library: the state of their main loops stays in registers."""
import struct
import subprocess

import msgpack
import pytest

import paper_2410_01028_amd as asd


def code_objects(lib):
    """The gfx950 code objects of the library, one for each source."""
    at = lib.find(b"__CLANG_OFFLOAD_BUNDLE__")
    while at >= 0:
        entry, n = at + 32, struct.unpack_from("<Q", lib, at + 24)[0]
        for _ in range(n if n < 8 else 0):                                # (the name of the format may be there as text too)
            offset, size, length = struct.unpack_from("<QQQ", lib, entry)
            if b"gfx950" in lib[entry + 24:entry + 24 + length]:
                yield lib[at + offset:at + offset + size]
            entry += 24 + length
        at = lib.find(b"__CLANG_OFFLOAD_BUNDLE__", at + 24)


def kernels_of(elf):
    sections, = struct.unpack_from("<Q", elf, 40)
    each, count = struct.unpack_from("<HH", elf, 58)
    for i in range(count):
        kind, = struct.unpack_from("<I", elf, sections + i * each + 4)
        at, size = struct.unpack_from("<QQ", elf, sections + i * each + 24)
        end = at + size
        while kind == 7 and at < end:                                     # SHT_NOTE
            n_name, n_desc, note = struct.unpack_from("<III", elf, at)
            desc = at + 12 + (n_name + 3) // 4 * 4
            if note == 32 and elf[at + 12:at + 18] == b"AMDGPU":           # NT_AMDGPU_METADATA
                yield from msgpack.unpackb(elf[desc:desc + n_desc])["amdhsa.kernels"]
            at = desc + (n_desc + 3) // 4 * 4


@pytest.fixture(scope="module")
def table():
    found = [k for elf in code_objects(open(asd.LIB_PATH, "rb").read()) for k in kernels_of(elf)]
    names = subprocess.run(["c++filt"], input="\n".join(k[".name"] for k in found), capture_output=True, text=True, check=True).stdout.splitlines()
    return {n.split("(")[0].removeprefix("void "): k for n, k in zip(names, found)}


def test_every_source_is_there(table):
    for name in ("pf_ring_kernel<", "kv_append_kernel<", "kv_attend_kernel<", "kv_rows_kernel<", "kv_window_rows_kernel<", "kv_both_rows_kernel<", "kv_apart_kernel<", "kv_parts_kernel<"):
        assert any(n.startswith(name) for n in table), name


def test_vector_registers_are_not_spilled(table):
    """But for two of the many-row kernels over 8-bit pages at head dim 128, which fill all 256: a value or two that a step with an edge asks for once."""
    spilled = {n: k[".vgpr_spill_count"] for n, k in table.items() if n.startswith("kv_") and k[".vgpr_spill_count"]}
    few = {"kv_window_rows_kernel<FP8, 128, 2, 4>": 2, "kv_both_rows_kernel<FP8, 128, 2, 4>": 2}
    assert {n: s for n, s in spilled.items() if s > few.get(n, 0)} == {}
