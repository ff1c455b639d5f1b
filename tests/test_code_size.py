"""Device functions that are called stay well within the reach of a branch.

A branch reaches 2^15 instruction words (128 KiB) to either side.  Beyond that the compiler jumps through a pair of scalar registers, which in a function that calls no other has been seen to be the
pair that holds its return address: such a call never returns.  Kernels, which return to nobody, may be of any size."""
import os
import struct

import pytest

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_03983_amd", "libtwist.so")
REACH = 4 << 15


def _device_objects(data):
    """The ELF files for the GPU among the bundles of a shared library."""
    magic = b"__CLANG_OFFLOAD_BUNDLE__"
    at = data.find(magic)
    while at >= 0:
        p = at + len(magic)
        (n,) = struct.unpack_from("<Q", data, p)
        p += 8
        for _ in range(n):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24: p + 24 + length]
            p += 24 + length
            if b"amdgcn" in name and size:
                yield data[at + offset: at + offset + size]
        at = data.find(magic, p)


def _functions(elf):
    """(name, size) of an ELF file's functions."""
    (shoff,) = struct.unpack_from("<Q", elf, 0x28)
    entry, count = struct.unpack_from("<HH", elf, 0x3A)
    sections = [struct.unpack_from("<IIQQQQIIQQ", elf, shoff + i * entry) for i in range(count)]
    for s in sections:
        if s[1] not in (2, 11):     # SHT_SYMTAB, SHT_DYNSYM
            continue
        names = sections[s[6]]
        for at in range(s[4], s[4] + s[5], 24):
            name, info, _, _, _, size = struct.unpack_from("<IBBHQQ", elf, at)
            if info & 15 == 2:      # STT_FUNC
                start = names[4] + name
                yield elf[start: elf.index(b"\0", start)].decode(), size


def test_called_device_functions_are_within_the_reach_of_a_branch():
    if not os.path.exists(LIB):
        pytest.skip("the library is not built")
    with open(LIB, "rb") as f:
        data = f.read()
    called, kernels = {}, 0
    for i, elf in enumerate(_device_objects(data)):
        assert elf[:4] == b"\x7fELF"
        functions = dict(_functions(elf))
        for name, size in functions.items():
            if "_kernel" in name or name + ".kd" in functions:
                kernels += 1
            else:
                called[i, name] = size
    assert kernels > 100                                        # the bundles were read
    assert any("draw_of_many" in name for _, name in called)       # and what is called is among them
    assert {n: s for n, s in called.items() if s > REACH * 3 // 4} == {}


def _symbols(elf):
    """(name, type, size) of an ELF file's symbols."""
    (shoff,) = struct.unpack_from("<Q", elf, 0x28)
    entry, count = struct.unpack_from("<HH", elf, 0x3A)
    sections = [struct.unpack_from("<IIQQQQIIQQ", elf, shoff + i * entry) for i in range(count)]
    for s in sections:
        if s[1] in (2, 11):
            for at in range(s[4], s[4] + s[5], 24):
                name, info, _, _, _, size = struct.unpack_from("<IBBHQQ", elf, at)
                start = sections[s[6]][4] + name
                yield elf[start: elf.index(b"\0", start)].decode(), info & 15, size


def test_functions_are_told_from_kernels_by_the_descriptors_that_launches_read():
    """Every kernel has one, an object of 64 bytes by its name; whatever has none is called, whatever its name."""
    if not os.path.exists(LIB):
        pytest.skip("the library is not built")
    with open(LIB, "rb") as f:
        data = f.read()
    kernels, called = 0, {}
    for i, elf in enumerate(_device_objects(data)):
        symbols = list(_symbols(elf))
        launched = {name[:-3] for name, kind, size in symbols if kind == 1 and name.endswith(".kd") and size == 64}      # STT_OBJECT
        functions = {name: size for name, kind, size in symbols if kind == 2}                                          # STT_FUNC
        assert launched <= set(functions)
        kernels += len(launched)
        called.update({(i, name): size for name, size in functions.items() if name not in launched})
    assert kernels > 100 and all(any(f in name for _, name in called) for f in ("draw_of_many", "list_of_many", "rest_behind"))
    assert {n: s for n, s in called.items() if s > REACH * 3 // 4} == {}
