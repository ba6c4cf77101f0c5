"""What the compiler notes about every kernel of the built library: registers, spills, scratch memory, LDS.

A code object carries its kernels' names and needs as a msgpack map in an ELF note; the library holds one code object to a
source file, in bundles behind a text header."""
import os
import struct
import subprocess

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_16294_amd", "libsfcgemm.so")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def unpacked(b, at=0):
    """(value, where it ends) of a msgpack value: what notes are made of (no floats, no extensions)."""
    t = b[at]
    at += 1
    if t < 0x80 or t >= 0xE0:
        return (t if t < 0x80 else t - 256), at
    if t in (0xC0, 0xC2, 0xC3):
        return {0xC0: None, 0xC2: False, 0xC3: True}[t], at
    if 0xCC <= t <= 0xD3:
        size = 1 << (t & 3)
        return int.from_bytes(b[at:at + size], "big", signed=t >= 0xD0), at + size
    if t < 0xC0:
        n, kind = (t & 0x1F, "text") if t >= 0xA0 else (t & 0xF, "list" if t >= 0x90 else "map")
    else:
        size, kind = {0xD9: (1, "text"), 0xDA: (2, "text"), 0xDB: (4, "text"), 0xDC: (2, "list"), 0xDD: (4, "list"),
                      0xDE: (2, "map"), 0xDF: (4, "map")}[t]
        n = int.from_bytes(b[at:at + size], "big")
        at += size
    if kind == "text":
        return b[at:at + n].decode(), at + n
    items = []
    for _ in range(n * (2 if kind == "map" else 1)):
        item, at = unpacked(b, at)
        items.append(item)
    return (dict(zip(items[::2], items[1::2])) if kind == "map" else items), at


def code_objects(data):
    at = data.find(MAGIC)
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + len(MAGIC))
        p = at + len(MAGIC) + 8
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24:p + 24 + length]
            p += 24 + length
            if b"gfx950" in name and size:
                yield data[at + offset:at + offset + size]
        at = data.find(MAGIC, at + 1)


def notes(elf):
    """The maps of the notes of type 32 (AMDGPU metadata) of an ELF file."""
    phoff, = struct.unpack_from("<Q", elf, 32)
    size, count = struct.unpack_from("<HH", elf, 54)
    for i in range(count):
        kind, _, offset, _, _, length = struct.unpack_from("<IIQQQQ", elf, phoff + i * size)
        end = offset + length
        while kind == 4 and offset + 12 <= end:
            n, d, t = struct.unpack_from("<III", elf, offset)
            start = offset + 12 + (n + 3) // 4 * 4
            if t == 32:
                yield unpacked(elf[start:start + d])[0]
            offset = start + (d + 3) // 4 * 4


def kernels():
    """{name without its namespaces and arguments: its notes} of every kernel of the library."""
    with open(LIB, "rb") as f:
        data = f.read()
    found = [k for elf in code_objects(data) for note in notes(elf) for k in note["amdhsa.kernels"]]
    names = subprocess.run(["c++filt"], input="\n".join(k[".name"] for k in found), capture_output=True, text=True, check=True).stdout.split("\n")
    out = {}
    for k, name in zip(found, names):
        name = name.replace("(anonymous namespace)::", "").replace("(sfc::MoeLayout)", "").replace("sfc::", "").removeprefix("void ")
        out[name.rsplit("(", 1)[0]] = k
    return out
