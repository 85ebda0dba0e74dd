"""CPU test of the gfx950 code of the products of rows in libsc.so, disassembled: rows of results have a streamed store and a plain one of each chunk, chosen by the
rows' alignment.  Both write the same values to the same address, so a compiler may take them for one."""
import os
import re
import struct
import subprocess

from paper_2402_07710_amd import binding, build

OBJDUMP = os.path.join(os.path.dirname(os.path.dirname(build.HIPCC)), "llvm", "bin", "llvm-objdump")
F32, FORWARD, INPUT_GRADIENT, BEHIND_ACTIVATION, WEIGHT_GRADIENT = 0, 0, 1, 2, 3


def product_kernels(library, tmp_path):
    """Template arguments (type, product, rows and columns of the tile, wavefronts along both, ...) and code of every k_product in a library."""
    data = open(library, "rb").read()
    for at in (m.start() for m in re.finditer(re.escape(b"__CLANG_OFFLOAD_BUNDLE__"), data)):
        count, pos = struct.unpack_from("<Q", data, at + 24)[0], at + 32
        for _ in range(count):
            offset, size, name_len = struct.unpack_from("<QQQ", data, pos)
            target = data[pos + 24:pos + 24 + name_len]
            pos += 24 + name_len
            if b"gfx950" not in target or b"k_productI" not in data[at + offset:at + offset + size]:
                continue
            path = tmp_path / "object.elf"
            path.write_bytes(data[at + offset:at + offset + size])
            text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(path)], capture_output=True, text=True, check=True).stdout
            for kernel in re.split(r"(?m)^[0-9a-f]+ <", text)[1:]:
                name = re.match(r"\w*k_productI((?:L[ib]\d+E)+)E", kernel)
                if name:
                    yield [int(v) for v in re.findall(r"L[ib](\d+)E", name.group(1))], kernel


def test_rows_are_streamed_or_not(tmp_path):
    binding.load()
    seen = 0
    for (kind, product, rows, columns, along, across, *rest), code in product_kernels(binding.LIB_PATH, tmp_path):
        stores = [line for line in code.splitlines() if "global_store_dwordx4" in line]
        streamed = sum(" nt" in line for line in stores)
        # a lane's chunks of eight columns; 16 bytes of each at a time: results, and forward the value ahead of the activation, in the rows' type and in 32 bits
        chunks = (rows // 16 // along) * (columns // 32 // across)
        narrow = 2 if kind == F32 else 1
        want = 0 if product == WEIGHT_GRADIENT else chunks * (2 * (2 + narrow) if product == FORWARD else narrow)
        what = (kind, product, rows, columns, along, across, *rest)
        assert streamed == want and len(stores) - streamed >= want, (what, streamed, len(stores) - streamed, want)
        seen += 1
    assert seen > 100
