"""CPU test of the gfx950 code of attention in libsc.so, disassembled: a load that takes its address from scalar registers needs five wait states behind a vector
instruction that wrote them, and the compiler does not look into inline assembly for it."""
import os
import re
import struct
import subprocess

from paper_2402_07710_amd import binding, build

OBJDUMP = os.path.join(os.path.dirname(os.path.dirname(build.HIPCC)), "llvm", "bin", "llvm-objdump")
NEEDED = 5


def code_of(library, name, tmp_path):
    """Instructions of each gfx950 code object that has kernels of this name, in order."""
    data = open(library, "rb").read()
    for at in (m.start() for m in re.finditer(re.escape(b"__CLANG_OFFLOAD_BUNDLE__"), data)):
        count, pos = struct.unpack_from("<Q", data, at + 24)[0], at + 32
        for _ in range(count):
            offset, size, name_len = struct.unpack_from("<QQQ", data, pos)
            target = data[pos + 24:pos + 24 + name_len]
            pos += 24 + name_len
            if b"gfx950" not in target or name not in data[at + offset:at + offset + size]:
                continue
            path = tmp_path / "object.elf"
            path.write_bytes(data[at + offset:at + offset + size])
            text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(path)], capture_output=True, text=True, check=True).stdout
            yield [line.split("//")[0].strip() for line in text.splitlines() if line.startswith("\t")]


def states(instruction):
    nop = re.match(r"s_nop (\d+)", instruction)
    return int(nop.group(1)) + 1 if nop else 1


def test_wait_states_between_a_vector_write_of_an_address_and_its_load(tmp_path):
    binding.load()
    sites, bad = 0, []
    for code in code_of(binding.LIB_PATH, b"k_attention", tmp_path):
        for i, line in enumerate(code):
            load = re.match(r"global_load_lds_\w+ v\d+, s\[(\d+):(\d+)\]", line)
            if load is None:
                continue
            sites += 1
            address, passed = range(int(load.group(1)), int(load.group(2)) + 1), 0
            for before in reversed(code[max(0, i - NEEDED):i]):
                if passed >= NEEDED:
                    break
                wrote = re.match(r"v_read(?:first)?lane_b32 s(\d+)", before)
                if wrote and int(wrote.group(1)) in address:
                    bad.append((before, line))
                    break
                passed += states(before)
    assert sites > 500
    assert not bad, f"{len(bad)} of {sites} loads, e.g. {bad[0]}"


def test_no_vector_register_is_spilled(tmp_path):
    """In a region that some lanes have left the compiler may save a register for the others alone, and read it back for all: the kernels of attention and of
    the group norm have branches of some lanes, so none of them may need more registers than there are."""
    readelf = os.path.join(os.path.dirname(OBJDUMP), "llvm-readelf")
    binding.load()
    data = open(binding.LIB_PATH, "rb").read()
    seen = 0
    for at in (m.start() for m in re.finditer(re.escape(b"__CLANG_OFFLOAD_BUNDLE__"), data)):
        count, pos = struct.unpack_from("<Q", data, at + 24)[0], at + 32
        for _ in range(count):
            offset, size, name_len = struct.unpack_from("<QQQ", data, pos)
            target = data[pos + 24:pos + 24 + name_len]
            pos += 24 + name_len
            if b"gfx950" not in target:
                continue
            path = tmp_path / "object.elf"
            path.write_bytes(data[at + offset:at + offset + size])
            notes = subprocess.run([readelf, "--notes", str(path)], capture_output=True, text=True, check=True).stdout
            for kernel in notes.split("- .agpr_count:")[1:]:
                name = re.search(r"\.name:\s+(\S+)", kernel).group(1)
                if "k_attention" not in name and "k_norm" not in name:
                    continue
                spilled = int(re.search(r"\.vgpr_spill_count:\s+(\d+)", kernel).group(1))
                scratch = int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", kernel).group(1))
                assert spilled == 0 and scratch == 0, (name, spilled, scratch)
                seen += 1
    assert seen > 80
