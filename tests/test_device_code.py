"""The instructions of the library that was built here, where a source cannot promise them by itself."""
import os
import re
import struct
import subprocess

import pytest

from paper_2605_16928_amd import rtp

OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")


def _code_objects(path):
    """The GPU code objects inside the library: bundles of {magic, count, (offset, size, name) of each}."""
    data, magic, found = open(path, "rb").read(), b"__CLANG_OFFLOAD_BUNDLE__", []
    at = data.find(magic)
    while at >= 0:
        n, p = struct.unpack_from("<Q", data, at + len(magic))[0], at + len(magic) + 8
        for _ in range(n if n < 16 else 0):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24:p + 24 + length]
            p += 24 + length
            if b"gfx950" in name and data[at + offset:at + offset + 4] == b"\x7fELF":
                found.append(data[at + offset:at + offset + size])
        at = data.find(magic, at + 1)
    return found


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    rtp.lib()
    folder, lines = tmp_path_factory.mktemp("code"), []
    for i, obj in enumerate(_code_objects(rtp.LIB_PATH)):
        (folder / f"{i}.co").write_bytes(obj)
        lines += subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(folder / f"{i}.co")], check=True, capture_output=True,
                                text=True).stdout.splitlines()
    return lines


def test_no_64_bit_shift_by_a_vector_register(listing):
    """Ranks came out wrong where the amount lay in a kernel's last register: masks are taken apart in 32-bit steps instead."""
    kernel, seen, bad = "", 0, []
    for line in listing:
        name = re.match(r"^[0-9a-f]+ <(\w+)>:", line)
        if name:
            kernel = name.group(1)
        shift = re.search(r"\bv_(lshlrev_b64|lshrrev_b64|ashrrev_i64)\S* \S+ (\S+),", line)
        if shift:
            seen += 1
            if shift.group(2).startswith("v"):
                bad.append(f"{kernel}: {line.strip()}")
    assert seen > 100, "the listing holds no shifts: it is not the library's"
    assert not bad, "\n".join(bad)
