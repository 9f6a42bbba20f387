"""Compiled code of the gated block's kernels: the library's own check, and no lane-conditional code where registers are relocated.

The compiler has been seen to place a register move inside a lane-conditional region although the value is live in all lanes; kernels that
keep values in accumulation registers or private memory therefore must not write the execution mask before their sums are complete (the
guarded stores at the end read them for the last time)."""
import re
import struct
import subprocess

import pytest

from paper_2501_13986_amd import binding as b

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
READELF = "/opt/rocm/llvm/bin/llvm-readelf"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


@pytest.fixture(scope="module")
def objects(tmp_path_factory):
    """The gfx950 code objects inside the library."""
    b.lib()
    data, out, at = open(b.LIB_PATH, "rb").read(), [], 0
    folder = tmp_path_factory.mktemp("objects")
    while (at := data.find(MAGIC, at)) >= 0:
        (n,) = struct.unpack_from("<Q", data, at + 24)
        p = at + 32
        for _ in range(n):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            triple = data[p + 24:p + 24 + length].decode()
            p += 24 + length
            if "gfx950" in triple and size:
                path = str(folder / f"{len(out)}.co")
                open(path, "wb").write(data[at + offset:at + offset + size])
                out.append(path)
        at += 24
    assert len(out) >= 3     # graph preparation, gated block in both types
    return out


def test_the_library_s_own_check(objects):
    for path in objects:
        assert b.check_code_object(path) == "", path


def kernels(path):
    """name -> (accumulation registers, private bytes)"""
    notes = subprocess.run([READELF, "--notes", path], capture_output=True, text=True, check=True).stdout
    out = {}
    for part in notes.split("- .agpr_count:")[1:]:
        out[re.search(r"\.name:\s+(\S+)", part).group(1)] = (int(part.split()[0]), int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", part).group(1)))
    return out


def test_no_lane_conditional_code_before_the_sums_are_complete(objects):
    seen = relocating = 0
    for path in objects:
        found = {k: v for k, v in kernels(path).items() if "k_gated" in k}
        if not found:
            continue
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", path], capture_output=True, text=True, check=True).stdout
        for block in re.split(r"\n(?=[0-9a-f]+ <)", text):
            m = re.match(r"[0-9a-f]+ <([^>]+)>:", block)
            if not m or m.group(1) not in found:
                continue
            seen += 1
            ins = [line.strip() for line in block.splitlines()[1:] if line.strip()]
            assert not any(i.startswith(("v_pk_add_f32", "v_pk_mul_f32", "v_pk_fma_f32")) for i in ins), m.group(1)
            if found[m.group(1)] == (0, 0):
                continue
            relocating += 1
            products = [j for j, i in enumerate(ins) if "mfma" in i]
            writes = [i for i in ins[:products[-1]] if "saveexec" in i or re.match(r"(s_\w+|v_cmpx\w*) exec\b", i)]
            assert not writes, (m.group(1), writes[:3])
    assert seen > 100 and relocating > 0

