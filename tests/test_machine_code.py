"""What the compiler cannot see to in inline assembly, checked in the library's machine code
(CPU only)."""
import os
import re
import struct
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2502_15572_amd import _lib

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def device_code(tmp):
    """Files of the gfx950 code objects that the library was linked from."""
    data = open(_lib.LIB_PATH, "rb").read()
    files, at = [], data.find(MAGIC)
    while at >= 0:
        n, = struct.unpack_from("<Q", data, at + 24)
        p = at + 32
        for _ in range(n if n < 16 else 0):
            off, size, length = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24:p + 24 + length]
            p += 24 + length
            if b"gfx950" in name and size:
                files.append(os.path.join(tmp, "%d.co" % len(files)))
                with open(files[-1], "wb") as f:
                    f.write(data[at + off:at + off + size])
        at = data.find(MAGIC, at + 24)
    return files


def instructions(path):
    text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", path], capture_output=True,
                          text=True, check=True).stdout
    return re.sub(r"\s*//.*", "", text)


def too_soon(text):
    """Copies to LDS that directly follow a write of M0, which they read: they need a wait state
    in between."""
    return re.findall(r"\n\ts_\w+ m0,[^\n]*\n\t((?:global|buffer)_load_(?:lds_\w+|\w+[^\n]* lds\b))",
                      text)


READS_SCC = ("s_cbranch_scc", "s_cselect", "s_addc", "s_subb", "s_cmov")
SETS_SCC = re.compile(r"s_(add|sub|cmp|bitcmp|and|or|xor|nand|nor|xnor|andn|orn|not|lsh|ash|min|max|"
                      r"abs|absdiff|bfe|bcnt|wqm|quadmask)")


def stale_scc(text):
    """Reads of the carry bit for which a sum into M0 (which only inline assembly forms) is the last
    to have set it."""
    found = []
    for after in text.split("\ts_add_u32 m0, m0,")[1:]:
        for line in after.split("\n")[1:]:
            op = line.strip().split(" ")[0]
            if op.startswith(READS_SCC):
                found.append(line)
            if not op or op.startswith(READS_SCC) or SETS_SCC.match(op) or op in (
                    "s_branch", "s_endpgm", "s_setpc_b64"):
                break
    return found


def test_the_check_itself():
    copy = "\tglobal_load_lds_dwordx4 v[2:3], off nt\n"
    assert too_soon("\n\ts_mov_b32 m0, s4\n" + copy)
    assert too_soon("\n\ts_add_u32 m0, m0, 0x400\n\tbuffer_load_dwordx4 v1, s[0:3], 0 offen lds\n")
    assert not too_soon("\n\ts_mov_b32 m0, s4\n\ts_nop 0\n" + copy)
    assert not too_soon("\n\ts_mov_b32 m0, s4\n\tglobal_load_dwordx4 v[2:5], v[0:1], off\n")
    add = "\ts_add_u32 s4, s4, s8\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n"
    assert stale_scc(add + copy + "\ts_addc_u32 s5, s5, 0\n")
    assert not stale_scc(add + copy + "\ts_cmp_eq_u32 s1, s2\n\ts_cbranch_scc1 12\n")


@pytest.fixture(scope="module")
def found(tmp_path_factory):
    """Of all kernels: copies to LDS, those too soon after their address, stale reads of the carry."""
    if not (os.path.exists(_lib.LIB_PATH) and os.path.exists(OBJDUMP)):
        pytest.skip("no built library or no disassembler")
    files = device_code(str(tmp_path_factory.mktemp("code")))
    assert files

    def one(path):
        text = instructions(path)
        return len(re.findall(r"\n\tglobal_load_lds_", text)), len(too_soon(text)), len(
            stale_scc(text))

    with ThreadPoolExecutor(4) as ex:
        return [sum(x) for x in zip(*ex.map(one, files))]


def test_copies_to_lds_wait_for_their_address(found):
    assert found[0] > 1000                      # (the copies are there to be looked at)
    assert found[1] == 0


def test_sums_into_m0_keep_no_carry_from_its_reader(found):
    assert found[2] == 0
