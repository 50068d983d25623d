"""Counted waits of the float by 4-bit products, in the built library's own code.

k_mx4_gemm has x's slabs written to LDS by the memory unit, and waits for them by
`s_waitcnt vmcnt(N)`: at most the N last loads may be out.  That is a wait for x
only if at least N loads were issued after x's last one, the loads of b that are
written below them in the source.  Nothing in the language keeps these there, so
they are counted here, in the assembly of the kernels built from this tree: between
a counted wait and the last load to LDS before it, with no jump or label between
the two, there have to be N vector memory operations or more.
"""

import os
import re
import struct
import subprocess

import pytest

from paper_2608_30384_amd import _lib as L
from paper_2608_30384_amd import build as B

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(path):
    """The gfx950 code objects of a built library."""
    data = open(path, "rb").read()
    at = data.find(MAGIC)
    while at >= 0:
        entries = struct.unpack_from("<Q", data, at + len(MAGIC))[0]
        p = at + len(MAGIC) + 8
        for _ in range(entries):
            offset, size, n = struct.unpack_from("<QQQ", data, p)
            if b"gfx950" in data[p + 24:p + 24 + n]:
                yield data[at + offset:at + offset + size]
            p += 24 + n
        at = data.find(MAGIC, p)


def functions(path, name, folder):
    """The instructions and labels of every kernel whose name has `name` in it."""
    found = {}
    for i, code in enumerate(c for c in code_objects(path) if name.encode() in c):
        elf = os.path.join(folder, f"code{i}.elf")
        with open(elf, "wb") as f:
            f.write(code)
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--symbolize-operands", elf], capture_output=True,
                              text=True, check=True).stdout
        current = None
        for line in text.splitlines():
            m = re.match(r"^[0-9a-f]+ <(\S+)>:", line)
            if m and not re.fullmatch(r"L\d+", m.group(1)):
                current = found.setdefault(m.group(1), []) if name in m.group(1) else None
            elif current is not None and line.strip():
                current.append(line.split("//")[0].strip())
    return found


def is_load_to_lds(i):
    return re.match(r"(global|buffer)_load_lds", i) or (i.startswith("buffer_load") and i.endswith(" lds"))


def counted_waits(code):
    """Of each counted wait ahead of a barrier: its N, and how many vector memory operations
    were issued since the last load to LDS (None where a jump or a label lies between)."""
    waits, issued = [], None
    for i, at in enumerate(code):
        if is_load_to_lds(at):
            issued = 0
        elif re.match(r"(global|buffer|flat|scratch)_", at):
            issued = None if issued is None else issued + 1
        elif at.startswith("s_cbranch") or at.startswith("s_branch") or at.endswith(">:"):
            issued = None
        m = re.match(r"s_waitcnt .*vmcnt\((\d+)\)", at)
        if m and int(m.group(1)) and code[i + 1].startswith("s_barrier"):
            waits.append((int(m.group(1)), issued))
    return waits


@pytest.fixture(scope="module")
def library():
    L.lib()   # built if it is not there
    if not os.path.exists(OBJDUMP):
        pytest.skip("llvm-objdump not available")
    return B.LIB


def test_loads_after_the_ones_waited_for(library, tmp_path):
    kernels = functions(library, "k_mx4_gemm", tmp_path)
    kernels = {k: v for k, v in kernels.items() if not k.endswith(".kd")}
    assert len(kernels) == 50        # 5 heights of tiles, 5 pairs of types, 2 directions
    for name, code in kernels.items():
        waits = counted_waits(code)
        assert len(waits) >= 2, name
        for n, issued in waits:
            assert issued is not None and issued >= n, (name, n, issued)


def test_the_count_itself():
    """A wait that is right, one with a load too few, and one behind a label."""
    lds, load, wait = "global_load_lds_dwordx4 v[0:1], off", "global_load_dwordx4 v[0:3], v[4:5], off", "s_waitcnt vmcnt(2) lgkmcnt(0)"
    assert counted_waits([lds, load, load, wait, "s_barrier"]) == [(2, 2)]
    assert counted_waits([load, lds, load, wait, "s_barrier"]) == [(2, 1)]
    assert counted_waits([lds, load, load, "<L3>:", wait, "s_barrier"]) == [(2, None)]
    assert counted_waits([lds, load, load, "s_waitcnt vmcnt(0)", "s_barrier"]) == []


def asm_statements(text):
    """Every inline assembly statement, from its parenthesis to the matching one."""
    for m in re.finditer(r"\basm\s*(?:volatile)?\s*\(", text):
        depth, quoted, i = 1, False, m.end()
        while depth:
            c = text[i]
            if c == '"' and text[i - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            i += 1
        yield text[m.end():i - 1]


def test_inline_assembly_leaves_m0_to_the_compiler():
    """Loads to LDS take their address in m0, where the compiler may keep values of its
    own: it is an operand of the statement, and no statement writes it."""
    seen = 0
    for f in sorted(os.listdir(B.CSRC)):
        for s in asm_statements(open(os.path.join(B.CSRC, f)).read()):
            assert not re.search(r"\b[sv]_\w+ m0\b", s), (f, s)
            if re.search(r"load_lds|offen lds", s):
                seen += 1
                assert re.search(r'"\{m0\}"', s), (f, s)
    assert seen == 2
