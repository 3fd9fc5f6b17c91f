"""The global-to-LDS copies of the causal attention in the built library: a copy is inline assembly,
in which the compiler looks for no hazards, so each has to bring the wait states that gfx9 wants
between a vector instruction that writes a scalar register and a memory instruction that reads
it.  CPU only: reads the disassembly of the code objects built here."""
import os
import re
import struct
import subprocess

import pytest

from paper_2607_03229_amd import build as B

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"
WANTED = 5


def code_objects(lib):
    """The gfx950 code objects of a library's offload bundles."""
    data = open(lib, "rb").read()
    at = data.find(MAGIC)
    while at >= 0:
        n, = struct.unpack_from("<Q", data, at + len(MAGIC))
        p = at + len(MAGIC) + 8
        for _ in range(n if n < 16 else 0):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24:p + 24 + length]
            if name.startswith(b"hip") and name.endswith(b"gfx950"):
                yield data[at + offset:at + offset + size]
            p += 24 + length
        at = data.find(MAGIC, at + 1)


def copies(listing):
    """(kernel, wait states that the instructions right before bring) of every buffer copy into LDS
    in a disassembly."""
    kernel, states = None, 0
    for line in listing.splitlines():
        head = re.match(r"[0-9a-f]+ <(\S+)>:", line)
        if head:
            kernel, states = head.group(1), 0
            continue
        text = line.split("//")[0].strip()
        if not text:
            continue
        nop = re.match(r"s_nop (\d+)$", text)
        if nop:
            states += int(nop.group(1)) + 1
        elif text.startswith("s_mov_b32 m0,"):
            states += 1
        else:
            if text.startswith("buffer_load") and text.endswith(" lds"):
                yield kernel, states
            states = 0


def test_scan_counts_wait_states():
    text = """0000000000001900 <kernel_a>:
\tv_readlane_b32 s24, v200, 3  // 000000001900: D2890018
\ts_mov_b32 m0, s41  // 000000001904: BEFC0029
\ts_nop 0  // 000000001908: BF800000
\tbuffer_load_dwordx4 v1, s[24:27], 0 offen lds  // 00000000190C: E05D1000
\ts_mov_b32 m0, s41  // 000000001914: BEFC0029
\ts_nop 3  // 000000001918: BF800003
\tbuffer_load_dword v1, s[24:27], 0 offen lds  // 00000000191C: E0511000
\tbuffer_load_dwordx4 v[0:3], v4, s[24:27], 0 offen  // 000000001924: E05C1000
"""
    assert list(copies(text)) == [("kernel_a", 2), ("kernel_a", 5)]


@pytest.mark.skipif(not (os.path.exists(B.LIB) and os.path.exists(OBJDUMP)),
                    reason="needs libmpipe.so and llvm-objdump")
def test_copies_bring_their_wait_states(tmp_path):
    seen = set()
    for i, code in enumerate(code_objects(B.LIB)):
        if b"causal_" not in code:
            continue
        path = tmp_path / f"{i}.co"
        path.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(path)], check=True,
                                 capture_output=True, text=True).stdout
        for kernel, states in copies(listing):
            if "causal_" in kernel:
                seen.add(kernel)
                assert states >= WANTED, (kernel, states)
    for name in ("causal_fwd_kernel", "causal_dq_kernel", "causal_dkdv_kernel"):
        assert any(name in k for k in seen), name
