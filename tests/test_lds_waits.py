"""The waits of kernels whose waves fill LDS buffers of their own, as the library was built (no GPU needed).

A buffer is filled again by loads from memory straight into LDS.  Those and the LDS reads of what the buffer held before go through
different queues, so a read that is still under way when the loads are issued is ordered before them by nothing but how long memory
takes.  Read from the machine code: between the last LDS read and a load into LDS stands a wait for all reads.
"""
import os
import re
import struct
import subprocess

import pytest

import paper_2412_16434_amd as S
from paper_2412_16434_amd import build

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def device_code(path):
    """The device code objects inside a library built by hipcc."""
    data = open(path, "rb").read()
    for m in re.finditer(re.escape(MAGIC), data):
        at = m.start() + len(MAGIC)
        n, = struct.unpack_from("<Q", data, at)
        at += 8
        for _ in range(n):
            offset, size, length = struct.unpack_from("<QQQ", data, at)
            name = data[at + 24:at + 24 + length]
            at += 24 + length
            if b"amdgcn" in name and size:
                yield data[m.start() + offset:m.start() + offset + size]


def loads_ahead_of_reads(listing):
    """{kernel: (loads into LDS, those with LDS reads under way)} of a disassembly."""
    found, kernel, under_way = {}, None, 0
    for line in listing:
        head = re.match(r"^(?:[0-9a-f]+ )?<(\S+)>:", line)
        if head:
            kernel, under_way = head.group(1), 0
            found[kernel] = [0, 0]
            continue
        op = line.strip()
        if kernel is None or not op:
            continue
        if op.startswith("ds_read"):
            under_way += 1
        elif op.startswith("s_waitcnt"):
            left = re.search(r"lgkmcnt\((\d+)\)", op)
            if left:
                under_way = min(under_way, int(left.group(1)))
        elif re.match(r"(buffer|global)_load_\w*lds|(buffer|global)_load_.*\blds\b", op):
            found[kernel][0] += 1
            found[kernel][1] += under_way > 0
    return {k: tuple(v) for k, v in found.items()}


def test_the_scan_itself():
    text = """0000000000001000 <one>:
	ds_read_b128 v[0:3], v9
	s_waitcnt lgkmcnt(0)
	buffer_load_dwordx4 v2, s[0:3], 0 offen nt lds
0000000000002000 <two>:
	ds_read_b64_tr_b16 v[0:1], v9
	ds_read_b64_tr_b16 v[2:3], v9
	s_waitcnt vmcnt(8) lgkmcnt(1)
	buffer_load_dwordx4 v2, s[0:3], 0 offen lds
	global_load_dwordx4 v[0:3], v[4:5], off
	s_waitcnt lgkmcnt(0)
	global_load_lds_dwordx4 v[0:1], off"""
    assert loads_ahead_of_reads(text.split("\n")) == {"one": (1, 0), "two": (2, 1)}


def test_streams_fill_a_buffer_only_after_its_reads(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    S.load_library()
    seen = 0
    for i, code in enumerate(device_code(build.LIB)):
        if b"tree_stream_kernel" not in code:
            continue
        path = tmp_path / f"{i}.o"
        path.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(path)], capture_output=True, text=True,
                                 check=True).stdout
        for kernel, (loads, ahead) in loads_ahead_of_reads(listing.split("\n")).items():
            if "tree_stream_kernel" in kernel:
                seen += 1
                assert loads > 0, kernel
                assert ahead == 0, f"{kernel}: {ahead} of {loads} loads into LDS are issued before its reads have returned"
    assert seen > 0
