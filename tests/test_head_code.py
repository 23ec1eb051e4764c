"""Distances in the built code that nothing but this test keeps.  The matrix products of the head operators are written out
(`npd_head_gemm.hpp`: buffer_load ... lds and v_mfma), and the compiler, which puts wait states between instructions that depend on
each other, does not look into what is written out.  Checked over the library's own code, along every path into an instruction:

  a scalar register that a vector instruction wrote (v_readfirstlane, v_readlane of a spilled one) is read by a memory
  instruction's descriptor five wait states later or more;
  a register that a vector instruction wrote is an operand of a matrix instruction two wait states later or more;
  the sums of a written-out 16 x 16 x 32 matrix instruction (eight passes) are read or overwritten by anything but the next product
  eleven wait states later or more.
"""
import os
import re
import shutil
import struct
import subprocess

import pytest

from paper_2605_05940_amd import binding

OBJDUMP = next((p for p in (os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump"),
                            shutil.which("llvm-objdump") or "") if os.path.exists(p)), None)


def registers(operand):
    found = set()
    for m in re.finditer(r"\b([sva])(\d+)\b|\b([sva])\[(\d+):(\d+)\]|\b(m0|vcc|exec)\b", operand):
        if m.group(1):
            found.add((m.group(1), int(m.group(2))))
        elif m.group(3):
            found |= {(m.group(3), i) for i in range(int(m.group(4)), int(m.group(5)) + 1)}
        else:
            found.add((m.group(6), 0))
    return frozenset(found)


def parse(listing):
    """{kernel: [(operation, operands, address, address of a branch's target)]} of a disassembly."""
    kernels, now, base = {}, None, 0
    for line in listing.splitlines():
        head = re.match(r"([0-9a-f]+) <(.*)>:$", line)
        if head:
            base, now = int(head.group(1), 16), kernels.setdefault(head.group(2), [])
            continue
        m = re.match(r"\s+(\S+)\s*(.*?)\s*//\s*([0-9A-F]+):(.*)", line)
        if m and now is not None:
            to = re.search(r"<[^>+]+(?:\+0x([0-9a-f]+))?>", m.group(4))
            now.append((m.group(1), m.group(2), int(m.group(3), 16), base + int(to.group(1) or "0", 16) if to else None))
    return kernels


NO_RESULT = ("s_cmp", "s_cbranch", "s_branch", "s_nop", "s_wait", "s_barrier", "buffer_store", "global_store", "ds_write", "scratch_store")


def matrix(op):
    return op.startswith("v_mfma")


def vector(op):
    return op.startswith("v_") and not matrix(op)


def too_close(code):
    """What is nearer than it may be: [(instruction, the one in front of it, wait states between)]."""
    at = {i[2]: k for k, i in enumerate(code)}
    into = {}
    for k, i in enumerate(code):
        if i[0].startswith(("s_branch", "s_cbranch")) and i[3] in at:
            into.setdefault(at[i[3]], []).append(k)

    def before(k):
        first = [k - 1] if k and code[k - 1][0] not in ("s_branch", "s_endpgm", "s_setpc_b64") else []
        return first + into.get(k, [])

    def wrote(k):
        return frozenset() if code[k][0].startswith(NO_RESULT) else registers(code[k][1].split(",")[0])

    def search(k, registers_wanted, need, kind):
        found, paths = [], [(j, 0, registers_wanted) for j in before(k)]
        while paths:
            j, states, wanted = paths.pop()
            if states >= need or not wanted:
                continue
            if kind(code[j][0]) and wrote(j) & wanted:
                found.append((code[k], code[j], states))
            states += int(code[j][1], 0) + 1 if code[j][0] == "s_nop" else 1
            paths += [(p, states, wanted - wrote(j)) for p in before(j)]
        return found

    bad, checked = [], 0
    written_out = any(i[0].startswith("buffer_load") and i[1].endswith(" lds") for i in code)
    for k, (op, operands, _, _) in enumerate(code):
        if op.startswith("buffer_load") and operands.endswith(" lds"):
            checked += 1
            bad += search(k, frozenset(r for r in registers(operands) if r[0] == "s"), 5, vector)
        elif not written_out:
            continue
        elif matrix(op):
            checked += 1
            bad += search(k, registers(operands.split(",", 1)[1]), 2, vector)
        else:
            touched = frozenset(r for r in registers(operands) if r[0] in "va")
            if touched:
                bad += search(k, touched, 11, lambda o: o.startswith("v_mfma_f32_16x16x32"))
    return bad, checked


def device_code(path):
    """The gfx950 code objects of a library built here (uncompressed bundles of the compiler)."""
    data = open(path, "rb").read()
    for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data):
        entries, = struct.unpack_from("<Q", data, m.start() + 24)
        at = m.start() + 32
        for _ in range(entries):
            offset, size, length = struct.unpack_from("<QQQ", data, at)
            if b"gfx950" in data[at + 24:at + 24 + length]:
                yield data[m.start() + offset:m.start() + offset + size]
            at += 24 + length


LISTING = """0000000000001000 <kernel>:
	v_readlane_b32 s6, v9, 3                                   // 000000001000: 00000000
	s_mov_b32 m0, s20                                          // 000000001004: 00000000
	s_nop 0                                                    // 000000001008: 00000000
	buffer_load_dwordx4 v2, s[4:7], 0 offen lds                // 00000000100C: 00000000
	v_mov_b32_e32 v8, v1                                       // 000000001010: 00000000
	v_mfma_f32_16x16x32_bf16 a[0:3], v[8:11], v[12:15], a[0:3] // 000000001014: 00000000
	v_mfma_f32_16x16x32_bf16 a[0:3], v[8:11], v[12:15], a[0:3] // 000000001018: 00000000
	s_nop 7                                                    // 00000000101C: 00000000
	v_accvgpr_read_b32 v0, a2                                  // 000000001020: 00000000
	s_cbranch_scc1 65528                                       // 000000001024: 00000000 <kernel+0x14>
"""


def test_the_check_finds_what_is_too_close():
    bad, checked = too_close(parse(LISTING)["kernel"])
    assert checked == 3
    assert [(a[2], b[2], n) for a, b, n in bad] == [(0x100c, 0x1000, 2), (0x1014, 0x1010, 0), (0x1018, 0x1010, 1), (0x1020, 0x1018, 8)]
    # far enough, or written again by what the next instruction waits for
    fine = LISTING.replace("s_nop 0 ", "s_nop 3 ").replace("v_mov_b32_e32 v8, v1", "v_mov_b32_e32 v7, v1").replace("s_nop 7", "s_nop 15")
    assert not too_close(parse(fine)["kernel"])[0]
    assert not too_close(parse(fine.replace("s_nop 3 ", "s_nop 0 ").replace("s_mov_b32 m0, s20", "s_mul_i32 s6, s6, 4"))["kernel"])[0]
    # along a branch: the last vector instruction of a loop in front of the product at its head
    loop = fine.replace("v_accvgpr_read_b32 v0, a2", "v_mov_b32_e32 v12, v0")
    for head in (0x14, 0x18):
        found = too_close(parse(loop.replace("kernel+0x14", f"kernel+{head:#x}"))["kernel"])[0]
        assert [(a[2], b[2], n) for a, b, n in found] == [(0x1000 + head, 0x1020, 1)]


@pytest.mark.skipif(OBJDUMP is None, reason="no llvm-objdump")
def test_the_products_keep_their_distances(tmp_path):
    binding.load()
    kernels = 0
    for n, code in enumerate(device_code(binding.LIB_PATH)):
        if b"head_forward_kernel" not in code and b"head_weight_kernel" not in code:
            continue
        path = tmp_path / f"{n}.o"
        path.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(path)], capture_output=True, text=True, check=True).stdout
        for name, instructions in parse(listing).items():
            bad, checked = too_close(instructions)
            kernels += checked > 0
            assert not bad, (name, bad[0])
    assert kernels > 20
