"""Distances in the built code of the int8 products, which nothing but this test keeps (as test_head_code.py does for the bf16 ones, whose
written-out loads and products these share; a product of 16 x 16 x 64 bytes takes the passes of one of 16 x 16 x 32 bf16 values)."""
import subprocess

import pytest

from paper_2605_05940_amd import binding
from test_head_code import LISTING, OBJDUMP, device_code, parse, too_close


def as_bf16(listing):
    return listing.replace("v_mfma_i32_16x16x64_i8", "v_mfma_f32_16x16x32_bf16")


def test_the_check_sees_int8_products():
    listing = LISTING.replace("v_mfma_f32_16x16x32_bf16", "v_mfma_i32_16x16x64_i8")
    found = too_close(parse(as_bf16(listing))["kernel"])[0]
    assert [(a[2], b[2]) for a, b, _ in found] == [(0x100c, 0x1000), (0x1014, 0x1010), (0x1018, 0x1010), (0x1020, 0x1018)]


@pytest.mark.skipif(OBJDUMP is None, reason="no llvm-objdump")
def test_the_products_keep_their_distances(tmp_path):
    binding.load()
    kernels = 0
    for n, code in enumerate(device_code(binding.LIB_PATH)):
        if b"int8_tiles_kernel" not in code:
            continue
        path = tmp_path / f"{n}.o"
        path.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(path)], capture_output=True, text=True, check=True).stdout
        assert "v_mfma_i32_16x16x64_i8" in listing
        for name, instructions in parse(as_bf16(listing)).items():
            bad, checked = too_close(instructions)
            kernels += checked > 0
            assert not bad, (name, bad[0])
    assert kernels == 8


def exchanges(instructions):
    """Of a kernel's LDS instructions and barriers in their order: what comes before each that writes LDS."""
    those = [i[0] for i in instructions if i[0].startswith("ds_") or i[0] == "s_barrier"]
    return [those[n - 1] if n else None for n, op in enumerate(those) if op.startswith("ds_write")]


@pytest.mark.skipif(OBJDUMP is None, reason="no llvm-objdump")
def test_the_tiles_factors_are_written_before_they_are_read(tmp_path):
    """A wave's factors lie in LDS, where lanes read what others wrote.  Nothing reads LDS between the barrier behind a tile's last step and the
    last of these writes, which follow each other: the reads are all behind them."""
    assert exchanges([(op,) for op in ("ds_read_b128", "s_barrier", "ds_write_b32", "ds_read_b32", "ds_write_b32")]) == ["s_barrier", "ds_read_b32"]
    binding.load()
    kernels = 0
    for n, code in enumerate(device_code(binding.LIB_PATH)):
        if b"int8_tiles_kernel" not in code:
            continue
        path = tmp_path / f"{n}.o"
        path.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(path)], capture_output=True, text=True, check=True).stdout
        for name, instructions in parse(listing).items():
            if "int8_tiles_kernel" not in name or len(instructions) < 100:
                continue
            before = exchanges(instructions)
            kernels += 1
            assert before and before[0] == "s_barrier", name
            assert all(op.startswith("ds_write") for op in before[1:]), (name, before)
    assert kernels == 8
