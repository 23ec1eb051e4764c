"""What the built code of the drawing of tokens may not hold: a branch of more than 128 KB in a function that is called.  Such a branch goes
through the registers of the function's return address; where the compiler has not saved them the function does not return."""
import subprocess

import pytest

from paper_2605_05940_amd import binding
from test_head_code import OBJDUMP, device_code, parse


def far_branches(kernels):
    return [(name, i) for name, code in kernels.items() for i in code if i[0] == "s_getpc_b64" and "s[30:31]" in i[1]]


def size(code):
    return code[-1][2] - code[0][2]


LISTING = """0000000000001000 <function>:
	s_getpc_b64 s[30:31]                                       // 000000001000: BE9E1C00
	s_setpc_b64 s[30:31]                                       // 000000001004: BE801D1E
"""


def test_the_check_finds_a_far_branch():
    kernels = parse(LISTING)
    assert len(far_branches(kernels)) == 1 and size(kernels["function"]) == 4
    assert not far_branches(parse(LISTING.replace("s_getpc_b64 s[30:31]", "s_getpc_b64 s[28:29]")))


@pytest.mark.skipif(OBJDUMP is None, reason="no llvm-objdump")
def test_functions_are_short(tmp_path):
    binding.load()
    functions = 0
    for n, code in enumerate(device_code(binding.LIB_PATH)):
        if b"sample_kernel" not in code:
            continue
        path = tmp_path / f"{n}.o"
        path.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(path)], capture_output=True, text=True, check=True).stdout
        kernels = parse(listing)
        assert not far_branches(kernels)
        for name, instructions in kernels.items():
            functions += 1
            assert size(instructions) < 1 << 17, (name, size(instructions))
    assert functions >= 4
