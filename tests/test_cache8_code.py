"""What the compiler made of the kernels on a cache held in 8 bits (host only: gfx950 assembly of the library's own sources)."""
import re

import pytest

from tests.test_kernel_code import assembly


@pytest.mark.parametrize("source,count,most", [("cache8_attention.hip", 16, 112), ("cache8_rows.hip", 27, 168), ("cache8_select.hip", 14, 112)])
def test_arguments_and_no_spilled_registers(source, count, most):
    """112 bytes of arguments at most, implicit ones included (a longer launch takes the host 0.7 us more), but for an append, which has ten pointers of its own; and
    nothing in scratch memory."""
    found = re.findall(r"\.kernarg_segment_size: (\d+).*?\.name: +(\w+).*?\.private_segment_fixed_size: (\d+).*?\.vgpr_spill_count: (\d+)", assembly(source), flags=re.S)
    assert len(found) == count
    for arguments, name, scratch, spilled in found:
        assert int(arguments) <= (most if "append" in name else 112) and int(scratch) == 0 and int(spilled) == 0, name


def test_products_of_two_take_their_constants_from_registers():
    """An operand of -1 that is part of the instruction is one of fp32 there, not the pair of bf16 numbers that the source has."""
    found = re.findall(r"v_dot2c?_f32_bf16\w* v\d+, (.*)", assembly("cache8_attention.hip"))
    assert found and all(re.match(r"[sv]\d+, ", operands) for operands in found)
