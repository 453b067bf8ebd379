"""What the compiler made of the cache's kernels (host only: gfx950 assembly of the library's own sources)."""
import re

import pytest

from tests.test_kernel_code import assembly


@pytest.mark.parametrize("source,count", [("cache_attention.hip", 16), ("cache_rows.hip", 6), ("cache_pages.hip", 8)])
def test_short_arguments_and_no_spilled_registers(source, count):
    """112 bytes of arguments at most, implicit ones included (a longer launch takes the host 0.7 us more), and nothing in scratch memory."""
    found = re.findall(r"\.kernarg_segment_size: (\d+).*?\.name: +(\w+).*?\.private_segment_fixed_size: (\d+).*?\.vgpr_spill_count: (\d+)", assembly(source), flags=re.S)
    assert len(found) == count
    for arguments, name, scratch, spilled in found:
        assert int(arguments) <= 112 and int(scratch) == 0 and int(spilled) == 0, name
