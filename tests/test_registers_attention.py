"""What the compiler makes of attention over the cache, whose kernels are the nearest to what registers there are: none keeps any in memory, and two of its
wavefronts fit a SIMD.  Compiles, needs no GPU."""
import os
import re
import shutil

import pytest

from tests import test_waits

pytestmark = pytest.mark.skipif(not shutil.which("hipcc") and not os.path.exists("/opt/rocm/bin/hipcc"), reason="needs hipcc")


def test_nothing_is_kept_in_memory(tmp_path):
    text = test_waits._assembly("pasa_attn_cache.hip", tmp_path)
    gap = r"\n(?:(?! +- ).*\n)*? +"
    found = re.findall(r"\.name: +(\S*pasa_\S+)" + gap + r"\.private_segment_fixed_size: +(\d+)" + gap + r"\.vgpr_count: +(\d+)" + gap + r"\.vgpr_spill_count: +(\d+)", text)
    # of each size of a head: formats, chosen pages and reads past the caches with 16 rows; formats and chosen pages with 32; two merges each
    assert len(found) == 2 * (3 * 2 * 2 + 3 * 2 + 4)
    assert all(int(memory) == 0 and int(spilled) == 0 and int(registers) <= 256 for _, memory, registers, spilled in found), found
