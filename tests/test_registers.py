"""What the compiler makes of the kernels of the cache, of positions and of pages: none keeps registers or arrays in memory.  Compiles, needs no GPU."""
import os
import re
import shutil

import pytest

from tests import test_waits

pytestmark = pytest.mark.skipif(not shutil.which("hipcc") and not os.path.exists("/opt/rocm/bin/hipcc"), reason="needs hipcc")


@pytest.mark.parametrize("source,kernels", [("pasa_rotary.hip", 9), ("pasa_pages.hip", 9), ("pasa_cache.hip", 29)])
def test_nothing_is_kept_in_memory(source, kernels, tmp_path):
    text = test_waits._assembly(source, tmp_path)
    found = re.findall(r"\.name: +(\S*pasa_\S+)\n(?:(?! +- ).*\n)*? +\.private_segment_fixed_size: +(\d+)\n(?:(?! +- ).*\n)*? +\.vgpr_spill_count: +(\d+)", text)
    assert len(found) == kernels and all(int(a) == 0 and int(b) == 0 for _, a, b in found), found
