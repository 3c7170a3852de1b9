"""No kernel of the operators around the 16-bit cache and of verified drafts may spill registers to scratch memory (compiles the device code to assembly, no GPU needed)."""
import re

import pytest

from test_no_spills import _kernels


@pytest.mark.parametrize("src", ["pv_kernels_kv16.hip", "pv_kernels_kv16_attention.hip", "pv_kernels_drafts.hip"])
def test_kernels_use_no_scratch(src):
    kernels = _kernels(src)
    assert kernels, "no kernel descriptors found"
    spilled = [name for name, body in kernels if int(re.search(r"\.amdhsa_private_segment_fixed_size\s+(\d+)", body).group(1)) > 0]
    assert not spilled, f"kernels with scratch (register spills): {spilled}"
