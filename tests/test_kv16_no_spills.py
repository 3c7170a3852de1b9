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


@pytest.mark.parametrize("src", ["pv_kernels_kv16.hip", "pv_kernels_kv16_attention.hip", "pv_kernels_drafts.hip"])
def test_kernels_do_not_read_the_launch_packet(src):
    """Arrays that the compiler moves to LDS make a kernel read the launch's packet, in host memory: some 15 us where every workgroup does."""
    asking = [name for name, body in _kernels(src) if re.search(r"\.amdhsa_user_sgpr_dispatch_ptr\s+1", body)]
    assert not asking, asking
