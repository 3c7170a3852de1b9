"""The copies into LDS of the attention over a 16-bit cache keep the rules that tests/test_lds_copies.py states: m0 put back, no read of it right behind, wait states before a copy reads scalar registers that a vector
instruction has written (no GPU needed)."""
import test_lds_copies


def test_m0_is_put_back(tmp_path):
    test_lds_copies.test_m0_is_put_back(tmp_path, '#include "pv_kernels_kv16_attention.hip"\n', {2, 4})
