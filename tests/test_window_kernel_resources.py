"""Waves per SIMD that the rules of windowed attention and the paged cache count on (csrc/attn_win_rules.hpp: places on the chip, row blocks for
two CUs; workgroups on a CU of the single-token kernels) stay in the compiled kernels.  CPU only."""
import re
import shutil

import pytest

from paper_2410_09397_amd import pmc_summary

# A workgroup of four waves has one on each SIMD: waves per SIMD are workgroups per CU.
OCCUPANCY = {
    # 128- and 64-row blocks: two on a CU up to d = 128, one at d = 256
    r"win_out_kernel<64, \d, 1, (true|false)>": 3, r"win_out_kernel<64, \d, 2, (true|false)>": 4, r"win_out_kernel<128, \d, \d, (true|false)>": 2,
    r"win_out_kernel<256, .*>": 1, r"win_dq_kernel<64, .*>": 3, r"win_dq_kernel<128, .*>": 2, r"win_dq_kernel<256, .*>": 1,
    # owners of keys: 512 places up to d = 128, 256 beyond
    r"win_dkdv_kernel<64, .*>": 3, r"win_dkdv_kernel<128, .*>": 2, r"win_dkdv_kernel<256, .*>": 1,
    # few rows: kOnePerCu of the single-token kernels, the launch bounds of the 32-row ones
    r"win_one_kernel<64, .*>": 4, r"win_one_kernel<128, .*>": 3, r"win_one_kernel<256, 2, false>": 2, r"win_one_kernel<256, 1, .*>": 1,
    r"win_few_kernel<64, .*>": 2, r"win_few_kernel<128, .*>": 2, r"win_few_kernel<256, .*>": 1,
    # fp32 arithmetic, by width
    r"win_plain_out_kernel<.*, (32|64|96), (true|false)>": 2, r"win_plain_dq_kernel<(32|64|96)>": 2, r"win_plain_dkdv_kernel<.*>": 1,
    # waves that wait for memory alone
    r"cache_(read|write)_kernel<.*>": 8, r"win_join_kernel<.*>": 8, r"win_keys_kernel<.*>": 8, r"win_rows_kernel": 8,
}


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_occupancies_that_the_rules_count_on():
    seen = pmc_summary.kernel_resources(["attn_win_fwd.hip", "attn_win_bwd.hip", "attn_win_plain.hip", "attn_cache.hip"])
    for pattern, waves in OCCUPANCY.items():
        of = [(r["kernel"], int(r["Occupancy [waves/SIMD]"])) for r in seen if re.match(pattern + "$", r["kernel"])]
        assert of and min(o for _, o in of) >= waves, (pattern, waves, of)
