"""The wait states of test_device_hazards.py in the kernels of the packed attention, and what their loops must not hold (no GPU)."""
import re

import pytest

from test_device_hazards import assembly, hazards


@pytest.mark.parametrize("src", ["lf_packed_attn.hip", "lf_packed_attn_wide.hip", "lf_packed_rows.hip", "lf_packed_bwd.hip", "lf_packed_dkv_wide.hip"])
def test_instructions_keep_their_distance_on_every_path(src):
    found = hazards(assembly(src))
    if src == "lf_packed_rows.hip":     # its products are the compiler's own, 16 x 16 ones of half the passes that the check counts with
        found = [f for f in found if "16x16x32" not in f[2]]
    for f in found[:10]:
        print(*f)
    assert not found


def test_the_sums_of_the_wide_gradient_kernel_stay_where_they_are():
    """No spilled register and no copy between the halves of the register file inside the loop: it has 64 products, and
    only what stands before it and behind it moves the sums."""
    lines = assembly("lf_packed_dkv_wide.hip")
    assert any(re.match(r"\s*\.private_segment_fixed_size:\s*0\b", line) for line in lines)
    labels = {m[1]: i for i, line in enumerate(lines) if (m := re.match(r"(\.LBB\d+_\d+):", line))}
    loops = [(labels[m[1]], i) for i, line in enumerate(lines) if (m := re.search(r"s_cbranch\w*\s+(\.LBB\d+_\d+)|s_branch\s+(\.LBB\d+_\d+)", line))
             and (m[1] or m[2]) in labels and m[1] and labels[m[1]] < i]
    with_products = [(a, b) for a, b in loops if sum("v_mfma" in line for line in lines[a:b]) >= 64]
    assert with_products
    a, b = min(with_products, key=lambda x: x[1] - x[0])
    assert sum("v_mfma" in line for line in lines[a:b]) == 64
    assert not [line for line in lines[a:b] if "accvgpr" in line or "scratch_" in line]
