"""No kernel of the selective scan, the short convolution and the norm spills a vector register or keeps an array in scratch memory (CPU only, from the
last build's report)."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_04250_amd", "csrc")

# a family's kernels and how many of them there are at least (types, widths, forms)
FAMILIES = {"select_tokens": 44, "select_prepare": 2, "select_scan": 24, "select_join": 12, "select_back": 12, "select_gradients": 12, "select_bc_sums": 2, "column_sums": 3,
            "conv_forward": 16, "conv_backward": 16, "conv_state_backward": 16, "rms_forward": 24, "rms_forward_long": 8, "rms_backward": 24, "rms_backward_long": 8}


def test_no_spills_and_no_scratch():
    reports = [p for u in ("select_*", "conv", "rms") for p in glob.glob(os.path.join(CSRC, f"cawn_{u}.res.txt"))]
    if not reports:
        pytest.skip("no resource report: library was not built by paper_2604_04250_amd.build")
    seen, name = dict.fromkeys(FAMILIES, 0), ""
    for path in reports:
        for line in open(path):
            key, _, val = (s.strip() for s in line.partition(":"))
            if key == "Function Name":
                name = val
                family = [f for f in FAMILIES if re.search(r"\d" + f + r"(?![a-z_])", name)]
                assert len(family) == 1, name
                seen[family[0]] += 1
            elif key.startswith("VGPRs Spill") or key.startswith("ScratchSize"):
                assert int(val) == 0, (name, key, val)
    assert all(seen[f] >= n for f, n in FAMILIES.items()), seen
