"""No kernel of the operators beside the scan spills a vector register or keeps an array in scratch memory (CPU only, from the last build's report)."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_04250_amd", "csrc")

# a family's kernels and how many of them there are at least (types, widths, modes)
FAMILIES = {"delta_tokens": 24, "delta_system": 6, "delta_scan": 16, "delta_join": 6, "delta_back": 14, "delta_gradients": 12, "group_norm_rows": 24, "group_norm_runs": 16,
            "group_norm_columns": 1, "dropout_units": 4, "dropout_elements": 4}


def test_no_spills_and_no_scratch():
    reports = [p for u in ("delta_*", "norm", "dropout") for p in glob.glob(os.path.join(CSRC, f"cawn_{u}.res.txt"))]
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
