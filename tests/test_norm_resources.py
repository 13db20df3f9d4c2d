"""Scratch memory of the built norm, gradient and dequantization kernels, from the library's own
metadata (no GPU needed): registers that a loop spills cost memory traffic without any wrong result."""
import os
import re
import subprocess

import pytest

from test_kernel_resources import READELF, code_objects


def test_scratch(tmp_path):
    import paper_2607_24953_amd as q2d
    if not os.path.exists(READELF):
        pytest.skip("no llvm-readelf")
    seen = 0
    for i, obj in enumerate(code_objects(q2d.lib_path)):
        f = tmp_path / ("%d.co" % i)
        f.write_bytes(obj)
        text = subprocess.run([READELF, "--notes", str(f)], check=True, capture_output=True, text=True).stdout
        for part in re.split(r"\n  - ", text)[1:]:
            name = re.search(r"\.symbol:\s*'?([\w.]+)", part)
            if name is None or not re.search(r"rmsnorm_|grad_(square|scale|norm)_|dequantize_", name.group(1)):
                continue
            seen += 1
            scratch = int(re.search(r"\.private_segment_fixed_size:\s*(\d+)", part).group(1))
            lds = int(re.search(r"\.group_segment_fixed_size:\s*(\d+)", part).group(1))
            assert scratch == 0, (name.group(1), scratch)
            # two workgroups fit a CU's 160 KB, but of the norm's gradient with 16 waves
            most = 144 if re.search(r"rmsnorm_grad_kernel.*Li1024E", name.group(1)) else 80
            assert lds <= most * 1024, (name.group(1), lds)
    assert seen > 60, seen
