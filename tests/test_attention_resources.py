"""Scratch memory of the built attention and cache kernels, from the library's own metadata (no GPU
needed): registers that a loop spills cost memory traffic without any wrong result."""
import os
import re
import subprocess

import pytest

from test_kernel_resources import READELF, code_objects

# kernel, element type and computed dims (in its mangled name) -> bytes a lane; the others take none
ALLOWED = {"attention_dq_kernelIDF16bLi128": 20, "attention_dq_kernelIfLi96": 44, "attention_dq_kernelIfLi128": 244,
           "attention_cached_rows_kernelILi128": 64}


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
            if name is None or not re.search(r"attention_|kv_write|kv_read|document_ranges", name.group(1)):
                continue
            seen += 1
            scratch = int(re.search(r"\.private_segment_fixed_size:\s*(\d+)", part).group(1))
            limit = max((n for k, n in ALLOWED.items() if k in name.group(1)), default=0)
            assert scratch <= limit, (name.group(1), scratch, limit)
    assert seen > 100
