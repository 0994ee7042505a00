"""The attention's and the cache's kernels as built: their sums, fragments and
blocks on the way stay in registers through their loops.  Memory of a lane's own
would also be waited for with the copies that run beside the products."""

import os
import re
import subprocess

import pytest

from paper_2607_14530_amd import xhc as X
from tests.test_lds_copies import code_objects

READELF = "/opt/rocm/llvm/bin/llvm-readelf"
KERNELS = ("k_attn", "k_rotate", "k_cache")


@pytest.mark.skipif(not (os.path.exists(READELF) and os.path.exists(X.LIB_PATH)),
                    reason="needs the library and llvm-readelf")
def test_no_scratch_memory(tmp_path):
    seen, bad = 0, []
    for k, code in enumerate(code_objects()):
        path = str(tmp_path / f"{k}.o")
        open(path, "wb").write(code)
        notes = subprocess.run([READELF, "--notes", path], capture_output=True, text=True, check=True).stdout
        for part in re.split(r"\n\s+- \.agpr_count", notes)[1:]:
            name = re.search(r"\n    \.name:\s+(\S+)", part)[1]
            size = int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", part)[1])
            if any(n in name for n in KERNELS):
                seen += 1
                if size:
                    bad.append((name, size))
    assert seen > 100, seen
    assert not bad, bad
