"""Registers of the built microscaled kernels, from the code objects in libmsd.so (no
GPU): none spills or takes scratch memory, and none has more LDS than a workgroup may."""
import os
import re
import subprocess

import pytest

from test_kernel_resources import READELF, code_objects


def test_no_microscaled_kernel_spills(tmp_path):
    from paper_2505_14260_amd import msd
    if not os.path.exists(msd.LIB_PATH) or not os.path.exists(READELF):
        pytest.skip("libmsd.so not built")
    seen, bad = 0, []
    for i, obj in enumerate(code_objects(open(msd.LIB_PATH, "rb").read())):
        path = tmp_path / f"{i}.co"
        path.write_bytes(obj)
        notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True,
                               check=True).stdout
        for k in re.split(r"\n\s+- \.agpr_count", notes)[1:]:
            kernel = re.findall(r"\.symbol:\s+(\S+)", k)[0]
            if "k_mx_" not in kernel:
                continue
            seen += 1
            if int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", k).group(1)):
                bad.append(kernel)
            assert int(re.search(r"\.group_segment_fixed_size:\s+(\d+)", k).group(1)) <= 160 * 1024
    assert seen >= 60, seen
    assert not bad, bad
