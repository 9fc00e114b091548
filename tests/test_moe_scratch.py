"""Norms, router and experts keep what they hold in registers: what the compiler says of the built library.  The experts' kernels of 1 and 2
bits may put a few words of what is kept from item to item aside, outside the loop over a row."""
import os
import re
import subprocess

import pytest

from paper_2602_15563_amd import kmq
from tests.test_lds_reads_in_flight import device_code
from tests.test_matrix_core_scratch import READELF


@pytest.mark.skipif(not os.path.exists(READELF), reason="no reader for the notes of code built here")
def test_spills(tmp_path):
    path, seen = tmp_path / "code", {}
    for code in device_code(kmq.LIB_PATH):
        path.write_bytes(code)
        notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, check=True).stdout
        for kernel in re.split(r"\n  - \.", notes)[1:]:
            name = re.search(r"\.name:\s+(\S*(?:moe_|route_|block_norm)\S*kernel\S*)", kernel)
            if name:
                seen[name[1]] = int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", kernel)[1])
    assert sum("moe_rows" in k for k in seen) >= 40 and sum("route_" in k for k in seen) == 8 and sum("block_norm" in k for k in seen) == 3, seen
    spilled = {k: v for k, v in seen.items() if v}
    assert all(v <= 32 and re.search(r"moe_rows_kernelILi[12]ELi4E", k) for k, v in spilled.items()), spilled
