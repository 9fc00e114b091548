"""The kernels of heads, cache and attention keep all they hold in registers: what the compiler says of the built library."""
import os
import re
import subprocess

import pytest

from paper_2602_15563_amd import kmq
from tests.test_lds_reads_in_flight import device_code
from tests.test_matrix_core_scratch import READELF


@pytest.mark.skipif(not os.path.exists(READELF), reason="no reader for the notes of code built here")
def test_no_instance_spills(tmp_path):
    path, seen, spilled = tmp_path / "code", [], []
    for code in device_code(kmq.LIB_PATH):
        path.write_bytes(code)
        notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, check=True).stdout
        for kernel in re.split(r"\n  - \.", notes)[1:]:
            name = re.search(r"\.name:\s+(\S*(?:attn_|heads_|kv_read_)\S*kernel\S*)", kernel)
            if name:
                seen.append(name[1])
                if re.search(r"\.private_segment_fixed_size:\s+[1-9]", kernel):
                    spilled.append(name[1])
    assert len(seen) >= 5 + 3 + 6 + 16 + 2, seen               # turns of waves, tiles, joins; heads; reads
    assert not spilled
