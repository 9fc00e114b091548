"""The instances of the experts' row kernel in the built library are those that calls reach, and the tests on the GPU go through all
that each of them does with a row."""
import os
import re
import subprocess

import pytest

from paper_2602_15563_amd import kmq
from tests.moe_launches import CASES, Instance, both, reachable
from tests.test_lds_reads_in_flight import device_code
from tests.test_matrix_core_scratch import READELF


@pytest.mark.skipif(not os.path.exists(READELF), reason="no reader for the notes of code built here")
def test_every_instance_is_reached(tmp_path):
    path, built = tmp_path / "code", set()
    for code in device_code(kmq.LIB_PATH):
        path.write_bytes(code)
        notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, check=True).stdout
        for m in re.finditer(r"moe_rows_kernelILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELb(\d)E", notes):
            built.add(Instance(*(int(n) for n in m.groups()[:5]), m[6] == "1"))
    reached = set(reachable())
    assert not reached - built, "the rules written out in moe_launches.py are not the library's"
    assert not built - reached, "built for no call"


def test_the_cases_go_through_every_path():
    seen = {}
    for case in CASES:
        for i, how in both(*case):
            seen.setdefault(i, set()).update(how)
    assert seen == reachable()
