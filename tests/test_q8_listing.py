"""The 8-bit tile kernels' listing, checked as the bf16 ones' is: accumulation registers named by number, wait states."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2402_01869_amd import build
from test_tile_listing import check, overwritten, parse


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    if not shutil.which("hipcc"):
        pytest.skip("hipcc not on PATH")
    out = str(tmp_path_factory.mktemp("q8") / "q8.s")
    r = subprocess.run(["hipcc"] + [f for f in build.FLAGS if f != "-shared"] + ["--cuda-device-only", "-S", os.path.join(build.CSRC, "q8_tile.hip"), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    with open(out) as f:
        return f.read()


@pytest.mark.parametrize("fmt", [2, 3])
@pytest.mark.parametrize("D,own", [(64, 56), (128, 104), (256, 104)])
def test_accumulation_registers_and_wait_states(listing, D, own, fmt):
    start = re.search(r"^\S*q8_tile_kernelILi%dELi%dE\S*:" % (D, fmt), listing, re.M).start()
    text = listing[start:listing.index(".section", start)]
    meta = listing[listing.index(".amdhsa_kernel", start):]
    assert int(re.search(r"\.amdhsa_next_free_vgpr (\d+)", meta).group(1)) <= 208        # two waves a SIMD, and one of the rows
    assert int(re.search(r"\.amdhsa_private_segment_fixed_size (\d+)", meta).group(1)) == 0
    insts, labels = parse(text)
    mine = [i for i in insts if i.asm and re.search(r"\ba\[", i.code)]
    assert sum("mfma" in i.code for i in mine) >= 60
    assert overwritten(insts, labels, own) == []
    assert check(insts, labels) == []


def test_rows_that_run_beside_the_tiles_fit_the_registers_left(tmp_path):
    """Two tile waves of 208 registers leave 96 of a SIMD's 512."""
    if not shutil.which("hipcc"):
        pytest.skip("hipcc not on PATH")
    out = str(tmp_path / "q8_rows.s")
    r = subprocess.run(["hipcc"] + [f for f in build.FLAGS if f != "-shared"] + ["--cuda-device-only", "-S", os.path.join(build.CSRC, "q8_rows.hip"), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    with open(out) as f:
        text = f.read()
    found = re.findall(r"\.amdhsa_kernel (\S*q8_rows_(slim_)?kernel\S*)\n(.*?)\.end_amdhsa_kernel", text, re.S)
    assert sum(bool(slim) for _, slim, _ in found) == 4 and len(found) == 16
    for _, slim, meta in found:
        assert int(re.search(r"\.amdhsa_next_free_vgpr (\d+)", meta).group(1)) <= (96 if slim else 256)
        assert int(re.search(r"\.amdhsa_private_segment_fixed_size (\d+)", meta).group(1)) == 0
        if not slim:  # two workgroups on a CU
            assert int(re.search(r"\.amdhsa_group_segment_fixed_size (\d+)", meta).group(1)) <= 80 * 1024
