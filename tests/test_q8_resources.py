"""What the 8-bit row kernels' builds take of a CU, from the compiler: the planner counts on the workgroups that fit."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2402_01869_amd import build


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{(head_dim, dtype, slim): (registers, bytes of LDS)}, the largest of the builds with and without merging."""
    if not shutil.which("hipcc"):
        pytest.skip("hipcc not on PATH")
    out = str(tmp_path_factory.mktemp("q8") / "rows.s")
    r = subprocess.run(["hipcc"] + [f for f in build.FLAGS if f != "-shared"] + ["--cuda-device-only", "-S", os.path.join(build.CSRC, "q8_rows.hip"), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    found = {}
    with open(out) as f:
        for slim, D, fmt, meta in re.findall(r"\.amdhsa_kernel \S*q8_rows_(slim_)?kernelILi(\d+)ELi(\d)E\S*\n(.*?)\.end_amdhsa_kernel", f.read(), re.S):
            need = tuple(int(re.search(r"\.amdhsa_%s (\d+)" % n, meta).group(1)) for n in ("next_free_vgpr", "group_segment_fixed_size"))
            key = int(D), int(fmt), bool(slim)
            found[key] = tuple(map(max, need, found.get(key, (0, 0))))
    return found


@pytest.mark.parametrize("fmt", [2, 3])
@pytest.mark.parametrize("D,places", [(64, 4), (128, 2), (256, 2)])
def test_workgroups_of_four_waves_on_a_cu(kernels, D, places, fmt):
    """Four waves of a workgroup are one on each SIMD, of 512 registers in steps of 8; 160 KiB of LDS."""
    vgpr, lds = kernels[D, fmt, False]
    assert 512 // (-(-vgpr // 8) * 8) >= places
    assert 160 * 1024 // lds >= places
