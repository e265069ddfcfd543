"""What the compiler reports for the kernels of layers in the clear, with the build's own flags: no scratch memory, which the runtime
would set up when such a kernel is first launched (the calls promise that nothing is allocated), and LDS within what lets as many workgroups
share a CU as the choice between tile sizes counts on."""
import os
import re
import shutil
import subprocess

import pytest

from paper_1806_03461_amd import build


def test_no_scratch_and_tiles_that_share_a_cu():
    if not shutil.which("hipcc"):
        pytest.skip("no hipcc")
    r = subprocess.run(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", "-Rpass-analysis=kernel-resource-usage", "-o", os.devnull,
                        os.path.join(build.CSRC, "clear_kernels.hip")], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert r.returncode == 0, r.stdout
    names = re.findall(r"Function Name: (\S+)", r.stdout)
    found = {key: [int(v) for v in re.findall(pattern + r": (\d+)", r.stdout)]
             for key, pattern in (("scratch", r"ScratchSize \[bytes/lane\]"), ("lds", r"LDS Size \[bytes/block\]"), ("waves", r"Occupancy \[waves/SIMD\]"))}
    assert all(len(v) == len(names) for v in found.values()), r.stdout
    assert [(n, s) for n, s in zip(names, found["scratch"]) if s] == []
    for kind in ("dense_few_kernel", "dense_tile_kernel", "rows_kernel"):
        assert any(kind in n for n in names), kind
    # tiles of 32 x 64 three to a CU, of 64 x 64 two, four waves each, a wave a SIMD; the others one
    for tile, at_once in (("ILi1ELi4ELi2ELi1ELi128E", 3), ("ILi2ELi2ELi2ELi2ELi128E", 2)):
        of_tile = [(n, lds, waves) for n, lds, waves in zip(names, found["lds"], found["waves"]) if "dense_tile_kernel" + tile in n]
        assert len(of_tile) == 2 and all(lds * at_once <= 160 * 1024 and waves >= at_once for _, lds, waves in of_tile), of_tile
