"""What the compiler makes of the norms' kernels: which variants there are, their wavefronts on a SIMD, and spilled registers, which their rules were
measured with."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2106_05609_amd import _build


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs the compiler")
def test_norms_keep_their_wavefronts():
    cmd = ["hipcc"] + [f for f in _build.FLAGS if f != "-shared"] + ["-c", os.path.join(_build.HERE, "csrc", "norm.hip"), "-o", os.devnull,
                                                                   "-Rpass-analysis=kernel-resource-usage"]
    text = subprocess.run(cmd, check=True, capture_output=True, text=True).stderr
    got = {}
    for part in text.split("Function Name:")[1:]:
        name = re.search(r"residual_norm_(bwd_)?rows_kernelILb(\d)ELi(\d+)ELi(\d+)ELi(\d)ELb(\d)ELb(\d)E", part)
        if name:
            bwd, bf, g, w, p, mask, all_ = (name.group(1) is not None, *map(int, name.groups()[1:]))
            got[bwd, bf, g, w, p, mask, all_] = (int(re.search(r"Occupancy \[waves/SIMD\]: (\d+)", part).group(1)),
                                                 int(re.search(r"VGPRs Spill: (\d+)", part).group(1)))
    narrow, one, several = [(1, 1, 1), (2, 1, 1), (4, 1, 1)], [(8, 1, 1), (16, 1, 1), (32, 1, 1)], [(64, 1, 2), (64, 1, 3)]
    wide = [(64, 1, 1), (64, 4, 1), (64, 6, 1), (64, 8, 1), (64, 12, 1), (64, 16, 1)]
    least = {}
    for bf in (0, 1):
        for mask in (0, 1):
            for layout in one + several + wide:            # (lanes of a row, wavefronts, pieces of a lane)
                least[(False, bf, *layout, mask, 1)] = 3 if bf else 4
            for layout in narrow + one + several + wide:
                least[(False, bf, *layout, mask, 0)] = 3 if bf else 4
                least[(True, bf, *layout, mask, 0)] = 1 if bf and layout == (64, 1, 3) else 2 if bf or layout == (64, 1, 3) else 3 if layout == (64, 1, 2) else 4
            for layout in one + several:                   # backward, known beforehand: where its registers pay
                least[(True, bf, *layout, mask, 1)] = 1 if bf and layout in several else 2 if bf or layout in several else 3
    assert set(got) == set(least)
    bad = {k: (got[k], n) for k, n in least.items() if got[k][0] < n}
    assert not bad
    spills = {k: s for k, (_, s) in got.items() if s}
    assert all(k[0] and k[1] and k[3] in (12, 16) and s <= {12: 20, 16: 110}[k[3]] for k, s in spills.items()), spills
