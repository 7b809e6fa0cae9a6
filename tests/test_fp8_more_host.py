"""Layers in 8-bit floating point, what needs no GPU: waits, refusals, the harness's streams and devices, sizes, the quotient."""
import os
import re

from paper_2511_19438_b200 import build as libbuild


def test_no_uniform_branch_on_a_lane_s_own_try():
    """mbarrier.try_wait answers each lane for itself: a branch that promises one answer for the warp (bra.uni) may not hang on it."""
    for f in sorted(os.listdir(libbuild.CSRC)):
        with open(os.path.join(libbuild.CSRC, f)) as h:
            for asm in re.findall(r"asm\s+volatile\s*\((.*?)\);", h.read(), re.S):
                assert not ("try_wait" in asm and "bra.uni" in asm), f
