"""What the digest of the measured kernels' sources covers, so that a profile of theirs goes stale with them alone."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2411_18462_amd", "csrc")


def test_the_measured_sources_name_nothing_of_the_heads_calls():
    files, left = {}, ["svip_kernels.hip"]
    while left:
        f = left.pop()
        if f not in files and "/" not in f:
            files[f] = open(os.path.join(CSRC, f)).read()
            left += re.findall(r'^#include "([^"]+)"', files[f], re.M)
    assert "svip_internal.h" in files and "host_calls.h" not in files
    for f, text in files.items():
        assert not re.findall(r"\b(?:mx|head)_\w+", text), f
