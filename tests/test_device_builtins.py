"""Sources compiled without IEEE mode: the device library is compiled with it, a function is not inlined into one of the other mode, and so threadIdx, blockIdx, gridDim,
blockDim and __umul24 would be calls whose results count as divergent.  These sources, and the headers of csrc/ that they include, use the builtins."""
import os
import re

import pytest

from paper_2409_12490_amd import build

WITHOUT_IEEE = sorted(src for src, flags in build.EXTRA.items() if "-mno-amdgpu-ieee" in flags)


def _with_headers(name, seen):
    if name in seen:
        return
    path = os.path.join(build.CSRC, name)
    if not os.path.exists(path):
        return
    with open(path) as f:
        seen[name] = re.sub(r"/\*.*?\*/|//[^\n]*", "", f.read(), flags=re.S)
    for other in re.findall(r'#include\s+"([^"]+)"', seen[name]):
        _with_headers(other, seen)


@pytest.mark.parametrize("src", WITHOUT_IEEE)
def test_no_calls_into_the_device_library(src):
    files = {}
    _with_headers(src, files)
    assert len(files) > 1
    for name, text in files.items():
        assert not re.findall(r"\b(?:threadIdx|blockIdx|gridDim|blockDim|__umul24)\b", text), name
