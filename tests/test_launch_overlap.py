"""Source rule of kernels that start while the one before them still runs: what that kernel writes (query fragments and
factors, partial results) is read by plain loads.  Read-only loads are taken to read what never changes, so that a
compiler may move them above the wait for that kernel; a test on the GPU would only see it where one does."""
import glob
import os
import re

import pytest

from paper_2403_20137_b200 import build


def overlapped():
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*.cu")) + glob.glob(os.path.join(build.CSRC, "*.cuh"))):
        with open(path) as f:
            code = f.read()
        if "pdl_wait();" in code and "void pdl_wait()" not in code:
            yield pytest.param(code, id=os.path.basename(path))


@pytest.mark.parametrize("code", list(overlapped()))
def test_workspace_is_read_by_plain_loads(code):
    code = re.sub(r"//[^\n]*", "", code)
    written = r"qmeta|partials|qfrag|views|plan|dpos|scores|lse|kept|rows"
    assert not re.search(r"__restrict__\s+(%s)\b" % written, code)
    views = set(re.findall(r"(\w+)\s*=\s*reinterpret_cast<const uint4\*>\(a\.qfrag\)", code))
    for _ in range(3):                                   # pointers derived from them
        views |= {m[0] for m in re.findall(r"(\w+)\s*=\s*(\w+)\s*\+", code) if m[1] in views}
    for name in re.findall(r"__ldg\(\s*(?:reinterpret_cast<[^>]*>\()?\s*(?:a\.)?(\w+)", code):
        assert name not in views and not re.fullmatch(written, name), name
