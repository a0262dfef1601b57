"""The traffic figures that bench.py reports are for the sources that they were
taken with: every header that shapes a kernel counts as one of its sources."""
import os
import re

import bench
import pytest

CSRC = os.path.join(os.path.dirname(os.path.abspath(bench.__file__)), "paper_2509_24626_amd", "csrc")


@pytest.mark.parametrize("kernel", sorted(bench.KERNEL_SOURCES))
def test_headers_of_a_kernel_are_among_its_sources(kernel):
    """All of its own headers; internal.hpp has the library's error reporting and the launch, and is everyone's."""
    listed = bench.KERNEL_SOURCES[kernel]
    for name in listed:
        with open(os.path.join(CSRC, name)) as f:
            headers = re.findall(r'#include "(\w+\.hpp)"', f.read())
        assert set(headers) - {"internal.hpp"} <= set(listed), name
