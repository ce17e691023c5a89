"""Registers of kernels whose speed hangs on how many of their CTAs fit an SM, from the report that ptxas wrote when the library was built."""
import os
import re
import subprocess

import pytest

from paper_2603_15619_b200 import build

REPORT = os.path.join(build.PKG, "build_ptxas.log")

# the merge of the plain decode step: 16 CTAs of 128 threads an SM at 32 registers, 12 at up to 40
LIMITS = {"decode_merge_kernel<64, false>": 32, "decode_merge_kernel<128, false>": 40}


def registers():
    found, name = {}, None
    for line in open(REPORT):
        if m := re.search(r"Compiling entry function '(\S+)'", line):
            name = m.group(1)
        elif (m := re.search(r"Used (\d+) registers", line)) and name:
            found.setdefault(name, int(m.group(1)))
    plain = subprocess.run(["c++filt"], input="\n".join(found), capture_output=True, text=True, check=True).stdout.splitlines()
    return {n.split("(")[0].replace("void ", "").replace("moda::", ""): v for n, v in zip(plain, found.values())}


@pytest.mark.skipif(not os.path.exists(REPORT), reason="the library was not built here")
@pytest.mark.parametrize("kernel", LIMITS)
def test_registers_stay_within_limits(kernel):
    assert registers()[kernel] <= LIMITS[kernel]
