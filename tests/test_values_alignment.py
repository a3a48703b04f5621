"""Tensors are aligned to their elements and no more, and the compiler has to know: what it assumes of an address it may use."""
import os
import subprocess

import pytest

from paper_1707_08265_amd import build as lib_build


@pytest.mark.parametrize("source", ["gated_scan.hip", "tensor_lists.hip"])
def test_no_access_assumes_more_than_its_element(source):
    r = subprocess.run(["hipcc", *lib_build.FLAGS, "-fsyntax-only", os.path.join(lib_build.CSRC, source)], capture_output=True,
                       text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    own = ("gated_scan.hip", "tensor_lists.hip", "values.h")
    found = [line for line in r.stderr.splitlines() if "align-mismatch" in line and os.path.basename(line.split(":")[0]) in own]
    assert not found, found[:5]
