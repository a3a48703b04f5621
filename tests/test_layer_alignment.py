"""Tensors are aligned to their elements and no more, in the sources of a selective layer too."""
import os
import subprocess

import pytest

from paper_1707_08265_amd import build as lib_build

OWN = ("causal_conv.hip", "select_forward.hip", "select_backward.hip", "dropout.hip", "gated_scan.hip", "select.h", "rows.h", "layer.h", "values.h")


@pytest.mark.parametrize("source", OWN[:5])
def test_no_access_assumes_more_than_its_element(source):
    r = subprocess.run(["hipcc", *lib_build.FLAGS, "-fsyntax-only", os.path.join(lib_build.CSRC, source)], capture_output=True,
                       text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    found = [line for line in r.stderr.splitlines() if "align-mismatch" in line and os.path.basename(line.split(":")[0]) in OWN]
    assert not found, found[:5]
