"""Rows may start at any element: accesses of 16 bytes say so to the compiler, in every kernel that makes them (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

from paper_2006_02924_amd import build


@pytest.mark.parametrize("source", ["adasum_embedding.hip", "adasum_checkpoint.hip", "adasum_weight_grad.hip"])
def test_no_access_claims_more_alignment_than_its_rows_have(source):
    if shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"):
        pytest.skip("no hipcc")
    subprocess.run([build.hipcc(), "-std=c++17", "-fsyntax-only", "--cuda-device-only", "-Wno-unused-command-line-argument",
                    "-Werror=align-mismatch", *build.DEVICE_FLAGS, "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                    os.path.join(build.CSRC, source)], check=True)
