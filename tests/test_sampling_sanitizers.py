"""The sampling phase's host code (paged_api.cpp: argument checks, the division of calls among workgroups) under AddressSanitizer and
UndefinedBehaviorSanitizer, on the CPU: a native program goes through the C ABI with host-only plans and lengths of every kind, and the same arithmetic runs in
the kernels."""
import os

import pytest

from tests.test_host_sanitizers import CSRC, NATIVE, ROOT, SAN_ENV, run


def test_sampling_host_side_under_sanitizers(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    exe = str(tmp_path / "paged_driver")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
    run([hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-x", "hip", *san, "-Wno-unused-command-line-argument",
         f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}", os.path.join(CSRC, "paged_api.cpp"), os.path.join(NATIVE, "paged_driver.cpp"), "-o", exe])
    assert "paged_driver: ok" in run([exe], env=SAN_ENV)
