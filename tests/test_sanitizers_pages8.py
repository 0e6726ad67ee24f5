"""Host code of the 8-bit cache under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only):
argument checks and launch plans (da_pages8_api.cpp on top of da_paged_api.cpp) with stub launchers and
a driver in tests/sanitize/.  No GPU code is built here.
"""
from __future__ import annotations

import os
import shutil

import pytest

from test_sanitizers import ENV, HERE, ROCM_LIB, ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists(ROCM_LIB + "/libamdhip64.so"),
                    reason="g++ or the HIP runtime library not found")
def test_pages8_host_layer_under_sanitizers(tmp_path):
    exe = str(tmp_path / "pages8_driver")
    csrc = os.path.join(ROOT, "paper_2505_11254_amd", "csrc")
    b = _run(["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
              "-I" + os.path.join(ROOT, "include"), "-I" + csrc, os.path.join(HERE, "pages8_driver.cpp"),
              os.path.join(csrc, "da_paged_api.cpp"), os.path.join(csrc, "da_pages8_api.cpp"),
              "-o", exe, "-L" + ROCM_LIB, "-Wl,-rpath," + ROCM_LIB, "-lamdhip64"])
    assert b.returncode == 0, b.stderr
    r = _run([exe], env=ENV)
    assert r.returncode == 0 and "runtime error" not in r.stderr, r.stdout + r.stderr
    assert "pages8 driver ok" in r.stdout
