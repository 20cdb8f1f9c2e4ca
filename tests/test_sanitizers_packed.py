"""Host sanitizer build (CPU only) of the calls over packed rows and the 4-bit cache: validation and dispatch under
AddressSanitizer and UndefinedBehaviorSanitizer (g++, host code only), driven by tests/sanitize/abi_packed_driver.cpp."""
import os
import shutil

import pytest

from test_sanitizers import HERE, ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"),
                    reason="g++ or the ROCm headers not available")
def test_packed_abi_under_asan_ubsan(tmp_path):
    exe = str(tmp_path / "abi_packed_driver")
    csrc = os.path.join(ROOT, "paper_2609_21704_amd", "csrc")
    _run(["g++", "-std=c++17", *SAN, "-I", os.path.join(ROOT, "include"), "-I", csrc, "-I", "/opt/rocm/include",
          "-D__HIP_PLATFORM_AMD__", os.path.join(HERE, "abi_packed_driver.cpp"), os.path.join(csrc, "abi_packed.cpp"),
          "-o", exe])
    assert "ABI OK" in _run([exe], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1"))
