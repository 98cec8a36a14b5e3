"""The expert layer's host code under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only): nuna_expert_api.cpp and the
sort's plan, against stand-ins for the launchers (tests/c/expert_host_stub.cpp) that check every size again in 128 bits,
driven at the documented limits and at random (tests/c/expert_sanitize_driver.cpp)."""
import os
import subprocess

import pytest

from test_sanitizers import CSRC, ENV, ROOT, SAN, _have_gxx

pytestmark = pytest.mark.skipif(not _have_gxx(), reason="needs g++ and the HIP headers")


def test_expert_host_code_is_clean_under_sanitizers():
    out = os.path.join(ROOT, "_build", "asan_expert")
    os.makedirs(out, exist_ok=True)
    exe = os.path.join(out, "expert_sanitize_driver")
    c = os.path.join(ROOT, "tests", "c")
    subprocess.run(["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
                    *(os.path.join(CSRC, f) for f in ("nuna_api.cpp", "nuna_expert_api.cpp", "nap_planner.cpp")),
                    *(os.path.join(c, f) for f in ("hip_host_stub.cpp", "expert_host_stub.cpp", "expert_sanitize_driver.cpp")),
                    "-o", exe], check=True, capture_output=True, text=True)
    r = subprocess.run([exe], env=ENV, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-6000:]
    assert "0 failed expectations, 0 failed launch checks" in r.stdout, r.stdout
