"""What nuna_init makes of the dispatch probe (CPU only): the map of workgroups to XCDs may be turned as a whole, as it is
once a process has used several streams; any other difference leaves XCD placement refused.  libnuna's host side runs
against the stand-in runtime of hip_host_stub.cpp, whose probe rotated_probe_stub.cpp replaces."""
import os
import subprocess

import pytest

from paper_2608_00867_amd import nuna
from test_sanitizers import CSRC, ENV, ROOT, SAN, _have_gxx

pytestmark = pytest.mark.skipif(not _have_gxx(), reason="needs g++ and the HIP headers")


@pytest.fixture(scope="module")
def driver():
    out = os.path.join(ROOT, "_build", "init_rotated")
    os.makedirs(out, exist_ok=True)
    exe = os.path.join(out, "init_driver")
    c = os.path.join(ROOT, "tests", "c")
    subprocess.run(["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-I" + c, os.path.join(CSRC, "nuna_api.cpp"),
                    os.path.join(CSRC, "nap_planner.cpp"), os.path.join(c, "rotated_probe_stub.cpp"),
                    os.path.join(c, "init_driver.cpp"), "-o", exe], check=True, capture_output=True, text=True)

    def run(probe):
        r = subprocess.run([exe], env=dict(ENV, STUB_MAP=probe), capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr[-3000:]
        return r.stdout.strip()
    return run


@pytest.mark.parametrize("turn", range(8))
def test_a_turned_map_is_the_map(driver, turn):
    assert driver(f"turned {turn}") == f"init {nuna.OK} info {nuna.OK} verified 1 allreduce {nuna.OK}"


@pytest.mark.parametrize("probe", ["mod4", "one_off", "one_xcd", "far"])
def test_other_maps_leave_xcd_placement_refused(driver, probe):
    bad = nuna.ERR_UNSUPPORTED
    assert driver(probe) == f"init {bad} info {nuna.OK} verified 0 allreduce {bad}"
