"""The host and device arithmetic of the 8-bit products' tiles (csrc/tile_order.h) on the CPU, with overflow reported."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_00867_amd", "csrc")
OUT = os.path.join(ROOT, "_build", "tile_order")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_tile_arithmetic_holds_over_the_sizes_the_calls_take():
    os.makedirs(OUT, exist_ok=True)
    exe = os.path.join(OUT, "tile_order_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Werror", "-fsanitize=undefined",
                    "-fno-sanitize-recover=all", "-I" + CSRC, os.path.join(ROOT, "tests", "c", "tile_order_check.cpp"),
                    "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    assert ", 0 mismatches" in r.stdout, r.stdout
