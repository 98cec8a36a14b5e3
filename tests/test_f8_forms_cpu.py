"""The forms of the 8-bit products that are built are those that a call can reach (CPU only: the names of the kernels in the
library that is built)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_00867_amd import nuna

F32_SCALE, E8M0 = 0, 1
F32_OUT, BF16_OUT = 0, 1
ALL = {(s, o) for s in (F32_SCALE, E8M0) for o in (F32_OUT, BF16_OUT)}

# Rows and columns of a tile, waves along each, stages, weights' gradient: the pairs of scale and result that reach it.
TILES = {(256, 256, 4, 2, 2, False): {(s, BF16_OUT) for s in (F32_SCALE, E8M0)},
         (128, 256, 2, 4, 3, False): ALL, (64, 128, 2, 2, 3, False): ALL, (64, 64, 2, 2, 4, False): ALL,
         (128, 128, 2, 2, 2, True): {(F32_SCALE, F32_OUT)},
         (128, 128, 4, 2, 2, True): ALL - {(F32_SCALE, F32_OUT)}}
FEW = {(1, 4, 4): ALL, (1, 1, 8): ALL, (1, 2, 8): ALL, (2, 2, 8): ALL}


@pytest.mark.skipif(shutil.which("nm") is None or not os.path.exists(nuna.LIB_PATH), reason="needs nm and the library")
def test_only_forms_that_a_call_reaches_are_built():
    names = subprocess.run(["nm", "-C", nuna.LIB_PATH], capture_output=True, text=True, check=True).stdout
    tiles, few = {}, {}
    for args in set(re.findall(r"__device_stub__k_f8_tiles<([^>]*)>", names)):
        *shape, kind, wgrad, out = (a.strip() for a in args.split(","))
        tiles.setdefault((*map(int, shape), wgrad == "true"), set()).add((int(kind), int(out)))
    for args in set(re.findall(r"__device_stub__k_f8_few<([^>]*)>", names)):
        *shape, kind, out = map(int, args.split(","))
        few.setdefault(tuple(shape), set()).add((kind, out))
    assert tiles == TILES and few == FEW
