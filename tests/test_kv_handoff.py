"""The chunk kernel's exchange of maxima through columns of O against the first product that writes O, in every order in which the
warps can take their steps (kv_handoff.h, kv_handoff_check.cpp).  No GPU."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("handoff") / "check")
    subprocess.run(["g++", "-O1", "-std=c++17", os.path.join(HERE, "kv_handoff_check.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("tiles", [1, 2, 5])
def test_no_product_writes_over_maxima_that_are_still_to_be_read(check, tiles):
    states, early, stuck = map(int, subprocess.run([check, str(tiles)], check=True, capture_output=True, text=True).stdout.split())
    assert states > 10 and stuck == 0
    assert early == 0
