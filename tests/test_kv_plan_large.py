"""Batches at the ends of what a batch may hold are cut like any other (kv_plan.h).  No GPU."""
import os
import resource
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-fsanitize=undefined,float-cast-overflow", "-fno-sanitize-recover=all", os.path.join(HERE, "kv_plan_large_check.cpp"), "-o", exe], check=True)

    def run(*args):
        limit = lambda: resource.setrlimit(resource.RLIMIT_AS, (6 << 30, 6 << 30))  # (rows without an end would take all memory)
        done = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=120, preexec_fn=limit)
        assert done.returncode == 0, done.stderr
        return tuple(map(int, done.stdout.split()))

    return run


@pytest.mark.parametrize("rows", [2 ** 31 - 1, 2 ** 31 - 128, 2 ** 31 - 257])
def test_rows_up_to_the_last_that_a_batch_may_have(cut, rows):
    """The last block of rows ends at the end of the 32-bit range."""
    workers, pieces, covered, units = cut(rows, 1, 256, 148)
    assert (workers, covered) == (148, rows) and pieces == units == -(-rows // 256)


def test_shares_beyond_32_bits(cut):
    """520 blocks of one row over 2^30 tokens, two workers: a share is more than 2^31 units of keys, and pieces are as long as they may be."""
    workers, pieces, covered, units = cut(520, 2 ** 30, 1, 2)
    assert workers == 2 and covered == 520 and units == 520 * 2 ** 23
    assert pieces <= 520 * 2 ** 23 // 512 + 1
