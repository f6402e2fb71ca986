"""What a batch is planned with for tallies, by whether its cache has any.  On stand-ins for the CUDA runtime and the kernel launchers.  No GPU."""
import numpy as np
import pytest

import test_kv_evict_host as base
from test_kv_evict_host import OK, batch, host, plan, weigh  # noqa: F401


@pytest.mark.parametrize("rows,lengths,q_heads", [([1000], [1000], 20), ([300, 2], [300, 40], 20), ([1041], [2000], 2)])
def test_a_cache_without_tallies_pays_for_none(host, rows, lengths, q_heads):
    """No trial cuts, no memory for parts of sums: the lists of where its sequences' keys begin are all that is there."""
    counts = [-(-n // 128) for n in lengths]
    args = rows, lengths, np.arange(sum(counts)) % 16, q_heads
    cache = base.base.cache_of(host, pages=16, page_size=128)
    b = batch(host, cache, *args)
    with_tallies, without = plan(host, batch(host, base.tracked(host, page_size=128), *args)), plan(host, b)
    assert with_tallies["parts"] > 1 and without["parts"] == 1
    sums = 4 * with_tallies["items"] * with_tallies["parts"] * with_tallies["block"]
    assert with_tallies["bytes"] - without["bytes"] >= sums - 256  # (what is empty takes 256)
    assert without["few"] == with_tallies["few"] and without["items"] > 0
    # tallies that come later are taken all the same
    before = host.fake_weighs()
    assert host.litevggt_kv_track(cache, base.base.memory(64)) == OK and weigh(host, cache, b) == OK and host.fake_weighs() > before


def test_sequences_of_few_rows_beside_one_of_many_leave_most_parts_empty(host):
    """(The batch of the GPU test of the same name.)"""
    rows, lengths = [4000, 17, 20, 40, 30, 9], [300, 300, 280, 900, 500, 260]
    counts = [-(-n // 32) for n in lengths]
    cache = base.base.cache_of(host, pages=sum(counts), page_size=32, kv_heads=4)
    assert host.litevggt_kv_track(cache, base.base.memory(64)) == OK
    p = plan(host, batch(host, cache, rows, lengths, np.arange(sum(counts)), 16))
    tiles = [-(-4 * r // 128) for r in rows]
    units = [4 * -(-n // p["block"]) * p["parts"] for n in lengths]
    full = [4 * -(-n // p["block"]) * min(t, p["parts"]) for n, t in zip(lengths, tiles)]
    assert p["parts"] > 2 and sum(units) > 148 and sum(full) < sum(units) / 2
