"""How a batch over the paged K/V cache is cut into pieces (kv_plan.h): every row meets every key that it sees, once, whatever the
lengths; no worker has much more to do than another.  No GPU."""
import os
import subprocess

import pytest

import kv_reference as ref

HERE = os.path.dirname(os.path.abspath(__file__))
FEW, TILES = (16, 128, 296, 2, 2 ** 31 - 1, 1.5), (256, 128, 148, 4, 512, 2.0)


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "check")
    subprocess.run(["g++", "-O1", "-std=c++17", os.path.join(HERE, "kv_plan_check.cpp"), "-o", exe], check=True)

    def run(seqs, group, kv_heads, causal_block, cut):
        args = [group, kv_heads, causal_block, *cut, *(f"{r},{n}" for r, n in seqs)]
        lines = subprocess.run([exe, *map(str, args)], check=True, capture_output=True, text=True).stdout.splitlines()
        workers, n, slots, joins = map(int, lines[0].split())
        names = ("seq_row0", "kv_head", "row0", "rows", "key0", "key1", "slot", "first_slot", "parts", "join", "next")
        pieces = [dict(zip(names, map(int, line.split()))) for line in lines[1:1 + n]]
        seen = [list(map(int, line.split())) for line in lines[1 + n:]]
        return workers, pieces, slots, joins, seen

    return run


CASES = [
    ([(1, 1)], 1, 1, 0, FEW),
    ([(1, 262)], 1, 16, 0, FEW),
    ([(1, 520500)], 1, 16, 0, FEW),
    ([(1, 4164 - 61 * i) for i in range(48)], 1, 16, 0, FEW),
    ([(2, 700), (0, 50), (5, 5), (4, 0), (1, 9001)], 3, 2, 1, FEW),
    ([(16, 128)], 1, 3, 7, FEW),
    ([(17, 17)], 1, 1, 0, TILES),
    ([(1041, 52050)], 1, 16, 0, TILES),
    ([(4164, 41640)], 1, 16, 1041, TILES),
    ([(2748, 21984)], 1, 16, 1374, TILES),
    ([(1741, 4099), (435, 1025), (900, 900), (18, 3000), (300, 100)], 4, 8, 1, TILES),
    ([(300, 83280 * 3)], 1, 2, 0, TILES),                 # longer than a piece may be
    ([(200, 0), (200, 10)], 1, 2, 1, TILES),              # rows that see nothing
    ([(100, 1000)], 8, 1, 2 ** 30, TILES),                # a block longer than the chunk
    ([(100, 129), (129, 5000)], 1, 1, 1, (128, 128, 7, 4, 512, 3.0)),
]


@pytest.mark.parametrize("seqs,group,kv_heads,causal_block,cut", CASES)
def test_every_row_meets_the_keys_that_it_sees_once(plan, seqs, group, kv_heads, causal_block, cut):
    row_block, unit, max_workers, min_units, max_units, overhead = cut
    workers, pieces, slots, joins, seen = plan(seqs, group, kv_heads, causal_block, cut)
    seen = [s for s in seen]
    assert 1 <= workers <= max_workers
    starts, at = {}, 0
    for (rows, length), s in zip(seqs, (x for x in _per_sequence(seqs, seen))):
        assert s == [ref_seen(length, rows, causal_block, i) for i in range(rows)]
        if rows:
            starts[at] = (rows, length, s)
        at += rows
    by_rows = {}
    for p in pieces:
        by_rows.setdefault((p["seq_row0"], p["kv_head"], p["row0"]), []).append(p)
    wanted = {(r0, h, b) for r0, (rows, _, _) in starts.items() for h in range(kv_heads) for b in range(0, rows * group, row_block)}
    assert set(by_rows) == wanted
    used, counters = set(), {}
    for (r0, h, b), parts in by_rows.items():
        rows, length, s = starts[r0]
        n = min(row_block, rows * group - b)
        last = max(0, s[(b + n - 1) // group])
        parts.sort(key=lambda p: p["key0"])
        assert all(p["rows"] == n for p in parts)
        assert parts[0]["key0"] == 0 and parts[-1]["key1"] == last
        assert all(x["key1"] == y["key0"] for x, y in zip(parts, parts[1:])) and all(p["key0"] % unit == 0 for p in parts)
        assert all(p["key1"] > p["key0"] for p in parts) or last == 0
        assert all(p["key1"] - p["key0"] <= max_units * unit for p in parts)
        if len(parts) == 1:
            assert parts[0]["slot"] == -1
            continue
        assert [p["slot"] for p in parts] == list(range(parts[0]["first_slot"], parts[0]["first_slot"] + len(parts)))
        assert all(p["parts"] == len(parts) and p["join"] == parts[0]["join"] for p in parts)
        used |= {p["slot"] for p in parts}
        assert counters.setdefault(parts[0]["join"], (r0, h, b)) == (r0, h, b)
    assert used == set(range(slots)) and set(counters) == set(range(joins))
    # the chains: worker w begins with piece w, every piece belongs to one worker
    met, loads = [], []
    for w in range(workers):
        load, i = 0.0, w
        while i >= 0:
            p = pieces[i]
            met.append(i)
            load += -(-(p["key1"] - p["key0"]) // unit) * (0.65 if 2 * p["rows"] <= row_block else 1.0) + overhead
            i = p["next"]
        loads.append(load)
    assert sorted(met) == list(range(len(pieces)))
    share = sum(loads) / max_workers
    assert max(loads) <= 1.1 * share + 2 * (min_units + overhead) + 1


def ref_seen(length, rows, causal_block, i):
    return length if causal_block == 0 else min(length, length - rows + (i // causal_block + 1) * causal_block)


def _per_sequence(seqs, lines):
    """Sequences without rows print no line."""
    lines = iter(lines)
    for rows, _ in seqs:
        yield next(lines) if rows else []


def test_the_reference_says_the_same_of_what_rows_see():
    for length, rows, c in ((10, 4, 1), (10, 4, 3), (3, 8, 1), (0, 5, 2), (7, 7, 100)):
        for i in range(rows):
            assert ref.seen(length, rows, c, i) == max(0, ref_seen(length, rows, c, i))
