"""How a plan's work units are launched and their results joined (hb_plan.cpp, no HIP), windowed or not, as layers
launch them and as hb_attention does from its records: every tile and item group is launched once, every row of every
kv head has one writer or one group of parts, a group's parts are those that its units write, over key ranges that
follow each other, in slots that nothing else writes, and all of its columns are merged once."""
import copy
import os
import subprocess
from collections import defaultdict

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_22562_amd", "csrc")
SINGLE, MERGED, TILE = 1, 2, 0
WAVES, ITEM_COLS = 4, 16

SHAPES = {"tiny": (256, 4, 2, 64, 688), "g1": (512, 4, 4, 128, 336), "g16": (1024, 16, 1, 64, 512),
          "tp8": (256, 8, 1, 128, 64), "8b": (64, 32, 8, 128, 16)}


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "wiring_driver")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    f"-I{CSRC}", f"-I{os.path.join(ROOT, 'include')}", os.path.join(ROOT, "tests", "wiring_driver.cpp"),
                    os.path.join(CSRC, "hb_plan.cpp"), "-o", exe], check=True)
    return exe


def run(exe, shape, cu, fit, reqs, window=0, sinks=0, split_tile=0, split_item=0):
    text = " ".join(map(str, (*shape, cu, int(fit), window, sinks, split_tile, split_item, len(reqs))))
    text += "\n" + "\n".join(f"{c} {x}" for c, x in reqs) + "\n"
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0")
    env.pop("LD_PRELOAD", None)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, env=env)
    assert out.returncode == 0, out.stderr[-2000:]
    plan = defaultdict(list)
    for ln in out.stdout.splitlines():
        k, *v = ln.split()
        plan[k].append([int(t) for t in v])
    return plan


def check(plan, shape, reqs):
    _, nq, nkv, _, _ = shape
    G = nq // nkv
    tile_cols, n_slots, n_tiles, n_items = plan["geom"][0]
    starts = np.concatenate([[0], np.cumsum([c for c, _ in reqs])])
    # launches
    units = [plan["wave"][i:i + WAVES] for i in range(0, len(plan["wave"]), WAVES)]
    tiles, groups4, results = [], [], []
    for waves in units:
        kinds = {w[0] for w in waves}
        assert len(kinds) == 1 and len(waves) == WAVES
        kind, items = kinds.pop(), [w[2:] for w in waves]
        if kind == TILE:
            assert all(w[1:] == waves[0][1:] for w in waves)
            tiles.append(waves[0][1])
            results.append((tile_cols, items[0]))
            continue
        groups4.append(waves[0][1] // WAVES)
        assert [w[1] for w in waves] == [WAVES * groups4[-1] + i for i in range(WAVES)]
        full = [it for it in items if it[5] < it[6]]
        assert full
        if kind == SINGLE:
            results += [(ITEM_COLS, it) for it in full]
            continue
        # one result of consecutive ranges; the empty ones are last
        assert kind == MERGED and full == items[:len(full)]
        assert all(it[:5] + it[7:] == items[0][:5] + items[0][7:] for it in items)
        assert all(a[6] == b[5] for a, b in zip(full, full[1:]))
        results.append((ITEM_COLS, items[0][:6] + [full[-1][6], items[0][7]]))
    assert sorted(tiles) == list(range(n_tiles)), "tiles not launched once each"
    assert sorted(groups4) == list(range(n_items // WAVES)) and n_items % WAVES == 0, "items not launched once each"
    # results
    writers, parts, used = defaultdict(list), defaultdict(list), np.zeros(n_slots, np.int64)
    for cols, (req, g, tok0, pos0, npos, kb, ke, part) in results:
        assert 0 <= g < nkv and npos >= 1 and npos * G <= cols and 0 <= kb < ke and kb % 64 == 0
        assert starts[req] <= tok0 and tok0 + npos <= starts[req + 1]
        if part < 0:
            assert (kb, ke) == (0, pos0 + npos)
            for t in range(tok0, tok0 + npos):
                writers[(t, g)].append("unit")
        else:
            assert part + npos * G <= n_slots
            used[part:part + npos * G] += 1
            parts[(tok0, g)].append((part, npos, pos0, kb, ke))
    assert (used <= 1).all(), "two parts in one slot"
    # merges
    merged = defaultdict(list)
    for *group, cols in plan["merge"]:
        merged[tuple(group)].append(cols)
    for (part0, nparts, stride, tok0, npos, g), cols in merged.items():
        assert sorted(cols) == list(range(-(-npos * G // 16))), "columns not merged once each"
        mine = sorted(parts.pop((tok0, g)))
        assert nparts > 1 and npos * G <= stride
        assert [p[0] for p in mine] == [part0 + s * stride for s in range(nparts)], "not the parts that are written"
        assert all(p[1:3] == (npos, mine[0][2]) for p in mine)
        assert mine[0][3] == 0 and mine[-1][4] == mine[0][2] + npos
        assert all(a[4] == b[3] for a, b in zip(mine, mine[1:])), "key ranges do not follow each other"
        for t in range(tok0, tok0 + npos):
            writers[(t, g)].append("merge")
    assert not parts, "parts that nothing merges"
    assert set(writers) == {(t, g) for t in range(starts[-1]) for g in range(nkv)}
    assert all(len(w) == 1 for w in writers.values()), "a row has several writers"


LAUNCHES = [
    ("tp8", 256, [(1, 300)], 0, 0), ("tp8", 256, [(1, 30000)], 0, 0), ("g1", 256, [(1, 9000)] * 8, 500, 0),
    ("8b", 256, [(64, 500)], 0, 0), ("8b", 256, [(128, 1000)], 300, 20), ("8b", 256, [(256, 200)], 0, 0),
    ("8b", 256, [(64, 2000)] + [(1, 3000)] * 4, 0, 0), ("8b", 256, [(512, 0)], 0, 0), ("8b", 256, [(1024, 1000)], 0, 0),
    ("8b", 256, [(512, 3431)] + [(1, 512 + 56 * i) for i in range(64)], 1024, 4), ("8b", 256, [(2048, 0)], 0, 0),
    ("tp8", 256, [(512, 2000)], 0, 0), ("tp8", 256, [(576, 0)] * 2, 0, 0), ("tp8", 256, [(64, 16000), (1, 100)], 0, 0),
    ("g16", 64, [(40, 600), (7, 90), (1, 3000)], 250, 47), ("tiny", 64, [(200, 0), (300, 1000)], 33, 21),
    ("tiny", 256, [(77, 1000)] + [(1, 80 * i) for i in range(9)], 100, 3), ("g1", 16, [(1, 5), (1, 0), (3, 64)], 1, 0),
]


@pytest.mark.parametrize("fit", [False, True], ids=["layer", "handle"])
@pytest.mark.parametrize("name,cu,reqs,window,sinks", LAUNCHES, ids=range(len(LAUNCHES)))
def test_launches(driver, fit, name, cu, reqs, window, sinks):
    check(run(driver, SHAPES[name], cu, fit, reqs, window, sinks), SHAPES[name], reqs)


@pytest.mark.parametrize("seed", range(60))
def test_random_launches(driver, seed):
    rng = np.random.default_rng(seed)
    shape = SHAPES[list(SHAPES)[seed % len(SHAPES)]]
    reqs = [(int(rng.choice([1, 1, rng.integers(1, 20), rng.integers(20, 700)])), int(np.exp(rng.uniform(0, 9.5))))
            for _ in range(rng.integers(1, 12))]
    window = int(rng.choice([0, 0, np.exp(rng.uniform(0, 9))]))
    plan = run(driver, shape, int(rng.choice([1, 16, 64, 256])), rng.random() < 0.8, reqs, window,
               int(rng.choice([0, 4, rng.integers(0, 80)])), int(rng.choice([0, 0, 64, 512])),
               int(rng.choice([0, 0, 64, 256])))
    check(plan, shape, reqs)


@pytest.mark.parametrize("fit", [False, True], ids=["layer", "handle"])
def test_the_most_keys_of_a_launch(driver, fit):
    """Heads and context at the interface's limits: 2^44 keys over 4096 waves are 2^32 each."""
    shape, reqs = (64, 1 << 14, 1 << 14, 64, 16), [(1, (1 << 30) - 1)]
    check(run(driver, shape, 256, fit, reqs), shape, reqs)


def test_the_check_sees_a_wrong_plan(driver):
    """Mistakes planted in a plan's text: a unit launched twice in another's place, parts that share a slot, a part or
    a column block that is not merged, a key range that misses a step."""
    shape, reqs = SHAPES["8b"], [(64, 2000)] + [(1, 3000)] * 4
    good = run(driver, shape, 256, True, reqs)
    check(good, shape, reqs)
    tile = next(i for i, w in enumerate(good["wave"]) if w[0] == TILE and w[-1] >= 0)
    item = next(i for i, w in enumerate(good["wave"]) if w[0] == MERGED and w[-1] >= 0)

    def twice(p):
        p["wave"][item:item + WAVES] = p["wave"][item + WAVES:item + 2 * WAVES]

    def shared_slot(p):
        for w in p["wave"]:
            if w[0] == MERGED and w[-1] >= 0 and w[4:6] == p["wave"][item][4:6]:
                w[-1] = p["wave"][item][-1]

    def part_left_out(p):
        for m in p["merge"]:
            if m[0] == p["wave"][tile][-1] or m[2] == 128:
                m[1] -= 1

    def part_too_many(p):
        p["merge"][0][1] += 1

    def column_left_out(p):
        del p["merge"][0]

    def keys_left_out(p):
        for w in p["wave"][tile:tile + WAVES]:
            w[7] += 64

    for wrong in (twice, shared_slot, part_left_out, part_too_many, column_left_out, keys_left_out):
        plan = copy.deepcopy(good)
        wrong(plan)
        assert plan != good
        with pytest.raises(AssertionError):
            check(plan, shape, reqs)
