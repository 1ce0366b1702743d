"""Sliding windows in the host planner (hb_plan.cpp, no HIP): every row of every
kv head meets each key it may see in exactly one work unit and no key besides,
through block ids looked up as the kernels do, with the entries of dead blocks
replaced by -1 in the caller's tables; the windowed work accounting; the rule of
dead blocks; compaction of block tables."""
import os
import subprocess
import sys
from collections import defaultdict

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_22562_amd", "csrc")
sys.path.insert(0, ROOT)


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "window_driver")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    f"-I{CSRC}", f"-I{os.path.join(ROOT, 'include')}", os.path.join(ROOT, "tests", "window_driver.cpp"),
                    os.path.join(CSRC, "hb_plan.cpp"), "-o", exe], check=True)
    return exe


def dead(window, sinks, pos):
    """The rule, key by key: blocks that no row at a position >= pos sees."""
    if not window:
        return []
    return [b for b in range(pos // 16 + 1)
            if all(j >= sinks and j <= pos - window for j in range(16 * b, 16 * b + 16))]


def run(exe, shape, cu, reqs, window, sinks, split_tile=0, split_item=0, dead_id=-1):
    H, nq, nkv, hd, F = shape
    lines = [f"{H} {nq} {nkv} {hd} {F} {cu} {len(reqs)} {window} {sinks} {split_tile} {split_item}"]
    nxt, where = 0, {}
    for r, (c, x) in enumerate(reqs):
        ids = []
        gone = set(dead(window, sinks, x))
        for b in range(-(-(c + x) // 16)):
            ids.append(dead_id if b in gone else nxt)
            where[nxt] = (r, b)
            nxt += 1
        lines.append(f"{c} {x} {len(ids)} " + " ".join(map(str, ids)))
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0")
    env.pop("LD_PRELOAD", None)
    out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, env=env)
    assert out.returncode == 0, out.stderr[-2000:]
    plan = defaultdict(list)
    for ln in out.stdout.splitlines():
        k, *v = ln.split()
        plan[k].append(v)
    return plan, where


def visible(window, sinks, p):
    return {j for j in range(p + 1) if not window or j > p - window or j < sinks}


def check(plan, where, shape, reqs, window, sinks):
    H, nq, nkv, hd, F = shape
    G = nq // nkv
    starts = np.concatenate([[0], np.cumsum([c for c, _ in reqs])])
    tile_cols, per_unit, windowed, sink_blocks = (int(v) for v in plan["geom"][0])
    assert windowed == any(window and x + c - window > sinks for c, x in reqs)
    assert all(int(o) % 16 == 0 and int(o) <= int(n) for o, n in plan["off"])
    assert plan["records"] == [["1"]]  # what hb_attention uploads says the same
    seen = defaultdict(list)
    for kind in ("tile", "item"):
        for v in plan[kind]:
            req, g, tok0, pos0, npos, kb, ke, part = (int(t) for t in v[:8])
            if kb == ke:
                continue
            ids = [int(t) for t in v[8:]]  # raises on an id outside the uploaded table
            assert kb % 64 == 0 and kb < ke and npos * G <= (tile_cols if kind == "tile" else 16)
            for i in range(npos):
                pos = pos0 + i  # on the unit's axis
                for j in range(kb, ke):
                    if j > pos or (window and windowed and j <= pos - window and j >= sinks):
                        continue
                    r, b = where[ids[j // 16 - kb // 16]]
                    assert r == req
                    seen[(tok0 + i, g)].append(16 * b + j % 16)
    for r, (c, x) in enumerate(reqs):
        for i in range(c):
            want = visible(window, sinks, x + i)
            for g in range(nkv):
                got = seen[(int(starts[r]) + i, g)]
                assert len(got) == len(want) and set(got) == want, (r, i, g)
        assert where[int(plan["slot"][r][0])] == (r, x // 16)


SHAPES = {"tiny": (256, 4, 2, 64, 688), "g1": (512, 4, 4, 128, 336), "g16": (1024, 16, 1, 64, 512),
          "tp8": (256, 8, 1, 128, 64)}


@pytest.mark.parametrize("name,reqs,window,sinks,splits", [
    ("tiny", [(64, 128)] + [(1, 256)] * 3, 100, 4, (0, 0)),
    ("tiny", [(1, 0), (1, 1), (1, 15), (1, 16), (1, 17), (2, 700)], 1, 0, (0, 0)),
    ("tiny", [(1, 300), (5, 290)], 16, 16, (0, 0)),
    ("tiny", [(1, 300), (5, 290)], 17, 33, (0, 0)),
    ("tiny", [(200, 0)], 64, 0, (0, 0)),             # rows before and behind the window's length in one chunk
    ("tiny", [(200, 0), (300, 1000)], 33, 21, (64, 0)),
    ("g1", [(300, 900), (1, 2000)], 500, 1, (128, 64)),
    ("g16", [(40, 600), (7, 90), (1, 3000)], 250, 47, (64, 64)),
    ("tp8", [(1, 5000)] * 3, 2000, 5, (0, 0)),
    ("tp8", [(33, 1000), (1, 1000)], 1 << 30, 1 << 30, (0, 0)),  # a window that hides nothing
    ("tp8", [(33, 1000), (1, 1000)], 0, 7, (0, 0)),
    ("tp8", [(20, 100)], 50, 60, (0, 0)),            # sinks and window meet
    ("tp8", [(20, 100)], 50, 1 << 30, (0, 0)),       # every key a sink
])
def test_rows_see_exactly_their_keys(driver, name, reqs, window, sinks, splits):
    plan, where = run(driver, SHAPES[name], 64, reqs, window, sinks, *splits)
    assert plan["status"] == [["0"]]
    check(plan, where, SHAPES[name], reqs, window, sinks)


@pytest.mark.parametrize("seed", range(30))
def test_random_windows(driver, seed):
    rng = np.random.default_rng(seed)
    shape = SHAPES[list(SHAPES)[seed % len(SHAPES)]]
    reqs = [(int(rng.choice([1, 1, rng.integers(1, 20), rng.integers(20, 150)])), int(rng.integers(0, 1500)))
            for _ in range(rng.integers(1, 5))]
    window, sinks = int(np.exp(rng.uniform(0, 7))), int(rng.choice([0, 1, 4, rng.integers(0, 80)]))
    plan, where = run(driver, shape, int(rng.choice([1, 16, 256])), reqs, window, sinks,
                      int(rng.choice([0, 64, 256])), int(rng.choice([0, 64, 128])))
    check(plan, where, shape, reqs, window, sinks)


@pytest.mark.parametrize("name,reqs,window,units", [
    ("tp8", [(1, 300)], 0, 1),                  # short ranges: one unit each
    ("g1", [(1, 9000)] * 8, 500, 32),
    ("tp8", [(1, 1000)], 0, 4),                 # longer ones in 64-key pieces a wave
    ("g1", [(1, 3000)] * 8, 0, 8 * 4 * 6),      # as finely as 256 workgroups allow: 128 keys a wave
    ("tp8", [(1, 30000)], 0, 40),               # no finer than sqrt(keys): 192
])
def test_small_launches_fit_one_round(driver, name, reqs, window, units):
    plan, where = run(driver, SHAPES[name], 256, reqs, window, 0)
    assert len(plan["unit"]) == units <= 256
    if max(x for _, x in reqs) < 5000:
        check(plan, where, SHAPES[name], reqs, window, 0)


@pytest.mark.parametrize("name,reqs,window,tiles,units", [
    # 256 item groups of two rows, 256 keys a wave: no tile
    ("tp8", [(512, 500)], 0, 0, 256),
    ("g1", [(512, 4000)], 512, 0, 128),
    # a wave would have more: 32 tiles, 2016 to 2512 keys in pieces of 320
    ("tp8", [(512, 2000)], 0, sum(-(-n // 320) for n in range(2016, 2513, 16)), None),
    ("tp8", [(64, 16000)], 0, 4 * 42, None),  # no finer than 3 sqrt(keys): 384
    ("tp8", [(550, 0)], 0, 0, 96 // 4 + 179),  # 275 groups, two workgroups per CU: 96 of up to 192 keys, a wave each
    ("tp8", [(576, 0)] * 2, 0, 144, 144),      # 576 groups are too many: two half tiles per CU, (256 - 72) 576 keys
    ("tp8", [(576, 1500)] * 2, 1480, 72 * 3, None),  # 1496 to 1511 keys of the window: in three
    ("tp8", [(64, 16000), (1, 100), (1, 100)], 0, 4 * 42, 4 * 42 + 2),  # (items are cut at 64 keys: a unit each)
])
def test_small_launches_with_chunks_fit_one_round(driver, name, reqs, window, tiles, units):
    plan, where = run(driver, SHAPES[name], 256, reqs, window, 0)
    assert len(plan["tile"]) == tiles and len(plan["unit"]) == (units or tiles) <= 256
    if max(x for _, x in reqs) < 5000:
        check(plan, where, SHAPES[name], reqs, window, 0)


def test_entries_of_dead_blocks_are_not_looked_at(driver):
    for dead_id in (-1, 1 << 30, -(1 << 31)):
        plan, where = run(driver, SHAPES["tp8"], 64, [(1, 5000), (40, 4000)], 300, 20, dead_id=dead_id)
        check(plan, where, SHAPES["tp8"], [(1, 5000), (40, 4000)], 300, 20)
    # a live entry is
    exe, H = driver, SHAPES["tp8"]
    lines = f"{H[0]} {H[1]} {H[2]} {H[3]} {H[4]} 64 1 16 0 0 0\n1 40 3 -1 -1 5\n"
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0")
    env.pop("LD_PRELOAD", None)
    out = subprocess.run([exe], input=lines, capture_output=True, text=True, env=env).stdout
    assert out.startswith("status 2"), out  # position 40 sees keys 25..40: block 1 is live


@pytest.mark.parametrize("reqs,window,sinks", [
    ([(1, 5000), (40, 100), (200, 0)], 150, 5), ([(7, 3)], 4, 2), ([(64, 64)], 1, 0), ([(3, 9)], 100, 3)])
def test_work_counts_what_rows_see(driver, reqs, window, sinks):
    H, nq, nkv, hd, F = shape = SHAPES["tiny"]
    base, _ = run(driver, shape, 64, reqs, 0, 0)
    plan, _ = run(driver, shape, 64, reqs, window, sinks)
    pairs = union = 0
    for c, x in reqs:
        rows = [visible(window, sinks, x + i) for i in range(c)]
        pairs += sum(x + i + 1 - len(v) for i, v in enumerate(rows))
        union += x + c - len(set().union(*rows))
    f0, b0 = (float(v) for v in base["work"][0])
    f1, b1 = (float(v) for v in plan["work"][0])
    assert f0 - f1 == 4.0 * nq * hd * pairs and b0 - b1 == 2.0 * nkv * hd * 2 * union


@pytest.fixture(scope="module")
def H():
    from paper_2503_22562_amd import hb
    hb.load()
    return hb


def test_dead_blocks(H):
    for window in (0, 1, 15, 16, 17, 40, 200):
        for sinks in (0, 1, 15, 16, 17, 50):
            for pos in (0, 1, 15, 16, 31, 32, 33, 63, 64, 100, 257):
                first, count = H.hb_window_dead_blocks(pos, window, sinks)
                assert list(range(first, first + count)) == dead(window, sinks, pos), (window, sinks, pos)
    assert H.hb_window_dead_blocks((1 << 31) - 1, 1 << 30, 1 << 30)[1] == 0
    for bad in ((-1, 5, 0), (5, -1, 0), (5, 1, -1), (5, (1 << 30) + 1, 0), (5, 1, (1 << 30) + 1)):
        with pytest.raises(H.HBError) as e:
            H.hb_window_dead_blocks(*bad)
        assert e.value.status == H.HB_ERR_INVALID
    assert H.load().hb_window_dead_blocks(5, 1, 0, None, None) == H.HB_ERR_INVALID


@pytest.mark.parametrize("seed", range(20))
def test_compaction(H, seed):
    rng = np.random.default_rng(seed)
    nb = int(rng.integers(1, 400))
    perm = rng.permutation(nb)
    tables, at = [], 0
    for _ in range(rng.integers(0, 12)):
        n = int(min(rng.integers(0, 30), nb - at))
        t = perm[at:at + n].copy()
        at += n
        if tables and rng.random() < 0.5:  # a shared prefix
            src = tables[rng.integers(len(tables))]
            t = np.concatenate([src[:rng.integers(0, len(src) + 1)], t])
        t[rng.random(len(t)) < 0.1] = -1
        tables.append(t.astype(np.int32))
    given = [t.copy() for t in tables]
    new, src, dst, used = H.hb_plan_compaction(nb, tables)
    assert all(np.array_equal(a, b) for a, b in zip(given, tables))  # the binding works on copies
    named = {int(b) for t in tables for b in t if b >= 0}
    assert used == len(named) and {int(b) for t in new for b in t if b >= 0} <= set(range(used))
    # contents move with the blocks
    pool = np.arange(nb)
    pool[dst] = pool[src]
    for a, b in zip(tables, new):
        assert len(a) == len(b) and np.array_equal(a < 0, b < 0)
        assert np.array_equal(pool[b[b >= 0]], a[a >= 0])
    # moves that hb_copy_blocks takes: ascending, from outside [0, used) to ids nobody names
    assert len(src) == len(dst) == len([b for b in named if b >= used]) <= nb // 2
    assert np.all(np.diff(src) > 0) and np.all(np.diff(dst) > 0)
    assert set(src.tolist()) <= named and not set(dst.tolist()) & named
    again = H.hb_plan_compaction(nb, new)
    assert len(again[1]) == 0 and all(np.array_equal(a, b) for a, b in zip(again[0], new))


def test_compaction_refusals(H):
    import ctypes as C
    for nb, tables, status in ((0, [], "INVALID"), (4, [[0, 4]], "RANGE"), (4, [[-2]], "RANGE")):
        with pytest.raises(H.HBError) as e:
            H.hb_plan_compaction(nb, tables)
        assert e.value.status == getattr(H, "HB_ERR_" + status)
    # a refused call writes nothing; one table named twice is rewritten once
    t = np.array([7, 2, 9], np.int32)
    src, dst = np.full(5, -7, np.int32), np.full(5, -7, np.int32)
    m, u = C.c_int32(-7), C.c_int32(-7)

    def call(nb, lens):
        ptrs = (C.c_void_p * 2)(t.ctypes.data, t.ctypes.data)
        n = np.array(lens, np.int32)
        return H.load().hb_plan_compaction(nb, ptrs, n.ctypes.data_as(C.POINTER(C.c_int32)), 2, src.ctypes.data,
                                           dst.ctypes.data, C.byref(m), C.byref(u))

    assert call(9, [3, 3]) == H.HB_ERR_RANGE and call(10, [3, -1]) == H.HB_ERR_INVALID
    assert t.tolist() == [7, 2, 9] and (src == -7).all() and (dst == -7).all() and m.value == u.value == -7
    assert call(10, [3, 3]) == H.HB_OK and t.tolist() == [0, 2, 1] and (m.value, u.value) == (2, 3)
    lib = H.load()
    assert lib.hb_plan_compaction(4, None, None, 1, src.ctypes.data, dst.ctypes.data, C.byref(m), C.byref(u)) \
        == H.HB_ERR_INVALID
    assert lib.hb_plan_compaction(4, None, None, 0, None, dst.ctypes.data, C.byref(m), C.byref(u)) == H.HB_ERR_INVALID


def test_calls_refused_before_any_device_work(H):
    """Null handles and configurations outside the limits: no HIP call is made, so this runs without a GPU."""
    import ctypes as C
    lib = H.load()

    class Shape:
        hidden, n_q_heads, n_kv_heads, head_dim, ffn_dim = 256, 4, 2, 64, 688
        rope_theta, rms_eps, kv_block = 5e5, 1e-5, 16

    def create(cfg, nb, out=True):
        h = C.c_void_p(7)
        st = lib.hb_create_attention(C.byref(cfg) if cfg is not None else None, nb, None, C.byref(h) if out else None)
        assert not out or h.value is None
        return st

    good = H.make_config(Shape, 16, 4)
    assert create(good, 4, out=False) == H.HB_ERR_INVALID
    assert create(good, 0) == create(good, -1) == create(None, 4) == H.HB_ERR_INVALID
    for field, value, status in (("head_dim", 96, "UNSUPPORTED"), ("kv_block", 32, "UNSUPPORTED"),
                                 ("n_kv_heads", 3, "UNSUPPORTED"), ("hidden", 0, "INVALID")):
        assert create(H.make_config(type("S", (Shape,), {field: value}), 16, 4), 4) == getattr(H, "HB_ERR_" + status)
    lib.hb_destroy_attention(None)
    ids = np.arange(2, dtype=np.int32).tobytes()
    pool = H.hb_kv_pool(0x1000, 0x1000, 4)
    for st in (lib.hb_plan_attention(None, 0, None, 0, 0), lib.hb_run_attention(None, pool, 0x1000, 256, 0x9000, 256),
               lib.hb_copy_blocks(None, ids, ids, 2), lib.hb_copy_model_blocks(None, ids, ids, 2),
               lib.hb_set_attention_window(None, 1, 0)):
        assert st == H.HB_ERR_INVALID
        assert "null" in H.hb_last_error()


def test_arguments_that_do_not_fit_32_bits(H):
    """Values whose low 32 bits would be a valid argument are refused by the binding, not shortened."""
    wide, ids = (1 << 32) + 1, np.arange(2)

    class Handle:
        handle, layer = None, None

    for call in (lambda: H.hb_set_attention_window(Handle, wide), lambda: H.hb_set_attention_window(Handle, 1, wide),
                 lambda: H.hb_window_dead_blocks(wide, 1), lambda: H.hb_window_dead_blocks(1, wide),
                 lambda: H.hb_plan_attention(Handle, [], wide), lambda: H.hb_plan_attention(Handle, [], 1, wide),
                 lambda: H.hb_copy_blocks(Handle, ids + wide, ids), lambda: H.hb_copy_blocks(Handle, ids, ids + 0.5),
                 lambda: H.hb_copy_model_blocks(Handle, ids, ids - wide),
                 lambda: H.hb_plan_compaction(4, [ids + wide])):
        with pytest.raises(ValueError):
            call()
    table = np.array([5, 3], np.int32)
    moved = H.hb_plan_compaction(6, [table, [5, -1]])
    assert [t.tolist() for t in moved[0]] == [[1, 0], [1, -1]] and moved[3] == 2
    assert table.tolist() == [5, 3]  # the caller's table is not rewritten


def test_the_copy_kernel_does_not_spill(tmp_path):
    import re
    import shutil
    from paper_2503_22562_amd import build as B
    if not os.path.exists(B.HIPCC) and shutil.which("hipcc") is None:
        pytest.skip("no hipcc")
    cmd = [B.HIPCC, *B.COMMON, *B.HIP_FLAGS, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-c",
           os.path.join(B.CSRC, "k_blocks.hip"), "-o", str(tmp_path / "k.o")]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    spills = [int(v) for v in re.findall(r"VGPRs Spill: (\d+)", r.stderr)]
    assert spills and not any(spills)
