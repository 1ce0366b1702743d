"""Plans of batches whose requests share prefixes (hb_plan.cpp, no HIP): every row of
every kv head meets each of its keys exactly once, through block ids looked up as the
kernels do; every partial result is written once and joined once; what is refused;
and the units by which a batch's new tokens are appended."""
import os
import subprocess
import sys
from collections import Counter, defaultdict

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_22562_amd", "csrc")
sys.path.insert(0, ROOT)

OK, INVALID, RANGE = 0, 1, 2


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "shared_driver")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    f"-I{CSRC}", f"-I{os.path.join(ROOT, 'include')}", os.path.join(ROOT, "tests", "shared_driver.cpp"),
                    os.path.join(CSRC, "hb_plan.cpp"), "-o", exe], check=True)
    return exe


def run(exe, heads, reqs, groups, cu=256, split_tile=0, split_item=0, check=0, share_all=1):
    """reqs: (chunk, context, table)."""
    lines = [" ".join(map(str, (*heads, cu, split_tile, split_item, share_all, check, len(reqs), len(groups))))]
    lines += [f"{c} {x} {len(t)} " + " ".join(map(str, t)) for c, x, t in reqs]
    lines += [" ".join(map(str, g)) for g in groups]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0")
    env.pop("LD_PRELOAD", None)
    out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, env=env)
    assert out.returncode == 0, out.stderr[-2000:]
    plan = defaultdict(list)
    for ln in out.stdout.splitlines():
        k, *v = ln.split()
        assert "differs" not in v, ln
        plan[k].append([int(x) for x in v])
    return plan


def batch(lens, groups):
    """Tables over ids of their own, but for the shared prefixes."""
    shared = {}
    nxt = 0
    for first, count, p in groups:
        for r in range(first, first + count):
            shared[r] = list(range(nxt, nxt + p // 16))
        nxt += p // 16
    reqs = []
    for r, (c, x) in enumerate(lens):
        t = list(shared.get(r, []))
        n = -(-(c + x) // 16) - len(t)
        reqs.append((c, x, t + list(range(nxt, nxt + n))))
        nxt += n
    return reqs


def check(plan, heads, reqs):
    nq, nkv, _ = heads
    G = nq // nkv
    tile_cols, n_slots, _ = plan["geom"][0]
    rows = [(r, x + i) for r, (c, x, _) in enumerate(reqs) for i in range(c)]
    seen = defaultdict(Counter)  # (row, kv head) -> keys, as (block, slot)
    parts = {}                   # column slot -> what it holds: (row, head), the keys' first and number
    direct = Counter()           # (row, kv head) written by its unit
    waves = plan["wave"]
    assert len(waves) % 4 == 0
    for u in range(0, len(waves), 4):
        kind = waves[u][0]
        assert all(w[0] == kind for w in waves[u:u + 4])
        if kind == 0:
            assert all(w[1:] == waves[u][1:] for w in waves[u:u + 4])
        units = waves[u:u + 1] if kind == 0 else waves[u:u + 4]
        stored = False
        for _, g, tok0, pos0, npos, b, e, part, *ids in units:
            if b >= e:
                continue
            assert npos * G <= (tile_cols if kind == 0 else 16) and b % 16 == 0
            for i in range(npos):
                r, pos = rows[tok0 + i]
                keys = range(b, min(e, pos0 + i + 1))
                seen[tok0 + i, g].update((ids[j // 16 - b // 16], j % 16) for j in keys)
            if kind == 2 and stored:  # a merged unit stores once
                continue
            stored = True
            for i in range(npos):
                if part < 0:
                    direct[tok0 + i, g] += 1
                    continue
                for h in range(G):
                    slot = part + i * G + h
                    assert 0 <= slot < n_slots and slot not in parts
                    parts[slot] = (tok0 + i, g, h)
    joined = Counter()
    for part0, nparts, stride, tok0, npos, g, cb in plan["merge"]:
        for c in range(16 * cb, min(16 * cb + 16, npos * G)):
            for s in range(nparts):
                assert parts.pop(part0 + s * stride + c) == (tok0 + c // G, g, c % G)
            joined[tok0 + c // G, g] += 1
    assert not parts
    for t, (r, pos) in enumerate(rows):
        table = reqs[r][2]
        want = Counter((table[j // 16], j % 16) for j in range(pos + 1))
        for g in range(nkv):
            assert seen[t, g] == want, (t, g)
            assert (direct[t, g], joined[t, g]) in ((1, 0), (0, G)), (t, g)


def check_append(plan, reqs):
    want = [(x + i, t[(x + i) // 16]) for c, x, t in reqs for i in range(c)]
    got = []
    for tok0, pos0, n, block in plan["append"]:
        assert n > 0 and pos0 // 16 == (pos0 + n - 1) // 16 and tok0 == len(got)
        got += [(pos0 + i, block) for i in range(n)]
    assert got == want


HEADS = [(4, 2, 64), (8, 2, 128), (16, 1, 64), (3, 3, 128)]
CASES = [
    ([(1, 40), (1, 33)], [(0, 2, 32)]),
    ([(1, 32), (1, 32), (1, 32)], [(0, 3, 32)]),                      # nothing but the new token of their own
    ([(1, 700 + 13 * i) for i in range(20)], [(0, 20, 688)]),
    ([(1, 700 + 13 * i) for i in range(20)], [(3, 9, 640), (12, 5, 16)]),
    ([(1, 5), (2, 3000), (1, 2100), (4, 2100), (1, 9)], [(1, 3, 2096)]),  # drafts of several tokens
    ([(1, 500), (90, 500), (1, 600), (1, 480), (70, 480)], [(0, 5, 480)]),  # chunks that fill tiles between decodes
    ([(1, 1000), (90, 500), (1, 600)], [(0, 3, 480)]),                # a run of one is none
    ([(1, 500)] * 70, [(0, 40, 496), (40, 30, 16)]),                  # more rows than a tile has columns
    ([(1, 9000)] + [(1, 2050)] * 33, [(0, 34, 2048)]),                # one long conversation among short ones
    ([(1, 40), (1, 40)], [(0, 2, 0)]),
    ([(1, 40), (1, 40)], [(0, 1, 32), (1, 1, 32)]),
    ([(1, 40), (1, 40)], []),
]


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("i", range(len(CASES)))
@pytest.mark.parametrize("cu,split_tile,split_item", [(256, 0, 0), (8, 0, 0), (256, 128, 64), (256, 1024, 256)])
def test_every_key_once(driver, heads, i, cu, split_tile, split_item):
    lens, groups = CASES[i]
    reqs = batch(lens, groups)
    for share_all in (1, 0):
        plan = run(driver, heads, reqs, groups, cu, split_tile, split_item, share_all=share_all)
        assert plan["status"] == [[OK]]
        check(plan, heads, reqs)
        check_append(plan, reqs)


@pytest.mark.parametrize("seed", range(30))
def test_random_batches(driver, seed):
    rng = np.random.default_rng(seed)
    lens, groups = [], []
    for _ in range(rng.integers(1, 4)):
        for _ in range(rng.integers(0, 3)):
            lens.append((int(rng.integers(1, 40)), int(rng.integers(0, 900))))
        p, n = 16 * int(rng.integers(0, 90)), int(rng.integers(1, 30))
        groups.append((len(lens), n, p))
        lens += [(int(rng.choice([1, 1, 1, 2, 7, 33])), p + int(rng.integers(0, 400))) for _ in range(n)]
    heads = HEADS[seed % len(HEADS)]
    reqs = batch(lens, groups)
    plan = run(driver, heads, reqs, groups, int(rng.choice([256, 64, 5])))
    check(plan, heads, reqs)
    check_append(plan, reqs)


def test_prefixes_that_are_read_once(driver):
    """64 decodes behind 4096 shared tokens: a unit's 16 columns hold four of them, which read the prefix once."""
    groups = [(0, 64, 4096)]
    reqs = batch([(1, 4096 + 50)] * 64, groups)
    plan = run(driver, (8, 2, 128), reqs, groups)
    read = 0
    for u in range(0, len(plan["wave"]), 4):
        units = plan["wave"][u:u + 1] if plan["wave"][u][0] == 0 else plan["wave"][u:u + 4]
        read += sum(max(0, w[6] - w[5]) for w in units)
    assert read == 2 * (64 // 4 * 4096 + 64 * 51)  # per kv head, and each request's own


@pytest.mark.parametrize("n,prefix,nkv,joined", [(2, 1008, 8, False), (2, 1024, 8, True), (64, 512, 8, False), (64, 512, 16, True),
                                                 (90, 512, 8, False), (93, 512, 8, True)])
def test_prefixes_that_are_too_short(driver, n, prefix, nkv, joined):
    """192 MB of K and V saved, or 1024 keys."""
    groups = [(0, n, prefix)]
    reqs = batch([(1, prefix + 20)] * n, groups)
    plan = run(driver, (nkv, nkv, 128), reqs, groups, share_all=0)
    seen = any(w[4] > 1 for w in plan["wave"])  # units whose rows are several requests'
    assert seen == joined
    check(plan, (nkv, nkv, 128), reqs)


@pytest.mark.parametrize("heads,n,prefix,own,pieces", [((32, 8, 128), 64, 8192, 31, 16), ((32, 8, 128), 256, 16384, 500, 4),
                                                       ((32, 8, 128), 64, 8192, 1000, 6), ((64, 8, 128), 64, 8192, 31, 8),
                                                       ((8, 1, 128), 256, 8192, 450, 16), ((16, 4, 64), 300, 4096, 20, 6)])
def test_pieces_of_a_prefix(driver, heads, n, prefix, own, pieces):
    """Even pieces of a prefix's tiles, and the tiles of one piece on one of the eight dies (workgroup index modulo 8)."""
    groups = [(0, n, prefix)]
    reqs = batch([(1, prefix + own)] * n, groups)
    plan = run(driver, heads, reqs, groups, share_all=0)
    tiles = defaultdict(set)
    for u in range(0, len(plan["wave"]), 4):
        kind, g, tok0, pos0, npos, b, e, part = plan["wave"][u][:8]
        if kind == 0:
            tiles[g, b, e].add((tok0, u // 4 % 8))
    assert len({(b, e) for _, b, e in tiles}) == pieces
    assert max(e - b for _, b, e in tiles) - min(e - b for _, b, e in tiles) < 64 * pieces
    rows = {t for t, _ in next(iter(tiles.values()))}
    for key, at in tiles.items():
        assert {t for t, _ in at} == rows
    spread = [len({die for _, die in at}) for at in tiles.values()]
    assert sum(spread) <= len(spread) + 8  # a die's last places may have to take a part of one more


def tiles_in_order(plan, heads, reqs):
    """(place, kv head, first key, keys, rows, whether it is a shared prefix's) of each tile."""
    request_of = [r for r, (c, _, _) in enumerate(reqs) for _ in range(c)]
    out = []
    for u in range(0, len(plan["wave"]), 4):
        kind, g, tok0, _, npos, b, e, _ = plan["wave"][u][:8]
        if kind == 0:
            c = reqs[request_of[tok0]][0]
            out.append((u // 4, g, b, e - b, npos, c * heads[0] // heads[1] < 64))  # (such requests fill no tile alone)
    return out


@pytest.mark.parametrize("lens,groups", [([(1, 8242)] * 64 + [(2048, 0)], [(0, 64, 8192)]),
                                         ([(1, 4146)] * 64 + [(2048, 0)], [(0, 64, 4096)]),
                                         ([(1, 8242)] * 64 + [(777, 5234)], [(0, 64, 8192)]),
                                         ([(1500, 300)] + [(1, 2098)] * 32 + [(777, 0), (900, 2000)], [(1, 32, 2048)])])
def test_chunks_beside_a_prefix(driver, lens, groups):
    """Tiles are handed out the longest first, a prefix's pieces too: none of the longest stands behind a shorter one of
    a chunk."""
    heads = (32, 8, 128)
    reqs = batch(lens, groups)
    plan = run(driver, heads, reqs, groups, share_all=0)
    check(plan, heads, reqs)
    tiles = tiles_in_order(plan, heads, reqs)
    assert any(t[5] for t in tiles) and any(not t[5] for t in tiles)
    own = [keys * rows for _, _, _, keys, rows, shared in tiles if not shared]
    assert own == sorted(own, reverse=True)
    longest = max(keys * rows for _, _, _, keys, rows, _ in tiles)
    last = max(i for i, t in enumerate(tiles) if t[3] * t[4] == longest)
    first = min(i for i, t in enumerate(tiles) if t[3] * t[4] < longest and not t[5])
    assert last < first


@pytest.mark.parametrize("sizes", [[(112, 12704), (17, 2224), (148, 2272), (50, 6416)], [(95, 5392), (96, 1056), (33, 4768)],
                                   [(141, 2448), (23, 4704)], [(107, 5104), (90, 1136), (21, 4704)]])
def test_prefixes_of_different_lengths(driver, sizes):
    """A die's tiles stand the longest first, however many rows read a prefix."""
    heads = (32, 8, 128)
    lens, groups = [], []
    for n, p in sizes:
        groups.append((len(lens), n, p))
        lens += [(1, p + 20)] * n
    lens.append((1000, 500))
    reqs = batch(lens, groups)
    plan = run(driver, heads, reqs, groups, share_all=0)
    check(plan, heads, reqs)
    ranges = defaultdict(list)  # key range -> (place, keys, rows) of the tiles that read it
    member = [i for i, (n, _) in enumerate(sizes) for _ in range(n)]
    for u in range(0, len(plan["wave"]), 4):
        kind, g, tok0, _, npos, b, e, _ = plan["wave"][u][:8]
        if kind == 0 and tok0 < len(member):
            ranges[member[tok0], g, b].append((u // 4, e - b, npos))
    for die in range(8):
        size = {}
        for tiles in ranges.values():
            for place, _, _ in tiles:
                if place % 8 == die:
                    size[place] = max(keys * rows for _, keys, rows in tiles)
        order = [size[place] for place in sorted(size)]
        assert order == sorted(order, reverse=True)


def test_refusals(driver):
    heads, lens = (4, 2, 64), [(1, 40), (1, 50), (1, 60)]
    good = [(0, 2, 32)]
    reqs = batch(lens, good)

    def status(groups, reqs=reqs):
        return run(driver, heads, reqs, groups, check=1)["status"][0][0]

    assert status(good) == OK and status([]) == OK and status([(0, 1, 32)]) == OK and status([(0, 2, 0)]) == OK
    assert status([(0, 1, 16), (1, 2, 0)]) == OK
    for bad in [(0, 2, 33), (0, 2, -16), (0, 2, 48), (0, 3, 32), (0, 4, 32), (-1, 2, 32), (0, 0, 32), (0, -1, 32),
                (2, 2, 16), (3, 1, 16), (2147483647, 2, 16), (0, 2147483647, 16)]:
        assert status([bad]) == INVALID, bad
    assert status([(0, 2, 32), (1, 2, 0)]) == INVALID and status([(1, 1, 32), (0, 1, 32)]) == INVALID
    # ids outside the pool: the first request's prefix, and what is a request's own
    for r, i in ((0, 0), (0, 1), (0, 2), (1, 3)):
        t = [list(q[2]) for q in reqs]
        t[r][i] = 1 << 20
        if i < 2:
            t[1][i] = 1 << 20
        assert status(good, [(c, x, tt) for (c, x, _), tt in zip(reqs, t)]) == RANGE, (r, i)
    # one that only differs
    t = [list(q[2]) for q in reqs]
    t[1][1] = 900
    assert status(good, [(c, x, tt) for (c, x, _), tt in zip(reqs, t)]) == INVALID
    # what hb_plan_attention refuses
    assert status(good, [(0, 40, reqs[0][2]), *reqs[1:]]) == INVALID
    assert status(good, [(1, 48, reqs[0][2]), *reqs[1:]]) == INVALID
