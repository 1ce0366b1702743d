"""hb_run_append (rotation and append of a planned batch) against fp64, through the C ABI.

Tolerance of a rotated value m (a cos - b sin): rounded to bf16 once, half a step (2^-8 of it). Before that: the angle's
fp64 product and reduction are off by 2^-51 of it, 2^-21 at 2^30 radians (a position times a frequency of at most 1 here);
its fp32 remainder, the series and the products by at most 2^-22 of |a| + |b| together: four roundings of 2^-24. So 2^-20
m (|a| + |b|) covers both. v, and dimensions that are not rotated, are the same bits."""
import math

import numpy as np
import pytest

from attnref import assert_close, reference
from hb_workloads import LayerShape, bf16_bits_to_f32, f32_to_bf16_bits

pytestmark = pytest.mark.gpu


def heads(nq, nkv, hd):
    return LayerShape(f"{nq}q{nkv}kv{hd}", 64, nq, nkv, hd, 16, weight_seed=7)


def rotated(x, pos, inv_freq, interleaved, magnitude):
    """x [T][heads][hd] fp64 -> the result and |a| + |b| of each value's pair (0 where nothing is rotated)."""
    r = 2 * len(inv_freq)
    first = np.arange(0, r, 2) if interleaved else np.arange(r // 2)
    second = first + 1 if interleaved else first + r // 2
    ang = np.asarray(pos, np.float64)[:, None, None] * np.asarray(inv_freq)
    a, b = x[..., first], x[..., second]
    y, size = x.copy(), np.zeros_like(x)
    y[..., first] = magnitude * (a * np.cos(ang) - b * np.sin(ang))
    y[..., second] = magnitude * (b * np.cos(ang) + a * np.sin(ang))
    size[..., first] = size[..., second] = magnitude * (np.abs(a) + np.abs(b))
    return y, size


def within(got, want, size, what):
    worst = np.max(np.abs(got - want) - (2.0 ** -8 * np.abs(want) + 2.0 ** -20 * size))
    assert worst <= 0, f"{what}: {worst} over the bound"


SENTINEL = 0x7FC1  # a NaN that nothing computes


class Batch:
    """Pools of sentinels, tables over a permutation, fused QKV rows, and a planned handle."""

    def __init__(self, H, shape, lens, inv_freq, layout=0, magnitude=1.0, seed=0, window=(0, 0), tables=None, blocks=None):
        import torch
        self.H, self.torch, self.shape, self.lens = H, torch, shape, lens
        self.inv_freq, self.layout, self.magnitude = np.asarray(inv_freq, np.float64), layout, magnitude
        rng = np.random.default_rng(seed)
        n = [-(-(c + x) // 16) for c, x in lens]
        self.blocks = blocks or sum(n) + 3
        if tables is None:
            perm = rng.permutation(self.blocks).astype(np.int32)
            ends = np.cumsum(n)
            tables = [perm[e - m:e].copy() for e, m in zip(ends, n)]
        self.tables = tables
        self.T = sum(c for c, _ in lens)
        nq, nkv, hd = shape.n_q_heads, shape.n_kv_heads, shape.head_dim
        self.bits = f32_to_bf16_bits(rng.standard_normal((self.T, nq + 2 * nkv, hd), dtype=np.float32))
        self.qkv = torch.from_numpy(self.bits.view(np.int16).reshape(self.T, -1)).cuda().view(torch.bfloat16)
        self.k_pool, self.v_pool = (torch.full((self.blocks, nkv, 16, hd), SENTINEL, dtype=torch.int16, device="cuda")
                                    .view(torch.bfloat16) for _ in range(2))
        self.out = torch.full((self.T, nq, hd), float("nan"), dtype=torch.bfloat16, device="cuda")
        cfg = H.make_config(shape, max(1, self.T), max(1, len(lens)))
        self.att = H.hb_create_attention(cfg, self.blocks)
        H.hb_set_attention_rope(self.att, self.inv_freq, layout, magnitude)
        self.requests = [(c, x, t) for (c, x), t in zip(lens, tables)]
        H.hb_plan_attention(self.att, self.requests, *window)

    def slices(self, t=None):
        t = self.qkv if t is None else t
        a = self.shape.n_q_heads * self.shape.head_dim
        b = a + self.shape.n_kv_heads * self.shape.head_dim
        return t[:, :a], t[:, a:b], t[:, b:b + (b - a)]

    def run(self, out=None):
        q, k, v = self.slices()
        self.H.hb_run_append(self.att, q, k, v, self.k_pool, self.v_pool, self.out if out is None else out)
        self.torch.cuda.synchronize()

    def check(self, out=None, what=""):
        from paper_2503_22562_amd.harness import bf16_bits, k_by_slot, v_by_slot
        nq, nkv, hd = self.shape.n_q_heads, self.shape.n_kv_heads, self.shape.head_dim
        pos = np.concatenate([np.arange(x, x + c) for c, x in self.lens])
        page = np.concatenate([np.asarray(t)[np.arange(x, x + c) // 16] for (c, x), t in zip(self.lens, self.tables)])
        x = bf16_bits_to_f32(self.bits).astype(np.float64)
        y, size = rotated(x[:, :nq + nkv], pos, self.inv_freq, self.layout == 1, self.magnitude)
        r = 2 * len(self.inv_freq)
        got = bf16_bits(self.out if out is None else out).reshape(self.T, nq, hd)
        k = k_by_slot(bf16_bits(self.k_pool)).copy()
        v = v_by_slot(bf16_bits(self.v_pool).reshape(self.blocks, nkv, 2, hd, 8)).copy()
        kn, vn = k[page, :, pos % 16], v[page, :, pos % 16]
        within(bf16_bits_to_f32(got).astype(np.float64), y[:, :nq], size[:, :nq], f"{what} q")
        within(bf16_bits_to_f32(kn).astype(np.float64), y[:, nq:], size[:, nq:], f"{what} k")
        assert np.array_equal(vn, self.bits[:, nq + nkv:]), f"{what} v"
        assert np.array_equal(got[..., r:], self.bits[:, :nq, r:]) and np.array_equal(kn[..., r:], self.bits[:, nq:nq + nkv, r:])
        k[page, :, pos % 16] = v[page, :, pos % 16] = SENTINEL
        assert (k == SENTINEL).all() and (v == SENTINEL).all(), f"{what}: slots that are not the new tokens' changed"


HEADS = [(4, 2, 64), (8, 2, 128), (32, 8, 128), (5, 5, 64), (7, 7, 128), (16, 1, 128), (36, 9, 64)]
LENS = [(1, 0), (1, 15), (1, 16), (17, 5), (1, 700), (8, 8), (16, 32), (7, 25), (40, 90), (2, 31)]


@pytest.mark.parametrize("nqkvhd", HEADS, ids=str)
@pytest.mark.parametrize("part", [1, 2, 4, 0])
@pytest.mark.parametrize("layout", [0, 1])
def test_rotated_and_appended(hb, nqkvhd, part, layout):
    f = hb.hb_rope_frequencies(nqkvhd[2] // part if part else 0, 5e5)
    b = Batch(hb, heads(*nqkvhd), LENS, f, layout, seed=part + layout)
    b.run()
    b.check()


@pytest.mark.parametrize("rotary", range(16, 129, 16))
@pytest.mark.parametrize("layout", [0, 1])
def test_every_rotary_dimension(hb, rotary, layout):
    b = Batch(hb, heads(8, 2, 128), [(3, 1000), (19, 44)], hb.hb_rope_frequencies(rotary, 1e4), layout, 1.25, seed=rotary)
    b.run()
    b.check()


@pytest.mark.parametrize("layout", [0, 1])
def test_far_positions_and_scaling(hb, layout):
    """Positions up to 2^30 - 1 (behind a window, so that the table may repeat an id), scaled frequencies, no magnitude."""
    nb = 40
    for x in (131071, (1 << 24) + 5, (1 << 30) - 9):
        table = np.full(-(-(x + 9) // 16), -1, np.int32)
        table[x // 16:] = np.arange(7, 7 + len(table) - x // 16)
        for f in (hb.hb_rope_frequencies(128, 5e5, 8.0, 1.0, 4.0, 8192), hb.hb_rope_frequencies(128, 5e5, 32.0), np.ones(64),
                  np.zeros(64)):
            b = Batch(hb, heads(8, 2, 128), [(9, x)], f, layout, 0.1 * math.log(8.0) + 1, seed=3, window=(1, 0), tables=[table],
                      blocks=nb)
            b.run()
            b.check(what=f"position {x}")


def test_in_place_and_between_rows(hb):
    """Queries rotated where they are, in the fused rows; k, v and what lies behind the rows untouched."""
    import torch
    for lens in (LENS, [(1, 77)]):
        b = Batch(hb, heads(8, 2, 128), lens, hb.hb_rope_frequencies(128, 5e5), seed=5)
        row = b.qkv.shape[1]
        wide = torch.full((b.T + 2, row + 24), 7.0, dtype=torch.bfloat16, device="cuda")
        wide[:b.T, :row] = b.qkv
        q, k, v = b.slices(wide[:b.T])
        before = wide.clone()
        hb.hb_run_append(b.att, q, k, v, b.k_pool, b.v_pool, q)
        torch.cuda.synchronize()
        b.check(q.contiguous())
        a = 8 * 128
        assert torch.equal(wide[b.T:], before[b.T:]) and torch.equal(wide[:, a:], before[:, a:])
        want = b.out.clone()
        hb.hb_run_append(b.att, *b.slices(before[:b.T]), b.k_pool, b.v_pool, want)
        torch.cuda.synchronize()
        assert torch.equal(want.view(b.T, -1), q)


def test_behind_a_window(hb):
    """Pages that the window freed are -1 in the tables."""
    lens = [(1, 3000), (20, 500), (1, 5)]
    n = [-(-(c + x) // 16) for c, x in lens]
    tables, at = [], 0
    for (c, x), m in zip(lens, n):
        t = np.arange(at, at + m, dtype=np.int32)
        at += m
        first, count = hb.hb_window_dead_blocks(x, 100, 4)
        t[first:first + count] = -1
        tables.append(t)
    b = Batch(hb, heads(8, 2, 128), lens, hb.hb_rope_frequencies(64, 5e5), seed=6, window=(100, 4), tables=tables)
    b.run()
    b.check()


def test_plans_in_turn_and_streams(hb):
    """A handle's later plan, another handle on a stream of its own, and a rotation changed between two runs."""
    import torch
    b = Batch(hb, heads(8, 2, 128), [(30, 3), (1, 100)], hb.hb_rope_frequencies(128, 5e5), seed=7)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        c = Batch(hb, heads(4, 2, 64), [(1, 9)] * 30, hb.hb_rope_frequencies(32, 1e4), 1, seed=8)
    torch.cuda.synchronize()
    for _ in range(3):
        q, k, v = c.slices()
        hb.hb_run_append(c.att, q, k, v, c.k_pool, c.v_pool, c.out)  # on its own stream, not the current one
        q, k, v = b.slices()
        hb.hb_run_append(b.att, q, k, v, b.k_pool, b.v_pool, b.out)
    torch.cuda.synchronize()
    b.check()
    c.check()
    b.inv_freq, b.layout, b.magnitude = hb.hb_rope_frequencies(64, 1e4, 2.0), 1, 0.5
    hb.hb_set_attention_rope(b.att, b.inv_freq, 1, 0.5)
    b.run()
    b.check()
    # a batch of other lengths, then none
    d = Batch(hb, b.shape, [(1, 5), (50, 0)], b.inv_freq, seed=9)
    hb.hb_plan_attention(b.att, [])
    with pytest.raises(ValueError):
        b.run()
    none = torch.empty(0, 8 * 128, dtype=torch.bfloat16, device="cuda")
    hb.hb_run_append(b.att, none, none[:, :256], none[:, :256], b.k_pool, b.v_pool, none)
    d.run()
    d.check()


def test_a_plan_that_stands_takes_the_latest_rotation(hb):
    """Only a plan made before the handle's first rotation cannot append."""
    b = Batch(hb, heads(8, 2, 128), [(30, 3), (1, 100)], hb.hb_rope_frequencies(128, 5e5), seed=14)
    for f, layout, magnitude in ((hb.hb_rope_frequencies(64, 1e4), 1, 1.0), (np.zeros(0), 0, 1.0),
                                 (hb.hb_rope_frequencies(128, 5e5, 4.0), 0, 1.5)):
        b.inv_freq, b.layout, b.magnitude = np.asarray(f, np.float64), layout, magnitude
        hb.hb_set_attention_rope(b.att, f, layout, magnitude)
        b.run()
        b.check()
    late = hb.hb_create_attention(b.att.cfg, b.blocks)
    hb.hb_plan_attention(late, b.requests)
    hb.hb_set_attention_rope(late, b.inv_freq)
    with pytest.raises(hb.HBError, match="before the handle's first hb_set_attention_rope"):
        hb.hb_run_append(late, *b.slices(), b.k_pool, b.v_pool, b.out)
    hb.hb_plan_attention(late, b.requests)
    hb.hb_run_append(late, *b.slices(), b.k_pool, b.v_pool, b.out)
    b.magnitude = 1.0
    b.torch.cuda.synchronize()
    b.check()


def test_calls_that_are_refused(hb):
    import torch
    b = Batch(hb, heads(8, 2, 128), [(3, 100), (1, 40)], hb.hb_rope_frequencies(128, 5e5), seed=10)
    q, k, v = b.slices()
    plain = hb.hb_create_attention(b.att.cfg, b.blocks)
    args = (q, k, v, b.k_pool, b.v_pool, b.out)
    for plan in (False, True):  # no plan; one made before the rotation was set
        with pytest.raises((hb.HBError, ValueError)):
            hb.hb_run_append(plain, *args)
        hb.hb_plan_attention(plain, b.requests)
    hb.hb_set_attention_rope(plain, b.inv_freq)
    with pytest.raises(hb.HBError) as e:
        hb.hb_run_append(plain, *args)
    assert e.value.status == hb.HB_ERR_INVALID and "hb_set_attention_rope" in str(e.value)
    # one slot written twice: attention may still read such a batch
    same = [(1, 40, b.tables[1]), (1, 40, b.tables[1])]
    hb.hb_plan_attention(plain, same)
    with pytest.raises(hb.HBError):
        hb.hb_run_append(plain, q[:2], k[:2], v[:2], b.k_pool, b.v_pool, b.out[:2])
    for bad in ((q.float(), *args[1:]), (q[:3], *args[1:]), (q, k[:, :128], *args[2:]), (q.cpu(), *args[1:]),
                (q, k, v, b.k_pool[:-1], *args[4:]), (q, k, v, b.k_pool.float(), *args[4:]),
                (q.t().contiguous().t(), *args[1:])):
        with pytest.raises(ValueError):
            hb.hb_run_append(b.att, *bad)
    for bad in ((*args[:5], k.new_empty(0).set_(k.untyped_storage(), 8, q.shape, q.stride())),
                (q, k, v, b.k_pool, b.k_pool, b.out)):
        with pytest.raises(hb.HBError):
            hb.hb_run_append(b.att, *bad)
    torch.cuda.synchronize()
    assert (b.k_pool.view(torch.int16) == SENTINEL).all() and b.out.isnan().all()
    b.run()
    b.check()


def test_under_graph_capture(hb):
    """Refused (a replay would read what the latest plan uploaded); the capture, the pool and later calls are unharmed."""
    import torch
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b = Batch(hb, heads(8, 2, 128), [(3, 100)], hb.hb_rope_frequencies(128, 5e5), seed=11)
        x = torch.zeros(64, device="cuda")
        side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        x.add_(1.0)
        with pytest.raises(hb.HBError) as e:
            hb.hb_run_append(b.att, *b.slices(), b.k_pool, b.v_pool, b.out)
        assert e.value.status == hb.HB_ERR_HIP
    with torch.cuda.stream(side):
        graph.replay()
        b.run()
    b.check()
    assert (x == 1.0).all()


def test_the_attention_that_follows(hb):
    """Two chunks of one sequence, each appended and attended by one plan: the second reads what the first wrote."""
    import torch
    shape = heads(8, 2, 128)
    f = hb.hb_rope_frequencies(128, 5e5)
    a = Batch(hb, shape, [(70, 0)], f, seed=12, blocks=9, tables=[np.arange(8, 3, -1, dtype=np.int32)])
    a.run()
    b = Batch(hb, shape, [(5, 70)], f, seed=13, blocks=9, tables=[np.arange(8, 3, -1, dtype=np.int32)])
    b.k_pool, b.v_pool = a.k_pool, a.v_pool
    b.run()
    out = torch.empty_like(b.out)
    hb.hb_run_attention(b.att, b.out, b.k_pool, b.v_pool, out)
    torch.cuda.synchronize()
    from paper_2503_22562_amd.harness import bf16_bits, k_by_slot, v_by_slot
    pos = np.arange(75)
    page = b.tables[0][pos // 16]
    k = bf16_bits_to_f32(k_by_slot(bf16_bits(b.k_pool))[page, :, pos % 16]).astype(np.float64)
    v = bf16_bits_to_f32(v_by_slot(bf16_bits(b.v_pool).reshape(9, 2, 2, 128, 8))[page, :, pos % 16]).astype(np.float64)
    q = b.out.float().cpu().numpy().astype(np.float64)
    o, pv = reference(q, k, v, np.arange(70, 75), 0, 0)
    assert_close(out.float().cpu().numpy().astype(np.float64), o, pv, "attention")
