"""hb_run_attention (paged attention on its own, sliding windows with sinks)
against 64-bit attention, through the C ABI. Pools are NaN wherever no row of a
request may look, and table entries of dead blocks are -1."""
import numpy as np
import pytest

from attnref import Cache, assert_close, reference
from hb_workloads import TINY, LayerShape, bf16_bits_to_f32

pytestmark = pytest.mark.gpu


def heads(nq, nkv, hd):
    return LayerShape(f"{nq}q{nkv}kv{hd}", 64, nq, nkv, hd, 16, weight_seed=7)


class Run:
    """One batch: cache, plan, queries; run() returns the fp64 output [T][nq][hd]."""

    def __init__(self, shape, lens, window, sinks, seed=0, cache=None, dead_id=-1):
        import torch
        from paper_2503_22562_amd import hb as H
        from paper_2503_22562_amd.harness import to_device_bf16
        nb = sum(-(-(c + x) // 16) for c, x in lens) + 3
        self.cache = cache or Cache(shape, nb, max(1, sum(c for c, _ in lens)), max(1, len(lens)), seed)
        self.shape, self.window, self.sinks = shape, window, sinks
        made = [self.cache.request(c, x, window, sinks, dead_id) for c, x in lens]
        self.reqs = [m[0] for m in made]
        self.kv = [m[1:] for m in made]
        self.T = sum(c for c, _ in lens)
        self.q_bits = self.cache.bits(self.T, shape.n_q_heads, shape.head_dim)
        self.q = to_device_bf16(self.q_bits)
        self.out = torch.full((self.T, shape.n_q_heads, shape.head_dim), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.att = H.hb_create_attention(self.cache.dl.cfg, self.cache.num_blocks)
        H.hb_plan_attention(self.att, self.reqs, window, sinks)

    def run(self, q=None, out=None):
        import torch
        from paper_2503_22562_amd import hb as H
        dl = self.cache.dl
        out = self.out if out is None else out
        H.hb_run_attention(self.att, self.q if q is None else q, dl.k_pool, dl.v_pool, out)
        torch.cuda.synchronize()
        return out.float().cpu().numpy().astype(np.float64).reshape(self.T, self.shape.n_q_heads, self.shape.head_dim)

    def check(self, got, what=""):
        q = bf16_bits_to_f32(self.q_bits).astype(np.float64)
        at, worst = 0, 0.0
        for (c, x, _), (k, v) in zip(self.reqs, self.kv):
            o, pv = reference(q[at:at + c], k, v, np.arange(x, x + c), self.window, self.sinks)
            worst = max(worst, assert_close(got[at:at + c], o, pv, f"{what} request ({c}, {x})"))
            at += c
        print(f"{what}: {worst:.3f} of the bound")


EDGES = [(1, 0), (1, 1), (1, 15), (1, 16), (1, 31), (1, 32), (1, 33), (1, 700), (2, 0), (17, 100), (5, 411)]


@pytest.mark.parametrize("nq,nkv,hd", [(4, 2, 64), (2, 2, 128), (8, 2, 128), (8, 1, 128), (16, 1, 64), (32, 8, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 4), (16, 0), (16, 16), (17, 33), (32, 1), (100, 21),
                                          (1000, 4), (5, 1000)])
def test_decodes_and_short_chunks(hb, nq, nkv, hd, window, sinks):
    r = Run(heads(nq, nkv, hd), EDGES, window, sinks, seed=nq + window)
    r.check(r.run())


@pytest.mark.parametrize("nq,nkv,hd", [(4, 2, 64), (2, 2, 128), (8, 2, 128), (8, 1, 128), (16, 1, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 2), (31, 0), (64, 64), (200, 5), (257, 300)])
def test_chunks(hb, nq, nkv, hd, window, sinks):
    r = Run(heads(nq, nkv, hd), [(130, 0), (64, 333), (200, 900), (1, 640)], window, sinks, seed=nq + window + 1)
    r.check(r.run())


@pytest.mark.parametrize("nq,nkv,hd", [(4, 2, 64), (2, 2, 128), (8, 2, 128), (8, 1, 128), (16, 1, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 2), (31, 0), (64, 64), (200, 5), (257, 300)])
def test_chunks_as_tiles(hb, monkeypatch, nq, nkv, hd, window, sinks):
    """A forced tile split keeps the planner from cutting these small launches into wave items."""
    monkeypatch.setenv("HB_ATTN_SPLIT_TILE", "4096")
    r = Run(heads(nq, nkv, hd), [(130, 0), (64, 333), (200, 900), (1, 640)], window, sinks, seed=nq + window + 1)
    r.check(r.run())


@pytest.mark.parametrize("lens", [[(64, 9000)], [(16, 7001), (1, 9), (33, 4000)], [(300, 2500), (1, 2500)], [(700, 0)],
                                  [(450, 300), (1, 5)]])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1999, 40)])
def test_chunks_that_leave_compute_units_idle(hb, lens, window, sinks):
    """Tiles and items cut to fill one round of workgroups (of one or two per CU), joined over tens of parts."""
    r = Run(heads(16, 2, 128), lens, window, sinks, seed=31)
    r.check(r.run())


@pytest.mark.parametrize("nq,nkv,hd,lens", [(4, 2, 64, [(800, 0)] * 3), (16, 1, 64, [(600, 0), (1, 77)]),
                                            (8, 8, 128, [(400, 10)] * 3), (32, 8, 128, [(301, 222), (1, 600)])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 3), (450, 70)])
def test_half_tiles(hb, nq, nkv, hd, lens, window, sinks):
    """More wave items than two rounds take, and few enough keys for two half tiles per CU."""
    r = Run(heads(nq, nkv, hd), lens, window, sinks, seed=32)
    r.check(r.run())


@pytest.mark.parametrize("split_tile,split_item", [(64, 64), (128, 64), (512, 256)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (333, 20), (900, 0)])
def test_split_over_the_length(hb, monkeypatch, split_tile, split_item, window, sinks):
    monkeypatch.setenv("HB_ATTN_SPLIT_TILE", str(split_tile))
    monkeypatch.setenv("HB_ATTN_SPLIT_ITEM", str(split_item))
    r = Run(heads(8, 2, 128), [(150, 1200), (1, 2500), (1, 1), (9, 1777)], window, sinks, seed=3)
    r.check(r.run())


def test_long_contexts(hb):
    for window, sinks in ((0, 0), (3000, 4)):
        r = Run(heads(8, 1, 128), [(1, 70001), (1, 12345), (70, 20000)], window, sinks, seed=4)
        r.check(r.run(), f"window {window}")


def test_scores_far_apart(hb):
    """Keys whose scores dominate by far, in the sinks, at the window's far edge and at the row itself."""
    import torch
    shape = heads(8, 2, 128)
    r = Run(shape, [(1, 900), (90, 500)], 300, 4, seed=5)
    q = torch.zeros_like(r.q)
    q[..., 0] = 60.0
    r.q, r.q_bits = q, q.view(torch.int16).cpu().numpy().view(np.uint16)
    r.check(r.run())
    q[..., 0] = -60.0
    r.q_bits = q.view(torch.int16).cpu().numpy().view(np.uint16)
    r.check(r.run())


def test_strided_rows_and_untouched_memory(hb):
    """q as a slice of a fused QKV output, out as a slice of a wider buffer."""
    import torch
    shape = heads(8, 2, 128)
    r = Run(shape, [(70, 100), (1, 300), (3, 40)], 150, 3, seed=6)
    row = 8 * 128
    want = r.run()
    r.check(want)
    fused = torch.randn(r.T, row + 2 * 2 * 128, device="cuda").to(torch.bfloat16)
    fused[:, :row] = r.q.view(r.T, row)
    wide = torch.full((r.T + 2, row + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    got = r.run(fused[:, :row], wide[1:1 + r.T, 8:8 + row])
    assert np.array_equal(got, want)
    keep = torch.ones_like(wide, dtype=torch.bool)
    keep[1:1 + r.T, 8:8 + row] = False
    assert bool((wide[keep] == 7.0).all())


def test_same_bits_as_the_layer(hb, monkeypatch):
    """The layer's attention over the same cache and the layer's own q, with and without a window. (With one split
    length for both: their planners choose it differently, and partial sums then add in another order.)"""
    monkeypatch.setenv("HB_ATTN_SPLIT_ITEM", "256")
    import torch
    from paper_2503_22562_amd import hb as H
    from paper_2503_22562_amd.harness import DeviceLayer
    from hb_workloads import make_weights
    lens = [(64, 128), (1, 256), (1, 1000), (20, 77)]
    rng = np.random.default_rng(8)
    perm = rng.permutation(256).astype(np.int32)
    reqs, at = [], 0
    for c, x in lens:
        n = -(-(c + x) // 16)
        reqs.append((c, x, perm[at:at + n]))
        at += n
    T = sum(c for c, _ in lens)
    dl = DeviceLayer(TINY, make_weights(TINY), 256, T, len(lens))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    for p in (dl.k_pool, dl.v_pool):
        p.normal_(0.0, 1.0, generator=gen)
    x = torch.randn(T, TINY.hidden, device="cuda", generator=gen).to(torch.bfloat16)
    att = H.hb_create_attention(dl.cfg, 256)
    for window, sinks in ((0, 0), (60, 4), (1 << 30, 0)):
        H.hb_set_attention_window(dl.layer, window, sinks)
        dl.run(reqs, x)
        q, want = dl.stage(H.HB_STAGE_Q, T), dl.stage(H.HB_STAGE_ATTN, T)
        out = torch.empty_like(q)
        H.hb_plan_attention(att, reqs, window, sinks)
        H.hb_run_attention(att, q, dl.k_pool, dl.v_pool, out)
        torch.cuda.synchronize()
        assert torch.equal(out, want), (window, sinks)


def test_plans_in_a_row(hb):
    """More plans and runs than there are staging slots, none waited for, on a stream of their own: growing and
    shrinking batches, every run with the plan that stood when it was called."""
    import torch
    from paper_2503_22562_amd import hb as H
    from paper_2503_22562_amd.harness import to_device_bf16
    shape = heads(8, 2, 128)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cache = Cache(shape, 1400, 512, 64, seed=9)
        batches = [[(1, 10)], [(100, 30)] + [(1, 400)] * 9, [(1, 3000)], [(1, 20)] * 40, [(1, 700), (33, 0)]]
        made = [[cache.request(c, x, 200, 4) for c, x in b] for b in batches]
        att = H.hb_create_attention(cache.dl.cfg, 1400)
        qs = [cache.bits(sum(c for c, _ in b), 8, 128) for b in batches]
        qd = [to_device_bf16(q) for q in qs]
        side.synchronize()
        outs = []
        for i in range(12):
            m = made[i % 5]
            H.hb_plan_attention(att, [r for r, _, _ in m], 200, 4)
            out = torch.full_like(qd[i % 5], float("nan"))
            for _ in range(2):
                H.hb_run_attention(att, qd[i % 5], cache.dl.k_pool, cache.dl.v_pool, out)
            outs.append(out)
        side.synchronize()
        for i, out in enumerate(outs):
            got, at = out.float().cpu().numpy().astype(np.float64), 0
            q = bf16_bits_to_f32(qs[i % 5]).astype(np.float64)
            for (c, x, _), k, v in made[i % 5]:
                o, pv = reference(q[at:at + c], k, v, np.arange(x, x + c), 200, 4)
                assert_close(got[at:at + c], o, pv, f"run {i} request ({c}, {x})")
                at += c


def test_two_handles_on_two_streams(hb):
    """Two plans of one cache at once, each on its own stream with its own split buffers; requests that share blocks."""
    import torch
    from paper_2503_22562_amd import hb as H
    from paper_2503_22562_amd.harness import to_device_bf16
    shape = heads(8, 1, 128)
    cache = Cache(shape, 700, 512, 64, seed=13)
    made = [cache.request(1, 9000, 0, 0), cache.request(120, 1500, 0, 0)]
    (_, _, t0), (_, _, t1) = made[0][0], made[1][0]
    # the same blocks under several requests: shorter contexts of the same sequences
    batches = [[(1, 9000, t0), (1, 4000, t0), (1, 0, t1)], [(120, 1500, t1), (3, 700, t1), (2, 8999, t0)]]
    kv = [(made[0][1:], made[0][1:], made[1][1:]), (made[1][1:], made[1][1:], made[0][1:])]
    torch.cuda.synchronize()
    streams, work = [torch.cuda.Stream() for _ in range(2)], []
    for s, b in zip(streams, batches):
        with torch.cuda.stream(s):
            q = cache.bits(sum(r[0] for r in b), 8, 128)
            qd = to_device_bf16(q)
            outs = [torch.full_like(qd, float("nan")) for _ in range(6)]
            att = H.hb_create_attention(cache.dl.cfg, 700)
            H.hb_plan_attention(att, b)
            work.append((att, q, qd, outs))
    torch.cuda.synchronize()
    for i in range(6):
        for att, _, qd, outs in work:
            H.hb_run_attention(att, qd, cache.dl.k_pool, cache.dl.v_pool, outs[i])
    torch.cuda.synchronize()
    for (att, q, _, outs), b, kvs in zip(work, batches, kv):
        assert all(torch.equal(outs[0], o) for o in outs[1:])
        got, at = outs[0].float().cpu().numpy().astype(np.float64), 0
        qf = bf16_bits_to_f32(q).astype(np.float64)
        for (c, x, _), (k, v) in zip(b, kvs):
            o, pv = reference(qf[at:at + c], k[:x + c], v[:x + c], np.arange(x, x + c), 0, 0)
            assert_close(got[at:at + c], o, pv, f"request ({c}, {x})")
            at += c


def test_offsets_past_32_bits(hb):
    """Blocks beyond 2^32 elements (8 GiB) of a pool, read and copied."""
    import torch
    from paper_2503_22562_amd import hb as H
    from paper_2503_22562_amd.harness import to_device_bf16
    shape = heads(32, 8, 128)
    nb = (1 << 32) // (8 * 16 * 128) + 4000
    cache = Cache(heads(32, 8, 128), 64, 80, 8, seed=10)
    (c, x, table), k, v = cache.request(70, 500, 0, 0)
    big = []
    for p in (cache.dl.k_pool, cache.dl.v_pool):
        b = torch.empty((nb, *p.shape[1:]), dtype=torch.bfloat16, device="cuda")
        b[nb - 64:] = p
        big.append(b)
    q = cache.bits(c, 32, 128)
    qd = to_device_bf16(q)
    out = torch.empty_like(qd)
    att = H.hb_create_attention(cache.dl.cfg, nb)
    layer = H.hb_create_layer(cache.dl.cfg, cache.dl.w, big[0], big[1], nb)
    o, pv = reference(bf16_bits_to_f32(q).astype(np.float64), k, v, np.arange(x, x + c), 0, 0)
    far = table + np.int32(nb - 64)
    moved = (nb - 128 + np.arange(len(table))).astype(np.int32)
    for t in (far, moved):
        if t is moved:
            H.hb_copy_blocks(layer, far, moved)
        out.fill_(float("nan"))
        H.hb_plan_attention(att, [(c, x, t)])
        H.hb_run_attention(att, qd, big[0], big[1], out)
        torch.cuda.synchronize()
        assert_close(out.float().cpu().numpy().astype(np.float64), o, pv, "far blocks")


def test_refusals(hb):
    import torch
    from paper_2503_22562_amd import hb as H
    shape = heads(8, 2, 128)
    r = Run(shape, [(5, 100), (1, 3)], 50, 0, seed=11)
    want, dl, lib = r.run(), r.cache.dl, H.load()
    C = __import__("ctypes")
    row = 8 * 128

    def call(pool=None, q=r.q.data_ptr(), qs=row, out=r.out.data_ptr(), os_=row, nb=r.cache.num_blocks, att=r.att):
        p = pool or H.hb_kv_pool(dl.k_pool.data_ptr(), dl.v_pool.data_ptr(), nb)
        return lib.hb_run_attention(att.handle, C.byref(p), C.c_void_p(q), qs, C.c_void_p(out), os_)

    fresh = H.hb_create_attention(dl.cfg, r.cache.num_blocks)
    for bad in (dict(q=0), dict(out=0), dict(qs=row - 8), dict(qs=row + 4), dict(os_=row - 8), dict(os_=row + 1),
                dict(q=r.q.data_ptr() + 2), dict(out=r.out.data_ptr() + 8), dict(nb=r.cache.num_blocks - 1),
                dict(out=r.q.data_ptr()), dict(out=r.q.data_ptr() + (r.T - 1) * row * 2), dict(att=fresh),
                dict(pool=H.hb_kv_pool(0, dl.v_pool.data_ptr(), r.cache.num_blocks)),
                dict(pool=H.hb_kv_pool(dl.k_pool.data_ptr(), dl.v_pool.data_ptr() + 2, r.cache.num_blocks))):
        assert call(**bad) == H.HB_ERR_INVALID, bad
        assert H.hb_last_error()
    t = r.reqs[0][2]
    for bad, status in (([(0, 5, t)], "INVALID"), ([(1, -1, t)], "INVALID"), ([(5, 100, t[:3])], "INVALID"),
                        ([(1, 0, [r.cache.num_blocks])], "RANGE"), ([(1, 30, [-1, 0])], "RANGE"),
                        ([(7, 0, t)], "RANGE"),  # t's first entries are dead: -1
                        ([(7, 0, np.arange(1))], "INVALID"), ([(1, 3, [0])] * 3, "INVALID")):
        with pytest.raises(H.HBError) as e:
            H.hb_plan_attention(r.att, bad, 50, 0)
        assert e.value.status == getattr(H, "HB_ERR_" + status), bad
    for w, s in ((-1, 0), (1, -1), ((1 << 30) + 1, 0)):
        with pytest.raises(H.HBError) as e:
            H.hb_plan_attention(r.att, r.reqs, w, s)
        assert e.value.status == H.HB_ERR_INVALID
    # what was refused left the plan; the binding's own checks
    r.out.fill_(float("nan"))
    assert np.array_equal(r.run(), want)
    for q, out, k in ((r.q[:-1], r.out, dl.k_pool), (r.q.float(), r.out, dl.k_pool), (r.q, r.out.transpose(1, 2), dl.k_pool),
                      (r.q, r.out, dl.k_pool[1:]), (r.q.cpu(), r.out, dl.k_pool), (r.q, r.out, dl.k_pool.float())):
        with pytest.raises(ValueError):
            H.hb_run_attention(r.att, q, k, dl.v_pool, out)
    # an empty batch
    H.hb_plan_attention(r.att, [])
    r.out.fill_(3.0)
    H.hb_run_attention(r.att, r.q[:0], dl.k_pool, dl.v_pool, r.out[:0])
    torch.cuda.synchronize()
    assert bool((r.out == 3.0).all())


def test_refused_under_capture(hb):
    import torch
    from paper_2503_22562_amd import hb as H
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        r = Run(heads(8, 2, 128), [(5, 100), (1, 300)], 50, 0, seed=12)
        want = r.run()
        pools = [p.clone() for p in (r.cache.dl.k_pool, r.cache.dl.v_pool)]
        count = torch.zeros(1, device="cuda")
        side.synchronize()
    graph, status = torch.cuda.CUDAGraph(), []
    with torch.cuda.graph(graph, stream=side):
        count.add_(1)
        for call in (lambda: H.hb_plan_attention(r.att, r.reqs, 50, 0),
                     lambda: H.hb_run_attention(r.att, r.q, r.cache.dl.k_pool, r.cache.dl.v_pool, r.out),
                     lambda: H.hb_copy_blocks(r.cache.dl.layer, [0], [1])):
            try:
                call()
                status.append(0)
            except H.HBError as e:
                status.append(e.status)
    assert status == [H.HB_ERR_HIP] * 3
    with torch.cuda.stream(side):
        for _ in range(3):
            graph.replay()
            r.out.fill_(float("nan"))
            assert np.array_equal(r.run(), want)
        assert count.item() == 3
        assert all(torch.equal(p.view(torch.int16), o.view(torch.int16))
                   for p, o in zip((r.cache.dl.k_pool, r.cache.dl.v_pool), pools))
