"""hb_run_attention where a lost, doubled or stale part of a key range must show: weights that are all equal (the
output counts the keys seen), one key that outweighs all others at the places where visibility changes, and random
inputs under a bound that shrinks with the length."""
import numpy as np
import pytest

from attnref import FP32_REL, OUT_REL, Cache
from hb_workloads import LayerShape, bf16_bits_to_f32, f32_to_bf16_bits

pytestmark = pytest.mark.gpu


def heads(nq, nkv, hd):
    return LayerShape(f"{nq}q{nkv}kv{hd}", 64, nq, nkv, hd, 16, weight_seed=7)


def visible(pos, n, window, sinks):
    """[rows][keys]"""
    j, p = np.arange(n)[None, :], np.asarray(pos)[:, None]
    see = j <= p
    return see & ((j > p - window) | (j < sinks)) if window else see


def run(cache, reqs, q_bits, window, sinks):
    """fp64 [T][nq][hd] of requests (c, x, table) whose keys are all in the cache."""
    import torch
    from paper_2503_22562_amd import hb as H
    from paper_2503_22562_amd.harness import to_device_bf16
    q = to_device_bf16(q_bits)
    out = torch.full_like(q, float("nan"))
    att = H.hb_create_attention(cache.dl.cfg, cache.num_blocks)
    H.hb_plan_attention(att, reqs, window, sinks)
    for _ in range(2):  # the second over the first one's split partials
        H.hb_run_attention(att, q, cache.dl.k_pool, cache.dl.v_pool, out)
    torch.cuda.synchronize()
    return out.float().cpu().numpy().astype(np.float64)


def put(cache, n, k_bits, v_bits):
    table = cache.perm[cache.used:cache.used + -(-n // 16)].copy()
    cache.used += len(table)
    cache.dl.append_kv(table, 0, k_bits, v_bits)
    return table


def make(shape, lens, seed):
    return Cache(shape, sum(-(-(c + x) // 16) for c, x in lens), sum(c for c, _ in lens), len(lens), seed)


LAUNCHES = [
    ((8, 1, 128), [(1, 70001), (1, 12345), (70, 20000)]), ((8, 2, 128), [(1, 3000)] * 3 + [(1, 250)]),
    ((32, 8, 128), [(64, 2000)] + [(1, 3000)] * 4), ((32, 8, 128), [(512, 0)]), ((32, 8, 128), [(128, 1000)]),
    ((4, 2, 64), [(800, 0)] * 3), ((16, 2, 128), [(64, 9000)]), ((16, 2, 128), [(700, 0)]),
    ((8, 1, 128), [(512, 2000)]), ((8, 1, 128), [(64, 16000), (1, 100)]), ((8, 1, 128), [(550, 0)]),
    ((2, 2, 128), [(300, 2500), (1, 2500)]), ((16, 1, 64), [(40, 600), (7, 90), (1, 3000)]),
]


@pytest.mark.parametrize("window,sinks", [(0, 0), (999, 21), (3000, 4)])
@pytest.mark.parametrize("nqkvhd,lens", LAUNCHES, ids=range(len(LAUNCHES)))
def test_every_key_counts_once(hb, nqkvhd, lens, window, sinks):
    """q is zero, so every visible key has the weight 1, exactly, and V of key j is the unit vector j / 64 mod hd: the
    output is the share of the row's keys in those runs of 64. Rounded: the reciprocal of the sum and the product with
    it (2^-20), the output (2^-8). A run of 64 lost or counted twice is more than a tenth of its value."""
    shape = heads(*nqkvhd)
    nq, nkv, hd = nqkvhd
    cache = make(shape, lens, 51)
    reqs, want = [], []
    for c, x in lens:
        n = x + c
        unit = np.zeros((n, hd), np.float32)
        unit[np.arange(n), np.arange(n) // 64 % hd] = 1.0
        v = np.broadcast_to(f32_to_bf16_bits(unit)[:, None, :], (n, nkv, hd))
        reqs.append((c, x, put(cache, n, cache.bits(n, nkv, hd), v.copy())))
        before = np.concatenate([np.zeros((1, hd)), np.cumsum(unit, 0, dtype=np.float64)])  # of the keys below j
        p = np.arange(x, n)
        lo = np.maximum(0, p - window + 1) if window else np.zeros(c, int)
        seen = before[p + 1] - before[lo] + before[np.minimum(lo, sinks)]
        want.append(np.repeat((seen / seen.sum(1, keepdims=True))[:, None, :], nq, 1))
    want = np.concatenate(want)
    got = run(cache, reqs, np.zeros(want.shape, np.uint16), window, sinks)
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= (OUT_REL + 2.0 ** -20) * want).all(), np.abs(got / np.maximum(want, 1e-9) - 1).max()


@pytest.mark.parametrize("place", ["first", "last sink", "behind the sinks", "behind the window", "in the window",
                                   "before itself", "itself"])
@pytest.mark.parametrize("nqkvhd,c,x", [((8, 2, 128), 1, 900), ((8, 2, 128), 90, 500), ((4, 2, 64), 17, 4000),
                                        ((32, 8, 128), 400, 600), ((8, 1, 128), 1, 20000)])
def test_one_key_outweighs_all(hb, nqkvhd, c, x, place):
    """A key whose score is 40 above the others' and whose values are 64 times theirs, where a row in the middle of the
    chunk begins or ceases to see it: rows that see it give its V, the others' outputs know nothing of it."""
    shape, window, sinks = heads(*nqkvhd), 300, 21
    nq, nkv, hd = nqkvhd
    row = x + c // 2
    at = {"first": 0, "last sink": sinks - 1, "behind the sinks": sinks, "behind the window": row - window,
          "in the window": row - window + 1, "before itself": row - 1, "itself": row}[place]
    n = x + c
    cache = make(shape, [(c, x)], 52)
    k, v = (bf16_bits_to_f32(cache.bits(n, nkv, hd)) for _ in range(2))
    q = np.zeros((c, nq, hd), np.float32)
    q[:, :, 0] = 4.0
    k[:, :, 0] = 0.0
    k[at, :, 0] = 10.0 * np.sqrt(hd)
    v[at] *= 64.0
    bits = [f32_to_bf16_bits(a) for a in (k, v, q)]
    k, v, q = (bf16_bits_to_f32(b).astype(np.float64) for b in bits)
    got = run(cache, [(c, x, put(cache, n, bits[0], bits[1]))], bits[2], window, sinks)
    see = visible(np.arange(x, n), n, window, sinks)
    for h in range(nq):
        g = h // (nq // nkv)
        s = np.where(see, q[:, h] @ k[:, g].T / np.sqrt(hd), -np.inf)
        w = np.exp(s - s.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        o, pv = w @ v[:, g], w @ np.abs(v[:, g])
        bound = (OUT_REL + FP32_REL) * (pv + np.abs(o))  # as in attnref: weights and output rounded to bf16
        assert (np.abs(got[:, h] - o) <= bound).all(), (place, h, np.max(np.abs(got[:, h] - o) / bound))


@pytest.mark.parametrize("window,sinks", [(0, 0), (3000, 4)])
@pytest.mark.parametrize("nqkvhd,lens", [((8, 1, 128), [(1, 70001), (1, 12345), (33, 20000)]),
                                         ((16, 2, 128), [(64, 9000), (1, 5000)]), ((4, 2, 64), [(400, 700), (1, 9000)]),
                                         ((32, 8, 128), [(64, 2000)] + [(1, 3000)] * 4)])
def test_random_inputs_under_a_statistical_bound(hb, nqkvhd, lens, window, sinks):
    """The roundings of the weights are independent: each is off by at most 2^-8 of the weight, evenly spread, 2^-8 /
    sqrt(3) in the mean square, so their sum has a standard deviation of 2^-8 / sqrt(3) sqrt(sum p^2 v^2). Seven of
    them, the output's rounding, and 2^-16 sum p|v| for the fp32 arithmetic (scores of 128 products and sums of up to
    2^12 weights in a lane, at random 2^-24 sqrt(128) and 2^-24 sqrt(2^12) = 2^-18 of their size)."""
    shape = heads(*nqkvhd)
    nq, nkv, hd = nqkvhd
    cache = make(shape, lens, 53)
    reqs, kv = [], []
    for c, x in lens:
        kb, vb = (cache.bits(x + c, nkv, hd) for _ in range(2))
        reqs.append((c, x, put(cache, x + c, kb, vb)))
        kv.append([bf16_bits_to_f32(b).astype(np.float64) for b in (kb, vb)])
    q_bits = cache.bits(sum(c for c, _ in lens), nq, hd)
    q = bf16_bits_to_f32(q_bits).astype(np.float64)
    got, at, worst = run(cache, reqs, q_bits, window, sinks), 0, 0.0
    for (c, x), (k, v) in zip(lens, kv):
        see = visible(np.arange(x, x + c), x + c, window, sinks)
        for h in range(nq):
            g = h // (nq // nkv)
            s = np.where(see, q[at:at + c, h] @ k[:, g].T / np.sqrt(hd), -np.inf)
            w = np.exp(s - s.max(1, keepdims=True))
            w /= w.sum(1, keepdims=True)
            o, pv, p2v2 = w @ v[:, g], w @ np.abs(v[:, g]), (w * w) @ (v[:, g] * v[:, g])
            bound = 7 / np.sqrt(3) * OUT_REL * np.sqrt(p2v2) + OUT_REL * np.abs(o) + 2.0 ** -16 * pv
            worst = max(worst, np.max(np.abs(got[at:at + c, h] - o) / bound))
        at += c
    print(f"{worst:.3f} of the bound")
    assert worst <= 1.0
