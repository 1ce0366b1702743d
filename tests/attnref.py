"""Windowed paged attention in 64 bits, and inputs whose every invisible slot is NaN.

Tolerance of an attention output o = sum_j p_j v_j computed from bf16 q, K and V:
each probability is rounded to bf16 before it meets V (half a step: 2^-8 of it,
so at most 2^-8 sum p|v|), the result is rounded to bf16 (2^-8 |o|), and the fp32
scores, exponentials and sums add at most 2^-12 of either: a score of n products
is off by n 2^-24 sum |q k| / sqrt(n), 6e-5 for n = 128 normal values, the weight
2^x by as much again, and the running sums of at most 2^12 weights per lane, each
2^-24 of the sum, by 2^-12 at the very most."""
import numpy as np

OUT_REL, FP32_REL = 2.0 ** -8, 2.0 ** -12


def visible_ranges(c, x, window, sinks):
    """Keys that some row of a request sees, as one or two ranges."""
    first = max(0, x - window + 1) if window else 0
    s = min(sinks, first) if window else 0
    return ([(0, s)] if s else []) + [(first, x + c)]


def reference(q, k, v, pos, window, sinks):
    """q [rows][nq][hd] at positions pos, k and v [keys][nkv][hd] of one request, fp64; keys no row sees may be
    NaN. Returns o and sum p|v|, [rows][nq][hd]."""
    rows, nq, hd = q.shape
    group = nq // k.shape[1]
    j, p = np.arange(k.shape[0])[None, :], np.asarray(pos)[:, None]
    see = j <= p
    if window:
        see &= (j > p - window) | (j < sinks)
    keys = see.any(0)
    k, v, see = np.repeat(k[keys], group, 1), np.repeat(v[keys], group, 1), see[:, keys]
    assert np.isfinite(k).all() and np.isfinite(v).all()
    s = np.einsum("rhd,jhd->hrj", q, k, optimize=True) / np.sqrt(hd)
    s = np.where(see[None], s, -np.inf)
    e = np.exp(s - s.max(-1, keepdims=True))
    w = e / e.sum(-1, keepdims=True)
    return (np.einsum("hrj,jhd->rhd", w, v, optimize=True), np.einsum("hrj,jhd->rhd", w, np.abs(v), optimize=True))


def assert_close(got, o, pv, what):
    assert np.isfinite(got).all(), f"{what}: not finite"
    bound = (OUT_REL + FP32_REL) * (pv + np.abs(o))
    worst = np.max(np.abs(got - o) / bound)
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound"
    return worst


class Cache:
    """A pool on the GPU, NaN everywhere, and the logical K and V of the requests put into it."""

    def __init__(self, shape, num_blocks, max_tokens=4096, max_requests=64, seed=0):
        from paper_2503_22562_amd.harness import DeviceLayer
        from hb_workloads import make_weights
        self.dl = DeviceLayer(shape, make_weights(shape), num_blocks, max_tokens, max_requests)
        self.shape, self.num_blocks = shape, num_blocks
        self.rng = np.random.default_rng(seed)
        self.perm = self.rng.permutation(num_blocks).astype(np.int32)
        self.used = 0

    def bits(self, *shape):
        from hb_workloads import f32_to_bf16_bits
        return f32_to_bf16_bits(self.rng.standard_normal(shape, dtype=np.float32))

    def request(self, c, x, window, sinks, dead_id=-1):
        """Write the keys that a request's rows see. Returns ((c, x, table), k, v), k and v fp64 with NaN elsewhere."""
        from hb_workloads import bf16_bits_to_f32
        from paper_2503_22562_amd import hb
        n = x + c
        nb = -(-n // 16)
        table = self.perm[self.used:self.used + nb].copy()
        assert len(table) == nb, "the test's pool is too small"
        first, count = hb.hb_window_dead_blocks(x, window, sinks)
        self.used += nb
        k, v = (np.full((n, self.shape.n_kv_heads, self.shape.head_dim), np.nan) for _ in range(2))
        for a, b in visible_ranges(c, x, window, sinks):
            kb, vb = (self.bits(b - a, self.shape.n_kv_heads, self.shape.head_dim) for _ in range(2))
            self.dl.append_kv(table, a, kb, vb)
            k[a:b], v[a:b] = bf16_bits_to_f32(kb), bf16_bits_to_f32(vb)
        table[first:first + count] = dead_id
        return (c, x, table), k, v
