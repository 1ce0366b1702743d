"""Attention over the paged KV cache and copies of its pages: the calls that a
serving loop makes of them beside the layer, and the same results in plain torch.

A case holds plain values only:
  op        "attention" (hb_run_attention) or "copy" (hb_copy_blocks, or
            hb_copy_model_blocks when layers > 0)
  nq, nkv, hd   query heads, kv heads, head dimension
attention:
  chunks, chunk_lo, chunk_hi, off_lo, off_hi   number of prefill chunks, the
            range of their lengths and of the contexts before them
  decodes, ctx_lo, ctx_hi   number of decodes, the range of their contexts
            (spread over the logarithm)
  mix       seed of the lengths, which thus belong to the case
  window, sinks   a row at position p sees the keys j <= p with j > p - window
            or j < sinks (window 0: all j <= p)
  freed     the pages that the window hides from every row are gone: their
            block-table entries are -1 and the pool has no room for them
copy:
  layers    layers of the model whose pools are copied in (0: one layer alone)
  blocks    pool blocks of a layer
  pairs     blocks copied
  pattern   "fork" (source blocks copied twice each) or
            "compact" (blocks of the pool's upper part moved to free ones below)
"""
import dataclasses
import math
import random

import numpy as np
import torch

own = False

BLOCK = 16


def _attn(name, heads, chunks, decodes, window, sinks, mix, freed=False):
    n, clo, chi, olo, ohi = chunks
    d, lo, hi = decodes
    c = {"op": "attention", "nq": heads[0], "nkv": heads[1], "hd": heads[2], "chunks": n, "chunk_lo": clo,
         "chunk_hi": chi, "off_lo": olo, "off_hi": ohi, "decodes": d, "ctx_lo": lo, "ctx_hi": hi, "window": window,
         "sinks": sinks, "mix": mix, "freed": freed}
    return dict(c, name=name) if name else c


def _copy(name, heads, layers, blocks, pairs, pattern, mix):
    c = {"op": "copy", "nq": heads[0], "nkv": heads[1], "hd": heads[2], "layers": layers, "blocks": blocks,
         "pairs": pairs, "pattern": pattern, "mix": mix}
    return dict(c, name=name) if name else c


# (query heads, kv heads, head dimension) of the shapes in hb_workloads, and of layers without shared heads
TINY, L8B, L70B, L8B_TP2, L70B_TP8 = (4, 2, 64), (32, 8, 128), (64, 8, 128), (16, 4, 128), (8, 1, 128)
MHA64, MHA128, MQA = (12, 12, 64), (16, 16, 128), (16, 1, 128)
NO_CHUNK, NO_DECODE = (0, 0, 0, 0, 0), (0, 0, 0)


def listed():
    return [
        # one user decoding alone behind a sliding window: launch latency and the longest wave's chain of loads
        _attn("dec1-w1024", L8B, NO_CHUNK, (1, 6001, 6001), 1024, 4, 1, True),
        # a lightly loaded tensor-parallel replica: few rows on one kv head, so the cache's length is split
        _attn("tp8-dec8", L70B_TP8, NO_CHUNK, (8, 512, 8192), 0, 0, 2),
        # a decode queue of long conversations, the pages behind their windows freed
        _attn("dec64-w4096-freed", L8B, NO_CHUNK, (64, 512, 32768), 4096, 4, 3, True),
        # the largest decode queue, every cached token visible: the K/V stream
        _attn("dec256", L8B, NO_CHUNK, (256, 256, 8192), 0, 0, 4),
        # a small test model: 64-wide heads, a window shorter than the chunk, odd lengths
        _attn("tiny-chunk77-dec9-w100", TINY, (1, 77, 77, 1000, 1000), (9, 1, 700), 100, 3, 5),
        # the usual hybrid batch (chunk 512 behind 3431 tokens, 64 decodes) under a window
        _attn("chunk512-dec64-w1024", L8B, (1, 512, 512, 3431, 3431), (64, 512, 4096), 1024, 4, 6),
        # the share of one of two GPUs, odd lengths throughout, sinks that end inside a page
        _attn("tp2-chunk777-dec45-w2001", L8B_TP2, (1, 777, 777, 5234, 5234), (45, 300, 6000), 2001, 21, 7),
        # a busy replica's prompts, most of whose keys a short window hides
        _attn("4chunks-w512", L8B, (4, 256, 2048, 0, 8192), NO_DECODE, 512, 16, 8),
        # the largest: long-context prefill of the 70B layer beside a few long decodes
        _attn("70b-chunk2048-dec8", L70B, (1, 2048, 2048, 30720, 30720), (8, 16384, 32768), 0, 0, 9),
        # one forked sequence gets a private copy of its last page, in one layer
        _copy("fork1", L8B, 0, 512, 1, "fork", 10),
        # 48 sequences forked (parallel sampling): their last pages in all 32 layers
        _copy("fork48-32layers", L8B, 32, 512, 48, "fork", 11),
        # a fragmented pool compacted before its upper part is given back
        _copy("compact9000", L8B, 0, 24576, 9000, "compact", 12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


# no drawn case costs more than the largest listed ones: the flops of 70b-chunk2048-dec8, the bytes of dec256
MAX_FLOPS, MAX_BYTES = 2.1e12, 2.5e9


def draw(rng):
    while True:
        if rng.random() < 0.25:
            heads = rng.choice([TINY, L8B, L8B, L70B_TP8, L8B_TP2, MHA64])
            layers = rng.choice([0, 0, rng.randint(1, 32)])
            pairs = _log_int(rng, 1, 8192 if layers == 0 else 64)
            pattern = rng.choice(["fork", "compact"])
            c = _copy("", heads, layers, 2 * pairs + rng.randint(3, 500), pairs, pattern, rng.randrange(1 << 30))
        else:
            heads = rng.choice([TINY, L8B, L8B, L8B, L70B, L8B_TP2, L70B_TP8, MHA64, MHA128, MQA])
            chunks = rng.choice([0, 0, 1, 1, 2, 4])
            hi = _log_int(rng, 1, 2048 // max(1, chunks))
            decodes = _log_int(rng, 1, 256)
            if chunks and rng.random() < 0.3:
                decodes = 0
            window = rng.choice([0, _log_int(rng, 1, 8192), _log_int(rng, 64, 8192)])
            sinks = rng.choice([0, 4, rng.randint(1, 100)]) if window else 0
            off = rng.choice([0, 1000, 8192, 30720])
            c = _attn("", heads, (chunks, max(1, hi // 3) if chunks > 1 else hi, hi, 0, off),
                      (decodes, 1, rng.choice([100, 2000, 8192, 32768])), window, sinks, rng.randrange(1 << 30),
                      bool(window) and rng.random() < 0.5)
        w = work(c)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES and _pool_bytes(c) <= 6e9:
            return c


def _lens(case):
    """(chunk_len, context_len) of each request, chunks first: a function of the case alone."""
    rng = random.Random(case["mix"])
    lens = [(rng.randint(case["chunk_lo"], case["chunk_hi"]), rng.randint(case["off_lo"], case["off_hi"]))
            for _ in range(case["chunks"])]
    return lens + [(1, _log_int(rng, case["ctx_lo"], case["ctx_hi"])) for _ in range(case["decodes"])]


def _seen(c, x, window, sinks):
    """Keys that some row of a request sees, as ranges [a, b), and the sum over its rows of the keys each sees."""
    first = max(0, x - window + 1) if window else 0
    s = min(sinks, first)
    pairs = 0
    for p in (range(x, x + c) if window else ()):
        lo = max(0, p - window + 1)
        pairs += p + 1 - lo + min(sinks, lo)
    if not window:
        pairs = c * x + c * (c + 1) // 2
    return ([(0, s)] if s else []) + [(first, x + c)], pairs


def _dead(c, x, window, sinks):
    """Blocks [a, b) of a request that none of its rows sees."""
    a, b = -(-sinks // BLOCK), max(0, x - window + 1) // BLOCK
    return (a, b) if window and b > a else (0, 0)


def _pool_bytes(case):
    tok = 4 * case["nkv"] * case["hd"]
    if case["op"] == "copy":
        return max(1, case["layers"]) * case["blocks"] * BLOCK * tok
    return sum(x + c for c, x in _lens(case)) * tok


def _normal(gen, shape, std=1.0):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=gen)


def _sources(case):
    """Different source blocks of a copy."""
    return -(-case["pairs"] // 2) if case["pattern"] == "fork" else case["pairs"]


def _pairs(case, perm):
    """Source and destination blocks of a copy, no destination among the sources."""
    n, nb = case["pairs"], case["blocks"]
    if case["pattern"] == "fork":
        ids = perm.permutation(nb).astype(np.int32)
        return ids[np.arange(n) % _sources(case)], ids[nb - n:].copy()
    # the lower half holds the free blocks, the upper half the blocks that move down, both ascending
    half = nb // 2
    dst = np.sort(perm.permutation(half)[:n]).astype(np.int32)
    src = np.sort(half + perm.permutation(nb - half)[:n]).astype(np.int32)
    return src, dst


def _inputs(case, seed):
    """Everything that a case's call reads, from the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    perm = np.random.default_rng(seed)
    nq, nkv, hd = case["nq"], case["nkv"], case["hd"]

    def pool(blocks):  # in the layouts of include/hb.h: K [2][hd/8][8][8], V [2][hd][8] per block and kv head
        return _normal(gen, (blocks, nkv, 16, hd)), _normal(gen, (blocks, nkv, 16, hd))

    if case["op"] == "copy":
        src, dst = _pairs(case, perm)
        return {"pools": [pool(case["blocks"]) for _ in range(max(1, case["layers"]))], "src": src, "dst": dst}
    lens = _lens(case)
    tables, used = [], 0
    for c, x in lens:
        n = -(-(c + x) // BLOCK)
        a, b = _dead(c, x, case["window"], case["sinks"]) if case["freed"] else (0, 0)
        t = np.arange(used, used + n, dtype=np.int32)
        t[b:] -= b - a
        t[a:b] = -1
        used += n - (b - a)
        tables.append(t)
    blocks = used + 16
    ids = perm.permutation(blocks).astype(np.int32)
    tables = [np.where(t >= 0, ids[t], -1).astype(np.int32) for t in tables]
    return {"requests": [(c, x, t) for (c, x), t in zip(lens, tables)], "blocks": blocks, "pools": [pool(blocks)],
            "q": _normal(gen, (sum(c for c, _ in lens), nq, hd))}


def _narrow(case, max_tokens, max_requests):
    """A layer configuration with the case's heads and no more of the rest than it must have."""
    from hb_workloads import LLAMA3_8B
    from paper_2503_22562_amd import hb
    s = dataclasses.replace(LLAMA3_8B, name="heads", hidden=64, n_q_heads=case["nq"], n_kv_heads=case["nkv"],
                            head_dim=case["hd"], ffn_dim=16)
    return s, hb.make_config(s, max_tokens, max_requests)


def _weights(s):
    z = dict(dtype=torch.bfloat16, device="cuda")
    qd = s.n_q_heads * s.head_dim
    return {"w_qkv": torch.zeros(s.qkv_dim, s.hidden, **z), "w_o": torch.zeros(s.hidden, qd, **z),
            "w_gate_up": torch.zeros(2 * s.ffn_dim, s.hidden, **z), "w_down": torch.zeros(s.hidden, s.ffn_dim, **z),
            "g_attn": torch.ones(s.hidden, **z), "g_ffn": torch.ones(s.hidden, **z)}


def prepare(case, seed):
    st = dict(_inputs(case, seed), case=case)
    if case["op"] == "attention":
        st["out"] = torch.empty_like(st["q"])
    if not own:
        # the plain forms look block ids up on the GPU
        if case["op"] == "copy":
            st["src_t"], st["dst_t"] = (torch.from_numpy(st[n]).long().cuda() for n in ("src", "dst"))
        else:
            st["tables"] = [torch.from_numpy(t).long().cuda() for _, _, t in st["requests"]]
        return st
    from paper_2503_22562_amd import hb
    if case["op"] == "attention":
        # one plan serves every layer of an iteration
        _, cfg = _narrow(case, max(1, st["q"].shape[0]), len(st["requests"]))
        st["attention"] = hb.hb_create_attention(cfg, st["blocks"])
        hb.hb_plan_attention(st["attention"], st["requests"], case["window"], case["sinks"])
        return st
    s, cfg = _narrow(case, 64, 8)
    if case["layers"]:
        z = torch.zeros(8, s.hidden, dtype=torch.bfloat16, device="cuda")
        st["model"] = hb.hb_create_model(cfg, [_weights(s)] * case["layers"], st["pools"], case["blocks"], z,
                                         torch.ones(s.hidden, dtype=torch.bfloat16, device="cuda"), z)
    else:
        (k, v), = st["pools"]
        st["layer"] = hb.hb_create_layer(cfg, _weights(s), k, v, case["blocks"])
    return st


def run(state):
    case = state["case"]
    if case["op"] == "copy":
        if not own:
            for pools in state["pools"]:
                for p in pools:
                    p[state["dst_t"]] = p[state["src_t"]]
        else:
            from paper_2503_22562_amd import hb
            if case["layers"]:
                hb.hb_copy_model_blocks(state["model"], state["src"], state["dst"])
            else:
                hb.hb_copy_blocks(state["layer"], state["src"], state["dst"])
        return {"pools": state["pools"]}
    if own:
        from paper_2503_22562_amd import hb
        (k, v), = state["pools"]
        hb.hb_run_attention(state["attention"], state["q"], k, v, state["out"])
        return {"out": state["out"]}
    return {"out": _plain_attention(state, case)}


# --- plain form ----------------------------------------------------------------
def _k_index(hd):
    """Flat positions of K[slot][dim] inside a stored block of one kv head."""
    s, d = torch.meshgrid(torch.arange(16, device="cuda"), torch.arange(hd, device="cuda"), indexing="ij")
    return (((s // 4 % 2) * (hd // 8) + d // 8) * 64 + (4 * (s // 8) + s % 4) * 8 + d % 8).reshape(-1)


def _v_index(hd):
    s, d = torch.meshgrid(torch.arange(16, device="cuda"), torch.arange(hd, device="cuda"), indexing="ij")
    return ((s // 8 * hd + d) * 8 + s % 8).reshape(-1)


def _plain_attention(state, case):
    nq, nkv, hd, window, sinks = (case[n] for n in ("nq", "nkv", "hd", "window", "sinks"))
    (kp, vp), = state["pools"]
    ki, vi = _k_index(hd), _v_index(hd)
    group, at = nq // nkv, 0
    for (c, x, _), table in zip(state["requests"], state["tables"]):
        # the blocks that some row sees
        ranges = [(a // BLOCK, -(-b // BLOCK)) for a, b in _seen(c, x, window, sinks)[0]]
        if len(ranges) == 2 and ranges[0][1] >= ranges[1][0]:
            ranges = [(ranges[0][0], ranges[1][1])]
        blk = torch.cat([torch.arange(a, b, device="cuda") for a, b in ranges])
        j = (blk[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")).reshape(-1)

        def rows(pool, index):  # [n_kv][keys][hd]
            r = pool.view(-1, nkv, 16 * hd)[table[blk]][:, :, index].float()
            return r.view(len(blk), nkv, 16, hd).transpose(0, 1).reshape(nkv, -1, hd)

        k, v = rows(kp, ki), rows(vp, vi)
        # a row past the end of the cache holds whatever the block does: no weight, and no 0 * NaN
        v = torch.where((j < x + c)[None, :, None], v, 0.0)
        q = state["q"][at:at + c].float().view(c, nkv, group, hd).transpose(0, 1)
        for r0 in range(0, c, 256):
            n = min(256, c - r0)
            pos = torch.arange(x + r0, x + r0 + n, device="cuda")
            see = j[None, :] <= pos[:, None]
            if window:
                see &= (j[None, :] > pos[:, None] - window) | (j[None, :] < sinks)
            s = torch.bmm(q[:, r0:r0 + n].reshape(nkv, n * group, hd), k.transpose(1, 2).contiguous())
            s = torch.where(see[None, :, None, :], s.view(nkv, n, group, -1) / math.sqrt(hd), -math.inf)
            e = torch.exp(s - s.amax(-1, keepdim=True))
            o = torch.bmm((e / e.sum(-1, keepdim=True)).view(nkv, n * group, -1), v).view(nkv, n, group, hd)
            state["out"][at + r0:at + r0 + n] = o.transpose(0, 1).reshape(n, nq, hd).to(torch.bfloat16)
        at += c
    return state["out"]


def work(case):
    tok = 4 * case["nkv"] * case["hd"]  # bytes of one token's K and V
    if case["op"] == "copy":
        return {"bytes": max(1, case["layers"]) * (case["pairs"] + _sources(case)) * BLOCK * tok, "flops": 0}
    keys = pairs = rows = 0
    for c, x in _lens(case):
        ranges, p = _seen(c, x, case["window"], case["sinks"])
        keys += sum(b - a for a, b in ranges)
        pairs += p
        rows += c
    return {"bytes": keys * tok + rows * case["nq"] * case["hd"] * 4, "flops": 4.0 * case["nq"] * case["hd"] * pairs}


# --- the same results in fp64 ---------------------------------------------------
def exact(case, seed):
    st = _inputs(case, seed)
    if case["op"] == "copy":
        # where each block's contents come from
        origin = np.arange(case["blocks"])
        for s, d in zip(st["src"], st["dst"]):
            origin[d] = s
        origin = torch.from_numpy(origin).cuda()
        return {"pools": [tuple(p[origin] for p in layer) for layer in st["pools"]]}
    nq, nkv, hd, window, sinks = (case[n] for n in ("nq", "nkv", "hd", "window", "sinks"))
    (kp, vp), = st["pools"]
    # element (slot s, dimension d) of a stored block
    k_block = kp.view(-1, nkv, 2, hd // 8, 8, 8)  # [group][d / 8][slot of the group][d % 8]
    v_block = vp.view(-1, nkv, 2, hd, 8)          # [s / 8][d][s % 8]
    group_of = [[0, 1, 2, 3, 8, 9, 10, 11], [4, 5, 6, 7, 12, 13, 14, 15]]
    order = torch.tensor(group_of[0] + group_of[1], device="cuda").argsort()
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for c, x, table in st["requests"]:
        table = torch.from_numpy(table).long().cuda()
        end = x + c
        held = table >= 0
        for g in range(nkv):
            ids = table.clamp_min(0)
            k = k_block[ids, g].permute(0, 1, 3, 2, 4).reshape(-1, 16, hd)[:, order].reshape(-1, hd)[:end].double()
            v = v_block[ids, g].permute(0, 1, 3, 2).reshape(-1, hd)[:end].double()
            key = torch.arange(end, device="cuda")
            for r0 in range(0, c, 512):
                n = min(512, c - r0)
                p = torch.arange(x + r0, x + r0 + n, device="cuda")[:, None]
                hidden = (key > p) | ~held[key // BLOCK]
                if window:
                    hidden |= (key <= p - window) & (key >= sinks)
                for h in range(g * (nq // nkv), (g + 1) * (nq // nkv)):
                    s = st["q"][at + r0:at + r0 + n, h].double() @ k.t() * hd ** -0.5
                    out[at + r0:at + r0 + n, h] = torch.softmax(s.masked_fill(hidden, -math.inf), -1) @ v
        at += c
    return {"out": out}
