"""Parallel sampling over the paged KV cache: the calls with which a serving loop
adds tokens to the cache, attends over a prompt that several requests share and
draws the next tokens, and the same results in plain torch.

A case holds plain values only:
  op        "append" (hb_run_append), "prefix" (hb_run_attention of a plan made by
            hb_plan_shared_attention) or "sample" (hb_sample)
  mix       seed of the lengths and settings, which thus belong to the case
append and prefix:
  nq, nkv, hd   query heads, kv heads, head dimension
append:
  chunks, chunk_lo, chunk_hi, off_lo, off_hi   number of prefill chunks, the
            range of their lengths and of the contexts before them
  decodes, ctx_lo, ctx_hi   number of decodes, the range of their contexts
            (spread over the logarithm)
  rotary    leading dimensions of a head that are rotated
  interleaved   pairs are neighbours (else: halves apart)
  scaling   "none", "linear" or "parts"
prefix:
  groups, members_lo, members_hi   groups of requests that share a prefix, and
            the range of their sizes
  prefix_lo, prefix_hi   range of the prefixes' lengths in tokens (rounded to pages)
  own_lo, own_hi   range of the tokens behind the prefix (spread over the logarithm)
  rows_hi   new tokens of a request: 1 to this many (1: decodes)
  alone     decodes that share nothing, with prefix_lo to prefix_hi tokens of their own
sample:
  rows, vocab
  bf16      logits in bf16 (else fp32)
  pad       values between the rows of the logits
  top_k, top_p, min_p   which limits the rows have (their values differ by row)
  flat, masked   share of the rows with nearly even logits, and of rows most of
            whose tokens a grammar has masked
"""
import dataclasses
import math
import random

import numpy as np
import torch

own = False

BLOCK = 16
THETA, FACTOR, LOW, HIGH, ORIGINAL = 5e5, 8.0, 1.0, 4.0, 8192


def _append(name, heads, chunks, decodes, rotary, interleaved, scaling, mix):
    n, clo, chi, olo, ohi = chunks
    d, lo, hi = decodes
    c = {"op": "append", "nq": heads[0], "nkv": heads[1], "hd": heads[2], "chunks": n, "chunk_lo": clo, "chunk_hi": chi,
         "off_lo": olo, "off_hi": ohi, "decodes": d, "ctx_lo": lo, "ctx_hi": hi, "rotary": rotary,
         "interleaved": interleaved, "scaling": scaling, "mix": mix}
    return dict(c, name=name) if name else c


def _prefix(name, heads, groups, members, prefix, tokens, rows_hi, alone, mix):
    c = {"op": "prefix", "nq": heads[0], "nkv": heads[1], "hd": heads[2], "groups": groups, "members_lo": members[0],
         "members_hi": members[1], "prefix_lo": prefix[0], "prefix_hi": prefix[1], "own_lo": tokens[0],
         "own_hi": tokens[1], "rows_hi": rows_hi, "alone": alone, "mix": mix}
    return dict(c, name=name) if name else c


def _sample(name, rows, vocab, bf16, pad, top_k, top_p, min_p, flat, masked, mix):
    c = {"op": "sample", "rows": rows, "vocab": vocab, "bf16": bf16, "pad": pad, "top_k": top_k, "top_p": top_p,
         "min_p": min_p, "flat": flat, "masked": masked, "mix": mix}
    return dict(c, name=name) if name else c


# (query heads, kv heads, head dimension) of the shapes in hb_workloads, and of layers without shared heads
TINY, L8B, L70B, L8B_TP2, L70B_TP8 = (4, 2, 64), (32, 8, 128), (64, 8, 128), (16, 4, 128), (8, 1, 128)
MHA64, MHA128, MQA = (12, 12, 64), (16, 16, 128), (16, 1, 128)
NO_CHUNK, NO_DECODE = (0, 0, 0, 0, 0), (0, 0, 0)


def listed():
    return [
        # one user's next token: launch latency
        _append("append-dec1", L8B, NO_CHUNK, (1, 6001, 6001), 128, False, "none", 1),
        # a decode queue of a model that rotates half of each head, neighbours paired
        _append("append-dec64-part32", MHA64, NO_CHUNK, (64, 1, 4096), 32, True, "none", 2),
        # the usual hybrid batch on one of two GPUs, long contexts, frequencies scaled by parts
        _append("append-tp2-chunk777-dec45", L8B_TP2, (1, 777, 777, 5234, 5234), (45, 300, 131072), 128, False, "parts", 3),
        # the largest: a busy replica's prompts, odd lengths
        _append("append-70b-4chunks", L70B, (4, 777, 1500, 0, 30720), (8, 512, 32768), 128, False, "linear", 4),
        # eight samples of one prompt, just begun
        _prefix("prefix-8-of-2048", L8B, 1, (8, 8), (2048, 2048), (1, 128), 1, 0, 5),
        # a tensor-parallel replica: one kv head, few rows, an agent's long instructions; drafts of up to four tokens
        _prefix("prefix-tp8-2groups", L70B_TP8, 2, (11, 16), (4000, 7000), (1, 900), 4, 3, 6),
        # a chat service: every request behind one system prompt, conversations of different lengths
        _prefix("prefix-64-of-8192", L8B, 1, (64, 64), (8192, 8192), (100, 2000), 1, 0, 7),
        # the largest: many samples each of three long documents' questions, and a few requests of others
        _prefix("prefix-3groups-256", L8B, 3, (80, 84), (12000, 16384), (16, 1024), 1, 10, 8),
        # one user's next token, nucleus sampling
        _sample("sample-1", 1, 128256, False, 0, False, True, False, 0.0, 0.0, 9),
        # a decode queue whose users chose different limits
        _sample("sample-64", 64, 128256, False, 0, True, True, True, 0.1, 0.1, 10),
        # a small odd vocabulary in bf16, many equal logits, rows inside a wider buffer
        _sample("sample-33-bf16", 33, 32003, True, 5, True, True, False, 0.2, 0.2, 11),
        # the largest decode queue, one row in four nearly even: a high temperature, or a model at the start of training
        _sample("sample-256", 256, 128256, False, 0, False, True, True, 0.25, 0.05, 12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


# no drawn case costs more than the largest listed ones: append-70b-4chunks, prefix-3groups-256, sample-256
MAX_BYTES = {"append": 1.7e8, "prefix": 7e8, "sample": 1.3e8}
MAX_FLOPS = {"append": 1e9, "prefix": 5.5e10, "sample": 1e9}


def draw(rng):
    while True:
        op = rng.choice(["append", "prefix", "sample"])
        mix = rng.randrange(1 << 30)
        if op == "append":
            heads = rng.choice([TINY, L8B, L8B, L70B, L8B_TP2, L70B_TP8, MHA64, MHA128, MQA])
            chunks = rng.choice([0, 0, 1, 1, 2, 4])
            hi = _log_int(rng, 1, 2048 // max(1, chunks))
            decodes = 0 if chunks and rng.random() < 0.3 else _log_int(rng, 1, 256)
            rotary = rng.choice([heads[2], heads[2], heads[2] // 2, heads[2] // 4, 16 * rng.randint(1, heads[2] // 16)])
            c = _append("", heads, (chunks, max(1, hi // 3) if chunks > 1 else hi, hi, 0, rng.choice([0, 1000, 30720])),
                        (decodes, 1, rng.choice([100, 8192, 131072])), rotary, rng.random() < 0.4,
                        rng.choice(["none", "linear", "parts"]), mix)
        elif op == "prefix":
            heads = rng.choice([TINY, L8B, L8B, L8B, L70B, L8B_TP2, L70B_TP8, MHA64, MHA128, MQA])
            groups = rng.choice([1, 1, 2, 4])
            members = _log_int(rng, 2, 256 // groups)
            plen = _log_int(rng, 64, 16384)
            c = _prefix("", heads, groups, (max(1, members // 2), members), (max(16, plen // 2), plen),
                        (1, rng.choice([64, 500, 2000])), rng.choice([1, 1, 1, 4]), rng.choice([0, 0, rng.randint(1, 16)]),
                        mix)
        else:
            vocab = rng.choice([128256, 32768, _log_int(rng, 1000, 128256)])
            c = _sample("", _log_int(rng, 1, 256), vocab, rng.random() < 0.3, rng.choice([0, 0, rng.randint(1, 64)]),
                        rng.random() < 0.5, rng.random() < 0.7, rng.random() < 0.4, rng.choice([0.0, 0.25]),
                        rng.choice([0.0, 0.25]), mix)
        w = work(c)
        if w["bytes"] <= MAX_BYTES[op] and w["flops"] <= MAX_FLOPS[op]:
            return c


# --- what a case's lengths and settings are: functions of the case alone -----------
def _append_lens(case):
    """(chunk_len, context_len) of each request, chunks first."""
    rng = random.Random(case["mix"])
    lens = [(rng.randint(case["chunk_lo"], case["chunk_hi"]), rng.randint(case["off_lo"], case["off_hi"]))
            for _ in range(case["chunks"])]
    return lens + [(1, _log_int(rng, case["ctx_lo"], case["ctx_hi"])) for _ in range(case["decodes"])]


def _prefix_lens(case):
    """(chunk_len, context_len) of each request, and (first, count, prefix_len) of each group."""
    rng = random.Random(case["mix"])
    lens, groups = [], []
    for _ in range(case["groups"]):
        p = max(BLOCK, rng.randint(case["prefix_lo"], case["prefix_hi"]) // BLOCK * BLOCK)
        n = rng.randint(case["members_lo"], case["members_hi"])
        groups.append((len(lens), n, p))
        for _ in range(n):
            c = rng.randint(1, case["rows_hi"])
            lens.append((c, p + _log_int(rng, case["own_lo"], case["own_hi"]) - 1))
    for _ in range(case["alone"]):
        lens.append((1, rng.randint(case["prefix_lo"], case["prefix_hi"])))
    return lens, groups


def _settings(case):
    """Temperature, top_k, top_p and min_p of each row."""
    rng = random.Random(case["mix"])
    rows = []
    for _ in range(case["rows"]):
        t = 0.0 if case["rows"] > 8 and rng.random() < 0.1 else rng.uniform(0.6, 1.2)
        rows.append((t, rng.choice([0, 1, 20, 50, rng.randint(1, case["vocab"])]) if case["top_k"] else 0,
                     rng.choice([0.5, 0.9, 0.95, 0.99, 1.0]) if case["top_p"] else 1.0,
                     rng.choice([0.0, 0.02, 0.05, 0.1]) if case["min_p"] else 0.0))
    t, k, p, m = zip(*rows)
    return {"temperature": np.array(t, np.float32), "top_k": np.array(k, np.int32), "top_p": np.array(p, np.float32),
            "min_p": np.array(m, np.float32)}


def work(case):
    if case["op"] == "sample":
        n = case["rows"] * case["vocab"]
        # per logit: its distance to the maximum, over the temperature, its weight, their sum
        return {"bytes": n * (2 if case["bf16"] else 4) + case["rows"] * 28, "flops": 4.0 * n}
    nq, nkv, hd = case["nq"], case["nkv"], case["hd"]
    if case["op"] == "append":
        rows = sum(c for c, _ in _append_lens(case))
        return {"bytes": rows * (nq + 2 * nkv) * hd * 4, "flops": 3.0 * rows * (nq + nkv) * case["rotary"]}
    lens, groups = _prefix_lens(case)
    keys = sum(c + x for c, x in lens) - sum((n - 1) * p for _, n, p in groups)
    rows = sum(c for c, _ in lens)
    pairs = sum(c * x + c * (c + 1) // 2 for c, x in lens)
    return {"bytes": keys * 4 * nkv * hd + rows * nq * hd * 4, "flops": 4.0 * nq * hd * pairs}


# --- inputs, from the seed alone -----------------------------------------------------
def _normal(gen, shape, std=1.0):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=gen)


def _logits(case, gen):
    """Rows as a language model's head gives them: a broad bulk and a few tens of likely tokens far above it."""
    rows, vocab = case["rows"], case["vocab"]
    rng = random.Random(case["mix"] + 1)
    x = torch.empty((rows, vocab), device="cuda").normal_(0.0, 1.0, generator=gen)
    likely = torch.rand((rows, 40), device="cuda", generator=gen)
    ids = (likely * vocab).long().clamp_(max=vocab - 1)
    rise = 16.0 - 3.0 * torch.log(1.0 + torch.arange(40, device="cuda")) + torch.rand((rows, 40), device="cuda", generator=gen)
    flat = torch.tensor([rng.random() < case["flat"] for _ in range(rows)], device="cuda")
    spread = torch.tensor([rng.uniform(1.5, 2.5) for _ in range(rows)], device="cuda")
    x = torch.where(flat[:, None], x, x * spread[:, None])
    x.scatter_(1, ids, torch.where(flat[:, None], x.gather(1, ids), rise))
    masked = torch.tensor([rng.random() < case["masked"] for _ in range(rows)], device="cuda")
    hide = masked[:, None] & (torch.rand((rows, vocab), device="cuda", generator=gen) < 0.99)
    hide[:, vocab // 2] = False  # a grammar leaves something
    x.masked_fill_(hide, -math.inf)
    out = torch.zeros((rows, vocab + case["pad"]), dtype=torch.bfloat16 if case["bf16"] else torch.float32, device="cuda")
    out[:, :vocab] = x
    return out[:, :vocab]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    perm = np.random.default_rng(seed)
    if case["op"] == "sample":
        return {"logits": _logits(case, gen), "u": torch.rand(case["rows"], device="cuda", generator=gen)}
    nq, nkv, hd = case["nq"], case["nkv"], case["hd"]
    tables, used = [], 0
    if case["op"] == "append":
        lens = _append_lens(case)
        # earlier tokens lie in pages that all of them share; the new tokens' pages are their own
        common = 64
        used = common
        for c, x in lens:
            n, first = -(-(c + x) // BLOCK), x // BLOCK
            t = np.arange(n, dtype=np.int32) % common
            t[first:] = np.arange(used, used + n - first)
            used += n - first
            tables.append(t)
    else:
        lens, groups = _prefix_lens(case)
        shared = {}  # request -> its group's (first page, number of pages)
        for first, n, p in groups:
            for r in range(first, first + n):
                shared[r] = (used, p // BLOCK)
            used += p // BLOCK
        for r, (c, x) in enumerate(lens):
            at, k = shared.get(r, (0, 0))
            n = -(-(c + x) // BLOCK)
            tables.append(np.concatenate([np.arange(at, at + k), np.arange(used, used + n - k)]).astype(np.int32))
            used += n - k
    blocks = used + 16
    ids = perm.permutation(blocks).astype(np.int32)
    st = {"requests": [(c, x, ids[t]) for (c, x), t in zip(lens, tables)], "blocks": blocks}
    rows = sum(c for c, _ in lens)
    # pools in the layouts of include/hb.h: K [2][hd/8][8][8], V [2][hd][8] per block and kv head
    st["k_pool"], st["v_pool"] = (_normal(gen, (blocks, nkv, 16, hd)) for _ in range(2))
    if case["op"] == "append":
        st["qkv"] = _normal(gen, (rows, (nq + 2 * nkv) * hd))
    else:
        st["q"] = _normal(gen, (rows, nq, hd))
        st["groups"] = groups
    return st


def _qkv(state, case):
    """q, k and v as slices of the fused projection's rows."""
    a, b = case["nq"] * case["hd"], (case["nq"] + case["nkv"]) * case["hd"]
    x = state["qkv"]
    return x[:, :a], x[:, a:b], x[:, b:]


def prepare(case, seed):
    st = dict(_inputs(case, seed), case=case)
    if case["op"] == "sample":
        for n, v in _settings(case).items():
            st[n] = torch.from_numpy(v).cuda()
        st["tokens"] = torch.empty(case["rows"], dtype=torch.int32, device="cuda")
        st["probs"] = torch.empty(case["rows"], device="cuda")
        if own:
            from paper_2503_22562_amd import hb
            st["sampler"] = hb.hb_create_sampler(case["rows"], case["vocab"])
        return st
    rows = sum(r[0] for r in st["requests"])
    st["out"] = torch.empty(rows, case["nq"], case["hd"], dtype=torch.bfloat16, device="cuda")
    if not own:
        # the plain forms look positions and pages up on the GPU
        if case["op"] == "append":
            pos = np.concatenate([np.arange(x, x + c) for c, x, _ in st["requests"]])
            page = np.concatenate([t[np.arange(x, x + c) // BLOCK] for c, x, t in st["requests"]])
            st["pos"], st["page"] = torch.from_numpy(pos).cuda(), torch.from_numpy(page).long().cuda()
        else:
            st["tables"] = [torch.from_numpy(t).long().cuda() for _, _, t in st["requests"]]
        return st
    from hb_workloads import LLAMA3_8B
    from paper_2503_22562_amd import hb
    shape = dataclasses.replace(LLAMA3_8B, name="heads", hidden=64, n_q_heads=case["nq"], n_kv_heads=case["nkv"],
                                head_dim=case["hd"], ffn_dim=16)
    # one plan serves every layer of an iteration
    att = st["attention"] = hb.hb_create_attention(hb.make_config(shape, rows, len(st["requests"])), st["blocks"])
    if case["op"] == "append":
        scaling = {"none": {}, "linear": dict(factor=FACTOR),
                   "parts": dict(factor=FACTOR, low=LOW, high=HIGH, original_context=ORIGINAL)}[case["scaling"]]
        hb.hb_set_attention_rope(att, hb.hb_rope_frequencies(case["rotary"], THETA, **scaling),
                                 hb.HB_ROPE_INTERLEAVED if case["interleaved"] else hb.HB_ROPE_HALF)
        hb.hb_plan_attention(att, st["requests"])
    else:
        hb.hb_plan_shared_attention(att, st["requests"], st["groups"])
    return st


def run(state):
    case = state["case"]
    if case["op"] == "append":
        if own:
            from paper_2503_22562_amd import hb
            q, k, v = _qkv(state, case)
            hb.hb_run_append(state["attention"], q, k, v, state["k_pool"], state["v_pool"], state["out"])
        else:
            _plain_append(state, case)
        return {"q": state["out"], "k_pool": state["k_pool"], "v_pool": state["v_pool"]}
    if case["op"] == "prefix":
        if own:
            from paper_2503_22562_amd import hb
            hb.hb_run_attention(state["attention"], state["q"], state["k_pool"], state["v_pool"], state["out"])
        else:
            _plain_attention(state, case)
        return {"out": state["out"]}
    if own:
        from paper_2503_22562_amd import hb
        hb.hb_sample(state["sampler"], state["logits"], state["u"], state["tokens"], temperature=state["temperature"],
                     top_k=state["top_k"], top_p=state["top_p"], min_p=state["min_p"], probs=state["probs"])
        return {"tokens": state["tokens"], "probs": state["probs"]}
    return _plain_sample(state, case)


# --- plain forms -----------------------------------------------------------------------
def _k_index(hd):
    """Flat positions of K[slot][dim] inside a stored block of one kv head."""
    s, d = torch.meshgrid(torch.arange(16, device="cuda"), torch.arange(hd, device="cuda"), indexing="ij")
    return ((s // 4 % 2) * (hd // 8) + d // 8) * 64 + (4 * (s // 8) + s % 4) * 8 + d % 8


def _v_index(hd):
    s, d = torch.meshgrid(torch.arange(16, device="cuda"), torch.arange(hd, device="cuda"), indexing="ij")
    return (s // 8 * hd + d) * 8 + s % 8


def _frequencies(case):
    r = case["rotary"]
    f = THETA ** (-2.0 * torch.arange(r // 2, dtype=torch.float64, device="cuda") / r)
    if case["scaling"] == "linear":
        f = f / FACTOR
    elif case["scaling"] == "parts":
        g = ((ORIGINAL * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
        f = f * (g + (1 - g) / FACTOR)
    return f


def _plain_append(state, case):
    nq, nkv, hd, r = case["nq"], case["nkv"], case["hd"], case["rotary"]
    angle = state["pos"].double()[:, None] * _frequencies(case)  # far positions: 64 bits
    cos, sin = (f(angle).float()[:, None, :] for f in (torch.cos, torch.sin))

    def rotated(x):
        a, b = (x[..., 0:r:2], x[..., 1:r:2]) if case["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
        y = (a * cos - b * sin, b * cos + a * sin)
        y = torch.stack(y, -1).flatten(-2) if case["interleaved"] else torch.cat(y, -1)
        return torch.cat([y, x[..., r:]], -1).to(torch.bfloat16)

    q, k, v = (x.reshape(x.shape[0], -1, hd) for x in _qkv(state, case))
    state["out"].copy_(rotated(q.float()))
    slot, head = state["pos"] % BLOCK, torch.arange(nkv, device="cuda")
    for pool, index, x in ((state["k_pool"], _k_index(hd), rotated(k.float())), (state["v_pool"], _v_index(hd), v)):
        pool.view(-1, nkv, 16 * hd)[state["page"][:, None, None], head[None, :, None], index[slot][:, None, :]] = x


def _plain_attention(state, case):
    nq, nkv, hd = case["nq"], case["nkv"], case["hd"]
    ki, vi = _k_index(hd).reshape(-1), _v_index(hd).reshape(-1)
    group, at = nq // nkv, 0
    for (c, x, _), table in zip(state["requests"], state["tables"]):
        def rows(pool, index):  # [n_kv][keys][hd]
            b = pool.view(-1, nkv, 16 * hd)[table][:, :, index].float()
            return b.view(len(table), nkv, 16, hd).transpose(0, 1).reshape(nkv, -1, hd)[:, :x + c]

        k, v = rows(state["k_pool"], ki), rows(state["v_pool"], vi)
        see = torch.arange(x + c, device="cuda")[None, :] <= torch.arange(x, x + c, device="cuda")[:, None]
        q = state["q"][at:at + c].float().view(c, nkv, group, hd).transpose(0, 1).reshape(nkv, c * group, hd)
        s = torch.bmm(q, k.transpose(1, 2).contiguous()).view(nkv, c, group, -1) / math.sqrt(hd)
        s = torch.where(see[None, :, None, :], s, -math.inf)
        e = torch.exp(s - s.amax(-1, keepdim=True))
        o = torch.bmm((e / e.sum(-1, keepdim=True)).view(nkv, c * group, -1), v.contiguous()).view(nkv, c, group, hd)
        state["out"][at:at + c] = o.transpose(0, 1).reshape(c, nq, hd).to(torch.bfloat16)
        at += c


def _plain_sample(state, case):
    """All rows sorted: the kept tokens are the first n of the descending order."""
    vocab = case["vocab"]
    x, order = torch.sort(state["logits"].float(), dim=-1, descending=True, stable=True)
    t = state["temperature"].double()
    greedy = t <= 0
    # weights and their sums decide between neighbours: 64 bits
    w = torch.exp((x.double() - x[:, :1].double()) / torch.where(greedy, 1.0, t)[:, None])
    k = torch.where((state["top_k"] <= 0) | (state["top_k"] > vocab), vocab, state["top_k"]).long()
    k = torch.where(greedy, 1, k)
    place = torch.arange(vocab, device="cuda")[None, :]
    w = torch.where(place < k[:, None], w, 0.0)
    cum = torch.cumsum(w, -1)
    p = state["top_p"].double()
    short = (cum < (p * cum[:, -1])[:, None]).sum(-1) + 1  # up to the token that reaches p
    n = torch.where(p < 1, torch.minimum(k, short), k)
    n = torch.minimum(n, (w >= state["min_p"].double()[:, None]).sum(-1)).clamp(min=1)
    total = cum.gather(1, n[:, None] - 1)
    j = (cum <= state["u"].double()[:, None] * total).sum(-1)
    j = torch.minimum(j, n - 1)[:, None]
    state["tokens"].copy_(order.gather(1, j)[:, 0])
    state["probs"].copy_((w.gather(1, j) / total)[:, 0])
    return {"tokens": state["tokens"], "probs": state["probs"]}


# --- the same results in fp64 -------------------------------------------------------------
def exact(case, seed):
    st = _inputs(case, seed)
    if case["op"] == "sample":
        return _exact_sample(case, st)
    nq, nkv, hd = case["nq"], case["nkv"], case["hd"]
    # element (slot, dimension) of a stored block: K [group][d / 8][slot of the group][d % 8], V [s / 8][d][s % 8]
    if case["op"] == "append":
        r = case["rotary"]
        out, at = torch.empty(st["qkv"].shape[0], nq, hd, dtype=torch.float64, device="cuda"), 0
        kp = st["k_pool"].double().view(-1, nkv, 2, hd // 8, 8, 8)
        vp = st["v_pool"].double().view(-1, nkv, 2, hd, 8)
        freq = []
        for j in range(r // 2):
            f = math.exp(-2.0 * j / r * math.log(THETA))
            if case["scaling"] == "linear":
                f /= FACTOR
            elif case["scaling"] == "parts":
                turns = ORIGINAL * f / (2 * math.pi)
                g = min(1.0, max(0.0, (turns - LOW) / (HIGH - LOW)))
                f = g * f + (1.0 - g) * f / FACTOR
            freq.append(f)
        first = list(range(0, r, 2)) if case["interleaved"] else list(range(r // 2))
        second = list(range(1, r, 2)) if case["interleaved"] else list(range(r // 2, r))
        for c, x, table in st["requests"]:
            pos = torch.arange(x, x + c, device="cuda")
            z = torch.polar(torch.ones(c, r // 2, dtype=torch.float64, device="cuda"),
                            pos.double()[:, None] * torch.tensor(freq, dtype=torch.float64, device="cuda"))[:, None, :]
            rows = st["qkv"][at:at + c].double().view(c, nq + 2 * nkv, hd)
            heads = rows[:, :nq + nkv]
            turned = torch.complex(heads[..., first], heads[..., second]) * z
            heads = heads.clone()
            heads[..., first], heads[..., second] = turned.real, turned.imag
            out[at:at + c] = heads[:, :nq]
            page, s = torch.from_numpy(table).long().cuda()[pos // BLOCK], pos % BLOCK
            for d8 in range(hd // 8):
                kp[page, :, (s >> 2) & 1, d8, 4 * (s >> 3) + (s & 3)] = heads[:, nq:, 8 * d8:8 * d8 + 8]
            vp[page, :, s >> 3, :, s & 7] = rows[:, nq + nkv:]
            at += c
        return {"q": out, "k_pool": kp.view(st["k_pool"].shape), "v_pool": vp.view(st["v_pool"].shape)}
    k_block, v_block = st["k_pool"].view(-1, nkv, 2, hd // 8, 8, 8), st["v_pool"].view(-1, nkv, 2, hd, 8)
    order = torch.tensor([0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15], device="cuda").argsort()
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for c, x, table in st["requests"]:
        ids, end = torch.from_numpy(table).long().cuda(), x + c
        hidden = torch.arange(end, device="cuda")[None, :] > torch.arange(x, end, device="cuda")[:, None]
        for g in range(nkv):
            k = k_block[ids, g].permute(0, 1, 3, 2, 4).reshape(-1, 16, hd)[:, order].reshape(-1, hd)[:end].double()
            v = v_block[ids, g].permute(0, 1, 3, 2).reshape(-1, hd)[:end].double()
            for h in range(g * (nq // nkv), (g + 1) * (nq // nkv)):
                s = st["q"][at:at + c, h].double() @ k.t() * hd ** -0.5
                out[at:at + c, h] = torch.softmax(s.masked_fill(hidden, -math.inf), -1) @ v
        at += c
    return {"out": out}


def _exact_sample(case, st):
    """Row by row on the host: thresholds on the values, sums in extended precision."""
    logits, u = st["logits"].float().cpu().numpy().astype(np.float64), st["u"].cpu().numpy().astype(np.float64)
    par = _settings(case)
    tokens, probs = np.zeros(case["rows"], np.int32), np.zeros(case["rows"])
    for r in range(case["rows"]):
        t, k, p, m = (float(par[n][r]) for n in ("temperature", "top_k", "top_p", "min_p"))
        x, top = logits[r], logits[r].max()
        if t <= 0:
            tokens[r], probs[r] = int(np.flatnonzero(x == top)[0]), 1.0
            continue
        rank = np.lexsort((np.arange(len(x)), -x))
        if 0 < k < len(x):
            rank = rank[:int(k)]
        w = np.exp((x[rank] - top) / t).astype(np.longdouble)
        if p < 1:
            reached = np.flatnonzero(np.cumsum(w) >= np.longdouble(p) * w.sum())
            w = w[:reached[0] + 1] if len(reached) else w
        w = w[w >= m]
        cum = np.cumsum(w)
        j = int(np.searchsorted(cum, np.longdouble(u[r]) * cum[-1], side="right"))
        j = min(j, len(w) - 1)
        tokens[r], probs[r] = rank[j], float(w[j] / cum[-1])
    return {"tokens": torch.from_numpy(tokens).cuda(), "probs": torch.from_numpy(probs).cuda()}
