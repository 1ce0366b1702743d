"""hb_sample against the definition in 64 bits, row by row on the host, through the C ABI.

Tokens are the same ones exactly. (Weights are summed as multiples of 2^-45 of the largest, off by 2^-46 each: with V
tokens some border moves by V 2^-46 at most, below 2^-29 of the kept weight here, and u, top_p and the weights are
random, so of the some 10^4 rows here none is expected to lie that close to one; where borders are met exactly, all
weights are powers of two and the sums exact.) probs are one division of such sums, rounded to fp32: half a step, 2^-24,
of the value, and 2^-29 for the sums."""
import numpy as np
import pytest

from hb_workloads import bf16_bits_to_f32, f32_to_bf16_bits

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def drawn(x, t, k, p, m, u):
    """(token, probability) of one row by the definition in hb.h."""
    x = np.where(np.isnan(x), -np.inf, np.minimum(x.astype(np.float64), float(np.finfo(np.float32).max)))
    top = x.max()
    if top == -np.inf:
        return 0, 0.0
    order = np.argsort(-x, kind="stable")
    if not t > 0:
        return int(order[0]), 1.0
    with np.errstate(over="ignore", invalid="ignore"):
        e = (x[order] - top) / float(t)
    w = np.where(x[order] == -np.inf, 0.0, np.exp(e))
    n = len(w) if k <= 0 else min(int(k), len(w))
    if p < 1:
        cum = np.cumsum(w[:n])
        n = min(n, int((cum < float(p) * cum[-1]).sum()) + 1)
    if m > 0:
        n = min(n, int((w >= float(m)).sum()))
    n = max(n, 1)
    u = min(float(u), 1 - 2.0 ** -24) if u > 0 else 0.0
    cum = np.cumsum(w[:n])
    j = min(int((cum <= u * cum[-1]).sum()), n - 1)
    return int(order[j]), float(w[j] / cum[-1])


def draw(hb, x, u, dtype="f32", pad=0, sampler=None, **settings):
    """Tokens and probs of the rows x (fp32, or values that bf16 holds)."""
    import torch
    rows, vocab = x.shape
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    wide = torch.full((rows * (vocab + pad) + 3,), 77.0, dtype=t, device="cuda")
    logits = torch.as_strided(wide, (rows, vocab), (vocab + pad, 1), pad % 3)
    if dtype == "f32":
        logits.copy_(torch.from_numpy(np.ascontiguousarray(x, np.float32)))
    else:
        bits = f32_to_bf16_bits(x)
        assert np.array_equal(bf16_bits_to_f32(bits), x, equal_nan=True)
        logits.copy_(torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16))
    dev = {n: torch.from_numpy(np.asarray(v, np.int32 if n == "top_k" else np.float32)).cuda() for n, v in settings.items()}
    tokens = torch.full((rows + 2,), -7, dtype=torch.int32, device="cuda")
    probs = torch.full((rows + 2,), -7.0, device="cuda")
    s = sampler or hb.hb_create_sampler(rows, vocab)
    hb.hb_sample(s, logits, torch.from_numpy(np.asarray(u, np.float32)).cuda(), tokens[:rows], probs=probs[:rows], **dev)
    torch.cuda.synchronize()
    assert (tokens[rows:] == -7).all() and (probs[rows:] == -7).all()
    return tokens[:rows].cpu().numpy(), probs[:rows].cpu().numpy()


def check(hb, x, u, dtype="f32", pad=0, **settings):
    tokens, probs = draw(hb, x, u, dtype, pad, **settings)
    full = {n: np.asarray(settings.get(n, [d] * len(x)), np.int32 if n == "top_k" else np.float32)
            for n, d in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0))}
    u = np.asarray(u, np.float32)
    for r in range(len(x)):
        t, k, p, m = (full[n][r] for n in ("temperature", "top_k", "top_p", "min_p"))
        tok, prob = drawn(x[r], t, k, p, m, u[r])
        assert tokens[r] == tok, (r, tokens[r], tok, t, k, p, m, u[r])
        assert abs(probs[r] - prob) <= (2.0 ** -24 + 2.0 ** -29) * prob + 1e-38, (r, probs[r], prob)
    return tokens


def settings(rng, rows, vocab):
    return dict(temperature=rng.choice([0.0, 0.3, 0.7, 1.0, 1.5, 5.0], rows),
                top_k=rng.choice([0, 1, 2, 50, vocab // 2, vocab, vocab + 5, -3], rows),
                top_p=rng.choice([0.0, 0.1, 0.5, 0.9, 0.999, 1.0, 2.0], rows),
                min_p=rng.choice([0.0, 1e-6, 0.02, 0.3, 1.0, -1.0], rows))


def peaked(rng, rows, vocab):
    x = 2.0 * rng.standard_normal((rows, vocab))
    for r in range(rows):
        n = min(vocab, 30)
        x[r, rng.permutation(vocab)[:n]] = 14 - 2.5 * np.log1p(np.arange(n)) + rng.random(n)
    return x.astype(np.float32)


VOCABS = [1, 2, 3, 5, 63, 64, 65, 255, 1000, 4096, 4097, 8191, 32003]


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("shape", ["peaked", "flat", "equal", "few values"])
def test_any_vocabulary(hb, vocab, shape):
    rng = np.random.default_rng(vocab)
    rows = 24
    x = {"peaked": lambda: peaked(rng, rows, vocab), "flat": lambda: rng.standard_normal((rows, vocab)),
         "equal": lambda: np.full((rows, vocab), 1.5),
         "few values": lambda: np.log(2.0) * rng.integers(-3, 1, (rows, vocab))}[shape]().astype(np.float32)
    s = settings(rng, rows, vocab)
    if shape == "few values":
        s["temperature"][:] = 1.0  # (other temperatures: sums of equal weights may meet top_p but for a rounding)
        s["top_p"][:] = 1.0
    check(hb, x, rng.random(rows), **s)
    for name in ("top_k", "top_p", "min_p", "temperature"):  # one setting alone
        check(hb, x, rng.random(rows), **{name: s[name]})


@pytest.mark.parametrize("vocab", [7, 4097, 32003])
@pytest.mark.parametrize("pad", [0, 1, 2, 3, 5, 13])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_types_and_strides(hb, vocab, pad, dtype):
    """Rows that begin anywhere; bf16: many equal logits, taken by their index."""
    rng = np.random.default_rng(vocab + pad)
    x = np.concatenate([peaked(rng, 8, vocab), rng.standard_normal((8, vocab)).astype(np.float32)])
    if dtype == "bf16":
        x = bf16_bits_to_f32(f32_to_bf16_bits(x))
    check(hb, x, rng.random(16), dtype, pad, **settings(rng, 16, vocab))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_vocabulary(hb, dtype):
    """Rows whose kept tokens are more than are ever sorted at a time, among them all equal and of few values."""
    vocab = 128256
    rng = np.random.default_rng(5)
    x = np.concatenate([peaked(rng, 6, vocab), rng.standard_normal((6, vocab)), 0.05 * rng.standard_normal((4, vocab)),
                        np.full((4, vocab), -3.0), rng.integers(0, 4, (4, vocab)) / 4.0]).astype(np.float32)
    if dtype == "bf16":
        x = bf16_bits_to_f32(f32_to_bf16_bits(x))
    rows = len(x)
    for i in range(4):
        s = settings(rng, rows, vocab)
        s["temperature"] = rng.choice([0.5, 1.0, 3.0], rows)
        if i == 0:
            s = dict(temperature=s["temperature"])
        if i == 1:
            s["top_k"][:] = rng.integers(4000, vocab, rows)
        check(hb, x, rng.random(rows), dtype, **s)


def test_vocabulary_limit(hb):
    rng = np.random.default_rng(6)
    x = np.concatenate([rng.standard_normal((2, 1 << 20)), np.zeros((1, 1 << 20))]).astype(np.float32)
    check(hb, x, rng.random(3))
    check(hb, x, rng.random(3), top_p=[0.5, 0.9, 0.25], top_k=[900000, 0, 700000])


def test_masked_tokens(hb):
    """Grammar masks: -infinity, NaN and the type's lowest value; one token left; none."""
    rng = np.random.default_rng(7)
    vocab, rows = 5000, 40
    x = peaked(rng, rows, vocab)
    lowest = np.finfo(np.float32).min
    for r in range(rows):
        hide = rng.random(vocab) < rng.choice([0.5, 0.99, 0.9999])
        x[r, hide] = [-np.inf, np.nan, lowest][r % 3]
    x[0] = -np.inf
    x[1] = np.nan
    x[2] = lowest
    x[3], x[3, 4321] = -np.inf, -50.0
    x[4], x[4, 0] = np.nan, lowest
    x[5, 77] = np.inf
    x[6, [99, 7, 4000]] = np.inf
    x[7, ::2], x[7, 1::2] = -np.inf, np.nan
    s = settings(rng, rows, vocab)
    tokens = check(hb, x, rng.random(rows), **s)
    assert tokens[0] == tokens[1] == tokens[7] == 0 and tokens[3] == 4321 and tokens[4] == 0 and tokens[5] == 77
    for _ in range(3):
        check(hb, x, rng.random(rows), temperature=s["temperature"])
    _, probs = draw(hb, x, rng.random(rows))
    assert probs[0] == probs[1] == probs[7] == 0 and probs[3] == probs[4] == probs[5] == 1


def test_settings_at_their_ends(hb):
    rng = np.random.default_rng(8)
    x = np.repeat(peaked(rng, 1, 999), 60, 0)
    rows = len(x)
    for name, values in (("temperature", [0.0, -0.0, -1.0, NAN, -INF, INF, 1e-30, 1e-45, 1e30, 3e38, 1e-3]),
                         ("top_k", [0, -1, 1, 2, 998, 999, 1000, 2147483647, -2147483648]),
                         ("top_p", [0.0, -1.0, NAN, INF, -INF, 1e-30, 1.0 - 2.0 ** -24, 1.0]),
                         ("min_p", [0.0, -1.0, NAN, 1.0, 1.0 - 2.0 ** -24, 2.0, INF, -INF, 1e-30, 1e-45])):
        check(hb, x, rng.random(rows), **{name: [values[i % len(values)] for i in range(rows)]})
    us = [0.0, -0.0, -1.0, NAN, 1.0, 2.0, INF, -INF, 1.0 - 2.0 ** -24, 2.0 ** -24, 1e-45]
    check(hb, x, [us[i % len(us)] for i in range(rows)])
    check(hb, x, [us[i % len(us)] for i in range(rows)], top_p=[0.9] * rows, temperature=[2.0] * rows)
    signs = np.zeros((4, 64), np.float32)  # zeros of both signs are equal
    signs[:, ::3] = -0.0
    check(hb, signs, [0.0, 0.3, 0.6, 0.99])
    check(hb, signs, [0.0, 0.3, 0.6, 0.99], top_k=[1, 5, 20, 40], temperature=[0.0, 1.0, 1.0, 1.0])


def test_borders_that_are_met_exactly(hb):
    """Equal logits, whose weights are all 1: u and top_p on a border, below it and above it."""
    x = np.zeros((33, 8), np.float32)
    x[:, 1:4] = -np.inf
    u = np.arange(33, dtype=np.float32) / 32
    tokens = check(hb, x, u, top_p=np.full(33, 0.8, np.float32))
    assert sorted(set(tokens)) == [0, 4, 5, 6, 7]  # fp32's 0.8 is 13421773 / 2^24, above 4/5: all five
    tokens = check(hb, x, u, top_p=np.full(33, np.nextafter(np.float32(0.8), np.float32(0))))
    assert sorted(set(tokens)) == [0, 4, 5, 6]
    x = np.zeros((33, 4), np.float32)
    tokens = check(hb, x, u)
    assert list(tokens[:32]) == [i // 8 for i in range(32)] and tokens[32] == 3
    tokens = check(hb, x, np.full(33, 0.999), top_p=u)
    assert list(tokens) == [max(0, (i + 7) // 8 - 1) for i in range(33)]
    tokens = check(hb, np.zeros((5, 40000), np.float32), [0.0, 0.25, 0.5, 0.75, 0.99999])
    assert list(tokens) == [0, 10000, 20000, 30000, 39999]


def test_every_token_has_its_share(hb):
    """u over a grid: each token's interval has the length of its weight."""
    import torch
    w = np.array([0.05, 0.3, 0.15, 0.4, 0.1])
    n = 4000
    x = np.repeat(np.log(w).astype(np.float32)[None], n, 0)
    tokens = check(hb, x, (np.arange(n) + 0.5) / n)
    assert np.abs(np.bincount(tokens, minlength=5) / n - w).max() <= 1.0 / n
    assert list(dict.fromkeys(tokens)) == [3, 1, 2, 4, 0]  # the most likely first


def test_rows_and_streams(hb):
    """More rows than CUs; fewer than the sampler's; a sampler on another stream than the current one; no rows; no probs."""
    import torch
    rng = np.random.default_rng(9)
    x = peaked(rng, 700, 2000)
    u = rng.random(700)
    a = check(hb, x, u, top_p=np.full(700, 0.9))
    s = hb.hb_create_sampler(700, 2000)
    for n in (1, 3, 699):
        t, _ = draw(hb, x[:n], u[:n], sampler=s, top_p=np.full(n, 0.9))
        assert np.array_equal(t, a[:n])
    side = torch.cuda.Stream()
    s = hb.hb_create_sampler(700, 2000, stream=side.cuda_stream)
    logits, un = torch.from_numpy(x).cuda(), torch.from_numpy(u.astype(np.float32)).cuda()
    p = torch.full((700,), 0.9, device="cuda")
    tokens = torch.zeros(700, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    hb.hb_sample(s, logits, un, tokens, top_p=p)
    side.synchronize()
    assert np.array_equal(tokens.cpu().numpy(), a)
    tokens.zero_()
    torch.cuda.synchronize()
    hb.hb_sample(s, logits[:0], un[:0], tokens[:0])
    side.synchronize()
    assert (tokens == 0).all()


@pytest.mark.parametrize("rows,vocab", [(1, 128256), (5, 40000), (300, 3000)])
def test_captured_and_replayed(hb, rows, vocab):
    """A replay reads the logits, settings and numbers of its time; eager calls in between do it no harm."""
    import torch
    rng = np.random.default_rng(10)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s = hb.hb_create_sampler(rows, vocab)
        logits = torch.zeros(rows, vocab, device="cuda")
        u, t, p = (torch.zeros(rows, device="cuda") for _ in range(3))
        k = torch.zeros(rows, dtype=torch.int32, device="cuda")
        tokens, probs = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, device="cuda")
        other = torch.zeros(rows, dtype=torch.int32, device="cuda")
        side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        hb.hb_sample(s, logits, u, tokens, temperature=t, top_k=k, top_p=p, probs=probs)
    for i in range(5):
        x = peaked(rng, rows, vocab) if i % 2 else rng.standard_normal((rows, vocab)).astype(np.float32)
        un, tn, pn = (rng.random(rows).astype(np.float32) for _ in range(3))
        kn = rng.integers(0, vocab, rows).astype(np.int32)
        with torch.cuda.stream(side):
            for dst, src in ((logits, x), (u, un), (t, tn + 0.5), (p, pn), (k, kn)):
                dst.copy_(torch.from_numpy(src))
            graph.replay()
            if i % 2:
                hb.hb_sample(s, logits, u, other)  # eager, behind the replay
            side.synchronize()
        for r in range(rows if rows < 10 else 10):
            want = drawn(x[r], (tn + np.float32(0.5))[r], kn[r], pn[r], 0.0, un[r])
            assert tokens[r].item() == want[0] and abs(probs[r].item() - want[1]) <= 2.0 ** -23 * want[1], (i, r)


def test_the_same_tokens_every_time(hb):
    import torch
    rng = np.random.default_rng(11)
    x = np.concatenate([rng.standard_normal((20, 50000)), np.zeros((10, 50000))]).astype(np.float32)
    u, s = rng.random(30), dict(top_p=np.full(30, 0.7), top_k=rng.integers(0, 50000, 30))
    first = draw(hb, x, u, **s)
    for _ in range(4):
        again = draw(hb, x, u, **s)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])


def test_calls_that_are_refused(hb):
    import torch
    s = hb.hb_create_sampler(4, 100)
    x, u = torch.zeros(4, 100, device="cuda"), torch.zeros(4, device="cuda")
    tokens = torch.full((4,), -7, dtype=torch.int32, device="cuda")
    for args, kw in (((x.double(), u, tokens), {}), ((x[:, :99], u, tokens), {}), ((x.t(), u, tokens), {}), ((x.cpu(), u, tokens), {}),
                     ((x, u[:3], tokens), {}), ((x, u.double(), tokens), {}), ((x, u, tokens.long()), {}),
                     ((x, u, tokens), dict(top_k=u)), ((x, u, tokens), dict(top_p=u[:2])), ((x, u, tokens), dict(probs=tokens)),
                     ((x, u, tokens), dict(temperature=torch.zeros(8, device="cuda")[::2])), ((x[0], u, tokens), {})):
        with pytest.raises(ValueError):
            hb.hb_sample(s, *args, **kw)
    for args, kw in (((torch.zeros(5, 100, device="cuda"), torch.zeros(5, device="cuda"),
                       torch.zeros(5, dtype=torch.int32, device="cuda")), {}),
                     ((x, u, tokens), dict(probs=u)), ((x, u, tokens), dict(probs=x.view(-1)[8:12]))):
        with pytest.raises(hb.HBError) as e:
            hb.hb_sample(s, *args, **kw)
        assert e.value.status == hb.HB_ERR_INVALID
    torch.cuda.synchronize()
    assert (tokens == -7).all()
    hb.hb_destroy_sampler(s)
    hb.hb_destroy_sampler(s)


def crowded():
    """Rows whose k-th token stands in a crowd of equal ones that weighs as much as all before it, so that top_p and u
    may end at any of hundreds of distinct logits before it."""
    rng = np.random.default_rng(31)
    rows, vocab = 60, 6000
    x = np.full((rows, vocab), -1.5, np.float32)
    k = np.zeros(rows, np.int32)
    for r in range(rows):
        spread = rng.integers(500, 900)
        x[r, :spread] = -1.4 * rng.random(spread)
        x[r, spread + 1100:] = -2.0 - 2.0 * rng.random(vocab - spread - 1100)
        k[r] = spread + rng.integers(300, 900)
        x[r] = rng.permutation(x[r])
    return x, rng.random(rows), dict(top_k=k, top_p=rng.choice([0.2, 0.4, 0.5, 0.7], rows))


def test_many_tokens_among_which_a_limit_may_lie(hb):
    x, u, limits = crowded()
    check(hb, x, u, **limits)


@pytest.mark.parametrize("vocab", [5, 999, 30000])
@pytest.mark.parametrize("k", [2, 3, 50])
def test_top_p_of_minus_infinity_among_few_tokens(hb, vocab, k):
    """Nothing but the first token, also where the first k all stand at the top."""
    rng = np.random.default_rng(vocab + k)
    x = np.concatenate([np.full((4, vocab), 0.5), 1e-3 * rng.standard_normal((4, vocab)), peaked(rng, 4, vocab)])
    u = np.tile([0.0, 0.3, 0.7, 1.0], 3)
    tokens = check(hb, x.astype(np.float32), u, top_k=np.full(12, k), top_p=np.full(12, -INF))
    assert np.array_equal(tokens, x.astype(np.float32).argmax(1))


@pytest.mark.parametrize("vocab", [5, 999, 30000])
def test_min_p_of_1_where_every_weight_is_1(hb, vocab):
    """At temperatures so high that all weights are 1 in fp64, min_p = 1 keeps all; above 1 it keeps the first token."""
    rng = np.random.default_rng(vocab)
    x = np.repeat(rng.standard_normal((1, vocab)), 12, 0).astype(np.float32)
    u = np.tile([0.0, 0.3, 0.7, 0.999], 3)
    t = np.repeat([INF, 3e38, 1e30], 4)
    tokens = check(hb, x, u, temperature=t, min_p=np.ones(12))
    assert len(set(tokens)) == 4
    check(hb, x, u, temperature=t, min_p=np.ones(12), top_k=np.full(12, max(1, vocab // 3)), top_p=np.full(12, 0.9))
    tokens = check(hb, x, u, temperature=t, min_p=np.full(12, 1.0 + 2.0 ** -23))
    assert len(set(tokens)) == 1
    # exp(-d / t) is 1 in fp64 where d / t <= 2^-54, half its step below 1 (numpy's exp may be off by a step there): of
    # logits 2^-24 apart, the first t 2^-30 and one, and the token is the first place above u times their number
    near = np.repeat(np.float32(1) - np.float32(2.0 ** -24) * np.arange(vocab, dtype=np.float32)[None], 4, 0)
    t = np.array([1.0, 1e9, 2.5 * 2.0 ** 30, 1e13], np.float32)
    n = np.minimum(vocab, np.floor(t.astype(np.float64) * 2.0 ** -30) + 1)
    tokens, probs = draw(hb, near, u[:4], min_p=np.ones(4), temperature=t)
    assert np.array_equal(tokens, np.floor(u[:4].astype(np.float32) * n.astype(np.float64)))
    assert (np.abs(probs - 1 / n) <= 2.0 ** -24 / n).all()
