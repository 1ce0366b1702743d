"""What hb_run_append, hb_set_attention_rope, hb_sample and hb_rope_frequencies refuse, and the frequencies (CPU)."""
import ctypes as C
import math
import os
import subprocess
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_22562_amd", "csrc")
sys.path.insert(0, ROOT)

OK, INVALID, UNSUPPORTED = 0, 1, 5


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("args") / "arguments_driver")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    f"-I{CSRC}", f"-I{os.path.join(ROOT, 'include')}", os.path.join(ROOT, "tests", "arguments_driver.cpp"),
                    os.path.join(CSRC, "hb_plan.cpp"), "-o", exe], check=True)

    def run(lines):
        env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0")
        env.pop("LD_PRELOAD", None)
        out = subprocess.run([exe], input="\n".join(" ".join(map(str, ln)) for ln in lines) + "\n", capture_output=True,
                             text=True, env=env)
        assert out.returncode == 0, out.stderr[-2000:]
        return [int(x) for x in out.stdout.split()]
    return run


NQ, NKV, HD, NB, T = 8, 2, 64, 10, 5
ROW, KV, POOL = NQ * HD, NKV * HD, NB * NKV * 16 * HD * 2
Q, KEYS, VALUES, OUT, KP, VP = (0x100000 * i for i in range(1, 7))


def append(**kw):
    a = dict(nq=NQ, nkv=NKV, hd=HD, nb=NB, T=T, blocks=NB, kp=KP, vp=VP, q=Q, qs=ROW, k=KEYS, ks=KV, v=VALUES, vs=KV, out=OUT,
             outs=ROW)
    assert set(kw) <= set(a)
    return ["append", *dict(a, **kw).values()]


def test_append_arguments(driver):
    fused = ROW + 2 * KV
    slices = dict(q=Q, qs=fused, k=Q + 2 * ROW, ks=fused, v=Q + 2 * (ROW + KV), vs=fused)
    end = 2 * ((T - 1) * ROW + ROW)  # of five rows of q
    good = [append(), append(blocks=NB + 1), append(out=Q), append(**slices), append(**slices, out=Q, outs=fused),
            append(qs=ROW + 8), append(qs=1 << 40, q=Q, out=Q, outs=1 << 40, T=1),
            append(out=Q, outs=ROW + 8, T=1),                       # in place; one row has no stride
            append(out=Q + end), append(out=Q - end), append(vp=KP + POOL), append(vp=KP - POOL),
            append(out=KP - end), append(out=VP + POOL), append(q=VP + POOL),
            # rows between the rows
            append(q=Q, qs=2 * ROW, out=Q + 2 * ROW, outs=2 * ROW), append(q=Q + 2 * ROW, qs=2 * ROW, out=Q, outs=2 * ROW),
            append(k=Q + 2 * ROW, ks=fused, q=Q, qs=fused, out=Q, outs=fused)]
    assert driver(good) == [OK] * len(good)
    bad = [append(q=0), append(k=0), append(v=0), append(out=0), append(kp=0), append(vp=0), append(blocks=NB - 1),
           append(qs=ROW - 8), append(qs=ROW + 4), append(qs=(1 << 40) + 8), append(qs=-ROW), append(qs=0),
           append(ks=KV - 8), append(vs=KV + 1), append(outs=ROW - 1), append(q=Q + 8), append(k=KEYS + 2), append(v=VALUES + 4),
           append(out=OUT + 8), append(kp=KP + 8), append(vp=VP + 2),
           append(out=Q, outs=ROW + 8), append(out=Q + 16), append(out=Q - 16), append(out=Q + end - 16),
           append(out=Q - end + 16), append(out=KEYS), append(out=VALUES + 16), append(vp=KP), append(vp=KP + POOL - 16),
           append(vp=KP - POOL + 16), append(out=KP), append(out=KP - end + 16), append(out=VP + POOL - 16),
           append(q=KP + 16), append(k=VP), append(v=KP),
           append(**slices, out=Q + 2 * ROW, outs=fused), append(**slices, out=Q + 2 * (ROW + KV), outs=fused),
           append(**slices, out=Q + 16, outs=fused), append(**slices, out=Q - 16, outs=fused),
           append(**slices, out=Q + 2 * fused, outs=fused),         # in place, one row further on
           append(**slices, out=Q, outs=fused + 8)]
    assert driver(bad) == [INVALID] * len(bad)


def test_rope_arguments(driver):
    def rope(hd=64, rotary=32, layout=0, magnitude=1.0, f=0.5, null=0):
        return ["rope", hd, rotary, layout, magnitude, f, null]

    good = [rope(), rope(rotary=64), rope(hd=128, rotary=128, layout=1), rope(rotary=16), rope(rotary=0, null=1),
            rope(magnitude=0.0), rope(f=0.0), rope(f=2.0 ** 20)]
    assert driver(good) == [OK] * len(good)
    bad = [rope(layout=2), rope(layout=-1), rope(null=1), rope(f="nan"), rope(f="inf"), rope(f=-0.5), rope(f=2.0 ** 20 + 1),
           rope(magnitude="nan"), rope(magnitude="inf"), rope(magnitude=-1.0), rope(magnitude=1e39)]
    assert driver(bad) == [INVALID] * len(bad)
    none = [rope(rotary=80), rope(rotary=-16), rope(rotary=8), rope(rotary=17), rope(rotary=1)]
    assert driver(none) == [UNSUPPORTED] * len(none)


ROWS, VOCAB = 4, 100
X = 0x100000
ARRAYS = {n: 0x1000 * (i + 1) for i, n in enumerate(("temperature", "top_k", "top_p", "min_p", "u", "tokens", "probs"))}


def sample(**kw):
    a = dict(rows=ROWS, vocab=VOCAB, n=ROWS, dtype=0, logits=X, stride=VOCAB, **ARRAYS)
    assert set(kw) <= set(a)
    return ["sample", *dict(a, **kw).values()]


def test_sample_arguments(driver):
    size = 4 * VOCAB * ROWS
    good = [sample(), sample(temperature=0, top_k=0, top_p=0, min_p=0, probs=0), sample(dtype=1, logits=X + 2),
            sample(stride=VOCAB + 1), sample(n=1), sample(n=0, logits=0, u=0, tokens=0), sample(tokens=X + size),
            sample(tokens=X - 4 * ROWS), sample(probs=ARRAYS["u"] + 4 * ROWS), sample(temperature=ARRAYS["u"]),
            sample(stride=1 << 40)]
    assert driver(good) == [OK] * len(good)
    bad = [sample(n=-1), sample(n=ROWS + 1), sample(dtype=2), sample(dtype=-1), sample(n=0, dtype=3), sample(logits=0), sample(u=0),
           sample(tokens=0), sample(stride=VOCAB - 1), sample(stride=(1 << 40) + 1), sample(stride=-VOCAB), sample(logits=X + 2),
           sample(dtype=1, logits=X + 1), sample(tokens=X + size - 4), sample(probs=X - 4 * ROWS + 4),
           sample(probs=ARRAYS["tokens"]), sample(tokens=ARRAYS["u"]), sample(probs=ARRAYS["min_p"] + 4 * ROWS - 4)]
    bad += [sample(**{n: at + 2}) for n, at in ARRAYS.items()]
    bad += [sample(tokens=ARRAYS[n]) for n in ("temperature", "top_k", "top_p", "min_p")]
    assert driver(bad) == [INVALID] * len(bad)


@pytest.fixture(scope="module")
def H():
    from paper_2503_22562_amd import hb
    hb.load()
    return hb


@pytest.mark.parametrize("rotary", [2, 32, 128])
def test_frequencies(H, rotary):
    theta, s, lo, hi, length = 5e5, 8.0, 1.0, 4.0, 8192
    f = [theta ** (-2 * j / rotary) for j in range(rotary // 2)]
    assert np.allclose(H.hb_rope_frequencies(rotary, theta), f, rtol=1e-14, atol=0)
    assert np.allclose(H.hb_rope_frequencies(rotary, theta, s), np.array(f) / s, rtol=1e-14, atol=0)
    got = H.hb_rope_frequencies(rotary, theta, s, lo, hi, length)
    for g, w in zip(got, f):
        turns = length * w / (2 * math.pi)
        if turns <= lo:
            w /= s
        elif turns < hi:
            part = (turns - lo) / (hi - lo)
            w = part * w + (1 - part) * w / s
        assert abs(g - w) <= 1e-14 * w
    if rotary == 128:  # the three parts are there
        r = np.array(f) * length / (2 * math.pi)
        assert (r > hi).any() and (r < lo).any() and ((r > lo) & (r < hi)).any()
    assert len(H.hb_rope_frequencies(0, theta)) == 0


def test_frequencies_refused(H):
    def status(rotary=32, theta=1e4, scaling=(0, 0, 0.0, 0.0, 0.0), out=True, none=False):
        f = np.zeros(64)
        return H.load().hb_rope_frequencies(rotary, theta, None if none else C.byref(H.hb_rope_scaling(*scaling)),
                                            f.ctypes.data if out else None)

    assert status() == OK and status(none=True) == OK and status(scaling=(1, 0, 0.5, 0, 0)) == OK
    assert status(scaling=(2, 1, 2.0, 0.0, 1.0)) == OK
    inf, nan = math.inf, math.nan
    for bad in (dict(out=False), dict(rotary=-2), dict(rotary=31), dict(theta=1.0), dict(theta=nan), dict(theta=inf), dict(theta=-5.0),
                *(dict(scaling=s) for s in ((3, 0, 1.0, 0, 0), (-1, 0, 1.0, 0, 0), (1, 0, 0.0, 0, 0), (1, 0, -1.0, 0, 0),
                                            (1, 0, inf, 0, 0), (1, 0, nan, 0, 0), (2, 0, 2.0, 1, 4), (2, 8192, 2.0, 4, 4),
                                            (2, 8192, 2.0, -1, 4), (2, 8192, 2.0, 1, inf), (2, 8192, 2.0, nan, 4),
                                            (2, 8192, 0.0, 1, 4)))):
        assert status(**bad) == INVALID, bad
    with pytest.raises(ValueError):
        H.hb_rope_frequencies(32, 1e4, low=1.0, high=4.0)
    with pytest.raises(ValueError):
        H.hb_rope_frequencies(32, 1e4, 8.0, low=1.0)
    with pytest.raises(H.HBError):
        H.hb_rope_frequencies(32, 1e4, 0.0)


def test_null_handles(H):
    lib = H.load()
    assert lib.hb_run_append(None, None, None, 0, None, 0, None, 0, None, 0) == INVALID
    assert lib.hb_plan_shared_attention(None, 0, None, 0, None) == INVALID
    assert lib.hb_set_attention_rope(None, 0, 0, None, 1.0) == INVALID
    assert lib.hb_sample(None, None) == INVALID
    assert lib.hb_create_sampler(1, 1, None, None) == INVALID
    out = C.c_void_p(5)
    for rows, vocab, want in ((0, 8, INVALID), (8, 0, INVALID), (-1, 8, INVALID), ((1 << 20) + 1, 8, UNSUPPORTED),
                              (8, (1 << 20) + 1, UNSUPPORTED)):
        assert lib.hb_create_sampler(rows, vocab, None, C.byref(out)) == want and not out.value
    lib.hb_destroy_sampler(None)


WIDE = 1 << 32


def test_groups_and_sizes_that_do_not_fit(H):
    class Handle:
        handle, n_tokens = None, 0

    good = [(1, 40, [0, 1, 2]), (1, 40, [0, 1, 3])]
    for groups in ([(WIDE, 2, 32)], [(0, WIDE + 2, 32)], [(0, 2, WIDE + 32)], np.array([[0, 2, WIDE + 32]]), [(0, 2)],
                   [(0, 2, 32, 1)], [0, 2, 32], [(0, 2, 32.5)]):
        with pytest.raises(ValueError):
            H.hb_plan_shared_attention(Handle, good, groups)
    for args in ((WIDE + 4, 100), (4, WIDE + 100)):
        with pytest.raises(ValueError):
            H.hb_create_sampler(*args, stream=0)
    with pytest.raises(ValueError):
        H.hb_rope_frequencies(WIDE + 32, 1e4)
    with pytest.raises(ValueError):
        H.hb_set_attention_rope(Handle, np.ones(16), layout=WIDE)
