"""hb_run_attention at the edges of what its documentation allows."""
import numpy as np
import pytest

from attnref import Cache
from hb_workloads import LayerShape

pytestmark = pytest.mark.gpu


def heads(nq, nkv, hd):
    return LayerShape(f"{nq}q{nkv}kv{hd}", 64, nq, nkv, hd, 16, weight_seed=7)


def test_out_must_not_overlap_a_pool(hb):
    """Rows written into the blocks that the same call reads are refused; memory right before and behind them is not."""
    import torch
    from paper_2503_22562_amd import hb as H
    from paper_2503_22562_amd.harness import to_device_bf16
    cache = Cache(heads(8, 2, 128), 12, 8, 4, seed=41)
    request, _, _ = cache.request(3, 100, 0, 0)
    row, n = 8 * 128, 12 * 2 * 16 * 128
    att = H.hb_create_attention(cache.dl.cfg, 12)
    H.hb_plan_attention(att, [request])
    q = to_device_bf16(cache.bits(3, 8, 128))
    # both pools in one allocation, with room for the three rows before, between and behind them
    gap = 4 * row
    arena = torch.zeros(3 * gap + 2 * n, dtype=torch.bfloat16, device="cuda")
    k, v = arena[gap:gap + n], arena[2 * gap + n:2 * gap + 2 * n]
    k.copy_(cache.dl.k_pool.reshape(-1))
    v.copy_(cache.dl.v_pool.reshape(-1))
    want = torch.empty(3, row, dtype=torch.bfloat16, device="cuda")
    H.hb_run_attention(att, q, k, v, want)
    before = arena.clone()

    def out(at, stride=row):
        return torch.as_strided(arena, (3, row), (stride, 1), at)

    for at, stride in ((gap, row), (gap - 8, row), (gap - 3 * row + 8, row), (gap + n - 8, row),
                       (2 * gap + n, row), (2 * gap + n - row, row), (2 * gap + 2 * n - row, row),
                       (0, gap + n)):  # rows before, between and behind the pools, which lie between them
        with pytest.raises(H.HBError) as e:
            H.hb_run_attention(att, q, k, v, out(at, stride))
        assert e.value.status == H.HB_ERR_INVALID and "pool" in str(e.value), (at, stride)
    torch.cuda.synchronize()
    assert torch.equal(arena.view(torch.int16), before.view(torch.int16))
    for at in (gap - 3 * row, gap + n, 2 * gap + n - 3 * row, 2 * gap + 2 * n):
        H.hb_run_attention(att, q, k, v, out(at))
        torch.cuda.synchronize()
        assert torch.equal(out(at), want), at


@pytest.mark.parametrize("nqkvhd,c,x,window", [((8, 2, 128), 1, 700, 1), ((4, 2, 64), 5, 40, 1), ((8, 2, 128), 90, 200, 1),
                                               ((8, 2, 128), 1, 3000, 0), ((8, 1, 128), 80, 900, 0)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_of_any_documented_size(hb, nqkvhd, c, x, window, sign):
    """Scores of 2^26 (exponents of 2^23 and 2^23.5), of either sign. Where a row sees one key, that key's V; where it
    sees them all, the mean of V over the first 7 keys, whose scores are equal and lie 2^20 and more above the others'.
    The weights are powers of two off by up to half a unit of the maximum, so they and the output are rounded once each."""
    import torch
    from paper_2503_22562_amd import hb as H
    from paper_2503_22562_amd.harness import to_device_bf16
    from hb_workloads import bf16_bits_to_f32, f32_to_bf16_bits
    nq, nkv, hd = nqkvhd
    n = x + c
    cache = Cache(heads(*nqkvhd), -(-n // 16), c, 1, seed=43)
    k, q = np.zeros((n, nkv, hd), np.float32), np.zeros((c, nq, hd), np.float32)
    q[:, :, 0] = 2.0 ** 13
    k[:, :, 0] = sign * 2.0 ** 13
    if not window:
        k[7:, :, 0] = sign * 2.0 ** 13 - 2.0 ** 8 * (1 + np.arange(n - 7) % 3)[:, None]
    kb, qb, vb = f32_to_bf16_bits(k), f32_to_bf16_bits(q), cache.bits(n, nkv, hd)
    table = cache.perm.copy()
    cache.dl.append_kv(table, 0, kb, vb)
    att = H.hb_create_attention(cache.dl.cfg, cache.num_blocks)
    H.hb_plan_attention(att, [(c, x, table)], window, 0)
    out = torch.empty(c, nq, hd, dtype=torch.bfloat16, device="cuda")
    H.hb_run_attention(att, to_device_bf16(qb), cache.dl.k_pool, cache.dl.v_pool, out)
    torch.cuda.synchronize()
    v = np.repeat(bf16_bits_to_f32(vb).astype(np.float64), nq // nkv, 1)
    want, size = (v[x:], np.abs(v[x:])) if window else (v[:7].mean(0)[None], np.abs(v[:7]).mean(0)[None])
    got = out.float().cpu().numpy().astype(np.float64)
    assert (np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -12) * (size + np.abs(want))).all()
