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
