"""The binding's requests: lengths and block tables whose low 32 bits would be valid are refused, not shortened."""
import numpy as np
import pytest

WIDE = 1 << 32


@pytest.fixture(scope="module")
def H():
    from paper_2503_22562_amd import hb
    hb.load()
    return hb


class Handle:
    handle, n_tokens = None, 0


class Shape:
    hidden, n_q_heads, n_kv_heads, head_dim, ffn_dim = 256, 4, 2, 64, 688
    rope_theta, rms_eps, kv_block = 5e5, 1e-5, 16


GOOD = (5, 20, np.arange(2, dtype=np.int32))
BAD = [(WIDE + 5, 20, [0, 1]), (5, WIDE + 20, [0, 1]), (5, 20 - WIDE, [0, 1]), (np.int64(WIDE + 5), 20, [0, 1]),
       (5, 20, np.arange(2) + WIDE), (5, 20, np.array([0, 1 - WIDE])), (5, 20, [0, WIDE]),
       (5, 20, np.array([0, 1 << 31])), (5, 20, np.array([0, WIDE], np.uint64)), (5, 20, np.array([0.0, 1.5])),
       (5, 20, np.array([0.0, WIDE + 1.0])), (5, 20, np.array([0.0, np.nan]))]


@pytest.mark.parametrize("bad", BAD, ids=range(len(BAD)))
def test_requests_that_do_not_fit(H, bad):
    cfg = H.make_config(Shape, 64, 4)
    for reqs in ([bad], [GOOD, bad], [bad, GOOD, GOOD]):
        for call in (lambda: H.hb_plan_attention(Handle, reqs), lambda: H.hb_run_iteration(Handle, reqs, None, None, 0),
                     lambda: H.hb_run_iteration_noalloc(Handle, reqs, None, None, 0),
                     lambda: H.hb_run_model(Handle, reqs, None, None),
                     lambda: H.hb_validate_batch(cfg, 4, reqs, 0x1000, 0x100000)):
            with pytest.raises(ValueError):
                call()


def test_other_tables_and_lengths(H):
    class Keys:
        shape = (5,)

        @staticmethod
        def data_ptr():
            return 0x1000

    class Many(Keys):
        shape = (WIDE + 5,)

    for table, context, k in ((np.array([0, WIDE + 1]), 20, Keys), ([0, 1], WIDE + 20, Keys), ([0, 1], 20, Many)):
        with pytest.raises(ValueError):
            H.hb_append_kv(Handle, table, context, k, k)
    cfg = H.make_config(Shape, 64, 4)
    with pytest.raises(ValueError):
        H.hb_latency_features(cfg, [(WIDE + 5, 20)])
    model = H.hb_latency_model()
    with pytest.raises(ValueError):
        H.hb_select_chunk(model, cfg, np.array([WIDE + 5]), [50.0], 0.0, 0, 64, 32)


@pytest.mark.parametrize("table", [np.array([7, 2], np.int32), np.array([7, 2]), np.array([7, 2], np.uint8), [7, 2],
                                   (7, 2), np.array([7.0, 2.0]), np.array([7, 9, 2, 9], np.int32)[::2]])
def test_requests_arrive_as_given(H, table):
    d, keep = H._desc([(5, 20, table), GOOD, (1, 0, [3, 3, 3])], 0, 0, H.HB_OUT_BF16)
    got = [(r.chunk_len, r.context_len, r.block_table[:r.n_blocks]) for r in (d.requests[i] for i in range(3))]
    assert got == [(5, 20, [7, 2]), (5, 20, [0, 1]), (1, 0, [3, 3, 3])]
    cfg = H.make_config(Shape, 64, 4)
    assert H.hb_validate_batch(cfg, 8, [(5, 20, table)], 0x1000, 0x100000) == H.HB_OK
    assert H.hb_validate_batch(cfg, 7, [(5, 20, table)], 0x1000, 0x100000) == H.HB_ERR_RANGE


def test_a_pool_of_too_many_blocks(H):
    """Refused before the list of its moves is allocated."""
    for num_blocks in (WIDE + 4, 1 << 45, -WIDE):
        with pytest.raises(ValueError):
            H.hb_plan_compaction(num_blocks, [[1, 2]])
