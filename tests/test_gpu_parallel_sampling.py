"""Several answers to one prompt, as a serving loop draws them: the prompt's pages shared through the tables, each new token
rotated, appended, attended and answered by a token drawn from the resulting logits, which is the next step's input."""
import numpy as np
import pytest

from attnref import assert_close, reference
from hb_workloads import LayerShape
from test_gpu_batch_append import rotated, within
from test_gpu_sample import drawn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nqkvhd,samples,prompt", [((8, 2, 128), 6, 165), ((4, 4, 64), 19, 48), ((32, 8, 128), 33, 1200)])
def test_parallel_sampling(hb, nqkvhd, samples, prompt):
    import torch
    from paper_2503_22562_amd.harness import bf16_bits, k_by_slot, v_by_slot
    from hb_workloads import bf16_bits_to_f32
    nq, nkv, hd = nqkvhd
    shape = LayerShape("heads", 64, nq, nkv, hd, 16, weight_seed=7)
    vocab, hidden, steps = 777, 256, 5
    gen = torch.Generator(device="cuda")
    gen.manual_seed(prompt)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    embed = rand(vocab, hidden).to(torch.bfloat16)
    w_qkv = (rand((nq + 2 * nkv) * hd, hidden) * hidden ** -0.5).to(torch.bfloat16)
    w_out = rand(vocab, nq * hd) * 3 * (nq * hd) ** -0.5
    blocks = -(-prompt // 16) + 3 * samples
    k_pool, v_pool = (torch.zeros(blocks, nkv, 16, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    f = hb.hb_rope_frequencies(hd, 5e5, 4.0, 1.0, 4.0, 512)
    a, b = nq * hd, (nq + nkv) * hd
    att = hb.hb_create_attention(hb.make_config(shape, max(prompt, samples), samples), blocks)
    hb.hb_set_attention_rope(att, f)
    sampler = hb.hb_create_sampler(samples, vocab)
    tables = [list(range(-(-prompt // 16)))]
    heads = lambda t: t.float().cpu().numpy().astype(np.float64).reshape(t.shape[0], -1, hd)

    def layer(requests, ids):
        """Queries rotated in place, keys and values appended, attention: the rows' outputs, all checked."""
        qkv = embed[ids] @ w_qkv.t()
        before = qkv.clone()
        hb.hb_run_append(att, qkv[:, :a], qkv[:, a:b], qkv[:, b:], k_pool, v_pool, qkv[:, :a])
        out = torch.empty(len(ids), nq, hd, dtype=torch.bfloat16, device="cuda")
        hb.hb_run_attention(att, qkv[:, :a], k_pool, v_pool, out)
        pos = np.concatenate([np.arange(x, x + c) for c, x, _ in requests])
        y, size = rotated(heads(before[:, :b]), pos, f, False, 1.0)
        within(heads(qkv[:, :a]), y[:, :nq], size[:, :nq], "queries")
        k_all = bf16_bits_to_f32(k_by_slot(bf16_bits(k_pool))).astype(np.float64)
        v_all = bf16_bits_to_f32(v_by_slot(bf16_bits(v_pool).reshape(blocks, nkv, 2, hd, 8))).astype(np.float64)
        at = 0
        for r, (c, x, t) in enumerate(requests):
            j = np.arange(x + c)
            page = np.asarray(t)[j // 16]
            k, v = k_all[page, :, j % 16], v_all[page, :, j % 16]
            within(k[x:], y[at:at + c, nq:], size[at:at + c, nq:], f"keys of request {r}")
            assert np.array_equal(v[x:], heads(before[at:at + c, b:]))
            o, pv = reference(heads(qkv[at:at + c, :a]), k, v, np.arange(x, x + c), 0, 0)
            assert_close(heads(out[at:at + c]), o, pv, f"request {r}")
            at += c
        return out

    requests = [(prompt, 0, tables[0])]
    hb.hb_plan_attention(att, requests)
    ids = torch.randint(0, vocab, (prompt,), generator=gen, device="cuda")
    out = layer(requests, ids)[-1:].expand(samples, nq, hd)
    # the fork: full pages shared, the last, partly filled one copied for each
    full, used = prompt // 16, -(-prompt // 16)
    own = np.arange(used, used + 3 * samples, dtype=np.int32).reshape(samples, 3)
    if prompt % 16:
        for p in (k_pool, v_pool):
            p[torch.from_numpy(own[:, 0]).long().cuda()] = p[full].clone()
    tables = [np.concatenate([np.arange(full), own[i]]).astype(np.int32) for i in range(samples)]
    t = torch.full((samples,), 0.9, device="cuda")
    top_p, top_k = torch.full((samples,), 0.9, device="cuda"), torch.full((samples,), 40, dtype=torch.int32, device="cuda")
    tokens, probs = torch.empty(samples, dtype=torch.int32, device="cuda"), torch.empty(samples, device="cuda")
    for step in range(steps):
        logits = out.reshape(samples, -1).float() @ w_out.t()
        u = torch.rand(samples, generator=gen, device="cuda")
        hb.hb_sample(sampler, logits, u, tokens, temperature=t, top_k=top_k, top_p=top_p, probs=probs)
        x, un = logits.cpu().numpy(), u.cpu().numpy()
        for i in range(samples):
            want = drawn(x[i], np.float32(0.9), 40, np.float32(0.9), 0.0, un[i])
            assert tokens[i].item() == want[0] and abs(probs[i].item() - want[1]) <= 2.0 ** -23 * want[1]
        requests = [(1, prompt + step, tables[i]) for i in range(samples)]
        hb.hb_plan_shared_attention(att, requests, [(0, samples, 16 * full)])
        out = layer(requests, tokens.long())
    assert len(set(tokens.tolist())) > 1
