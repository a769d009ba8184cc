"""The batch calls as a serving program uses them: prompts prefilled here and written to an 8-bit store, whose images become
pages of the decoding pool; then tokens one after another for all sequences at once, each call checked against the definition
on the very operands it was given; the same steps replayed from a graph."""
import numpy as np
import pytest

import synth_inputs as si
from oracle import serving
from q8_helpers import Batch, attention_bound, engine

pytestmark = pytest.mark.gpu
PT = 64


def decoding(kind, n_q, n_kv, hd, prompts, spare):
    """An engine with a head, its prompts' pages in a pool of 8-bit pages, and the batch's arrays with room for `spare` tokens."""
    import torch
    import paper_2410_03065_amd as cake
    shape = si.ModelShape("q8-serving", 2, 256, n_q, n_kv, hd, 512, 997, kind)
    eng = cake.Engine(shape, None, max_tokens=256, max_chunk=256, page_tokens=PT, with_head=True, seed=4)
    per = [(n + spare + PT - 1) // PT for n in prompts]
    pool = eng.new_q8_pool(sum(per) + 2, PT)
    order = np.random.default_rng(6).permutation(sum(per) + 2)[:sum(per)].astype(np.int32)
    table, at = np.full((len(prompts), max(per)), -1, np.int32), 0
    page = cake.q8_page_bytes(shape, PT)
    ids = [np.random.default_rng([n, 8]).integers(0, shape.vocab, n).astype(np.int32) for n in prompts]
    for s, n in enumerate(prompts):
        table[s, :per[s]] = order[at:at + per[s]]
        at += per[s]
        eng.clear_pool()
        eng.prefill_chunk(ids[s], 0, n)
        images = eng.write_store(n, cake.STORE_INT8)                     # [pages][layers of a page]
        assert images.shape[1] == shape.n_layers * page
        for p in range(len(images)):
            pool[:, int(table[s, p])] = images[p].view(shape.n_layers, page).cuda()
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    return eng, pool, table, i32(table), i32(prompts), i32(np.arange(len(prompts) + 1)), ids


@pytest.mark.parametrize("kind,n_q,n_kv,hd", [("bf16", 8, 2, 64), ("bf16", 4, 1, 128), ("f32", 4, 4, 64)])
def test_tokens_one_after_another_from_a_written_store(kind, n_q, n_kv, hd):
    import torch
    import paper_2410_03065_amd as cake
    prompts = [150, 64, 1]                                               # inside a page, at its end, a single token
    eng, pool, table, d_table, lens, begin, ids = decoding(kind, n_q, n_kv, hd, prompts, 4)
    s = eng.shape
    batch = eng.q8_batch(pool, d_table, lens, begin, n_rows=3, page_tokens=PT, max_rows=1, max_len=256)
    rope = cake.rope(s.rope_theta, hd)
    freq, magnitude = serving.rope_frequencies(s.rope_theta, hd)
    u = torch.tensor([0.2, 0.9, 0.5], device="cuda")
    k, p = torch.tensor([0, 50, 0], dtype=torch.int32, device="cuda"), torch.tensor([0.9, 0.8, 1.0], device="cuda")
    tokens = torch.tensor([int(i[-1]) for i in ids], device="cuda")
    lens.sub_(1)                                                         # the prompts' last tokens again, as the first rows
    half = 2.0 ** -8 if kind == "bf16" else 2.0 ** -24
    for step in range(4):
        lens.add_(1)
        host_lens = lens.cpu().numpy()
        x = eng.embed[tokens.long()].float()
        for layer, w in enumerate(eng.layer_tensors):
            qkv = eng.op_gemm(eng.op_rmsnorm(x, w["attn_norm"]), w["wqkv"])
            pages = serving.Pages(pool.shape[1], n_kv, PT, hd, 1).take(pool[layer].cpu().numpy())
            q = eng.op_append_q8(qkv, layer, batch, rope)
            want_q, _ = serving.append(pages, qkv.cpu().numpy(), table, host_lens, np.arange(4), n_q, freq, magnitude, "pairs")
            np.testing.assert_array_equal(pool[layer].cpu().numpy(), pages.bytes())
            got_q = q.double().cpu().numpy()
            assert (np.abs(got_q - want_q) <= half * np.abs(want_q) + 2.0 ** -24 * np.abs(want_q) + 1e-9).all()
            o = eng.op_attention_q8(q, layer, batch)
            want, size, mass, reach = serving.attention(pages, got_q, table, host_lens, np.arange(4))
            got = o.double().cpu().numpy().reshape(want.shape)
            assert (np.abs(got - want) <= attention_bound(kind, hd, want, size, mass, reach, int(host_lens.max()))).all()
            x = eng.op_gemm_residual(o, w["wo"], x)
            x = eng.op_gemm_residual(eng.op_gemm_swiglu(eng.op_rmsnorm(x, w["ffn_norm"]), w["w_gate"], w["w_up"]), w["w_down"], x)
        logits = eng.op_gemm(eng.op_rmsnorm(x, eng.final_norm), eng.lm_head) * 20
        tokens, logprobs = eng.op_sample(logits, u, top_k=k, top_p=p)
        want_t, want_lp = serving.sample(logits.cpu().numpy(), u.cpu().numpy(), None, k.cpu().numpy(), p.cpu().numpy())
        np.testing.assert_array_equal(tokens.cpu().numpy(), want_t)
        assert (np.abs(logprobs.double().cpu().numpy() - want_lp) <= 2.0 ** -24 * np.abs(want_lp) + 1e-7).all()
    assert lens.tolist() == [n + 3 for n in prompts]


def test_steps_replayed_from_a_graph():
    """Append, attention, sampling and the lengths' advance in one graph, replayed beside eager work of the program: every replay
    leaves what the same step leaves when it is called."""
    import torch
    import paper_2410_03065_amd as cake
    eng, pool, _, d_table, lens, begin, _ = decoding("bf16", 8, 2, 64, [150, 60, 1], 9)
    rope = cake.rope(10000.0, 64)
    qkv, u = torch.zeros((3, 12 * 64), device="cuda"), torch.rand(3, device="cuda")
    p = torch.full((3,), 0.9, device="cuda")

    def step(pool, lens):
        batch = eng.q8_batch(pool, d_table, lens, begin, n_rows=3, page_tokens=PT, max_rows=1, max_len=192)
        lens.add_(1)
        o = eng.op_attention_q8(eng.op_append_q8(qkv, 1, batch, rope), 1, batch, window=100, sinks=4)
        return eng.op_sample(o.float(), u, top_p=p)[0]
    other, other_lens = pool.clone(), lens.clone()
    step(pool.clone(), lens.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(pool, lens)
    for seed in range(8):
        qkv.copy_(torch.from_numpy(np.random.default_rng(seed).standard_normal(qkv.shape).astype(np.float32)))
        u.uniform_()
        graph.replay()
        tokens = got.clone()
        want = step(other, other_lens)
        torch.cuda.synchronize()
        assert torch.equal(tokens, want) and torch.equal(pool, other) and torch.equal(lens, other_lens)


def test_a_batch_of_another_model_is_refused():
    import torch
    import paper_2410_03065_amd as cake
    b = Batch(engine(4, 2, 64, "bf16"), [70], [1])
    other, same = engine(4, 4, 64, "bf16"), engine(8, 2, 64, "bf16")
    with pytest.raises(cake.CakeError):
        other.op_attention_q8(torch.zeros((4, 1, 64), dtype=torch.bfloat16, device="cuda"), 0, b.q8)
    with pytest.raises(cake.CakeError):
        other.op_append_q8(torch.zeros((1, 12 * 64), device="cuda"), 0, b.q8, cake.rope(10000.0, 64))
    assert same.op_attention_q8(torch.zeros((8, 1, 64), dtype=torch.bfloat16, device="cuda"), 0, b.q8).shape == (1, 512)


def test_an_engine_on_the_default_stream_refuses_a_capture():
    import torch
    import paper_2410_03065_amd as cake
    eng = engine(4, 2, 64, "bf16", compute_stream=torch.cuda.default_stream())
    b = Batch(eng, [70], [1])
    q = torch.zeros((4, 1, 64), dtype=torch.bfloat16, device="cuda")
    want = eng.op_attention_q8(q, 0, b.q8).clone()
    held = torch.zeros(4, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held.add_(1)
        with pytest.raises(cake.CakeError) as e:
            eng.op_attention_q8(q, 0, b.q8)
    assert e.value.code == cake.E_STATE
    graph.replay()
    assert held.tolist() == [1.0] * 4 and torch.equal(eng.op_attention_q8(q, 0, b.q8), want)
