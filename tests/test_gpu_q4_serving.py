"""A decoding step in 4 bits as a serving program runs it: projections packed, prompts prefilled and written to a 4-bit store, whose images become
pages of the decoding pool; then tokens one after another through products with 4-bit weights, append, attention and sampling, each call checked
against the definition on the very operands it was given; a drafted chunk checked in one call; the same steps replayed from a graph."""
import numpy as np
import pytest

import synth_inputs as si
from oracle import serving
from test_gpu_q4_attention import bound_of

pytestmark = pytest.mark.gpu
PT = 64


class Pool:
    """What bound_of reads of a batch."""

    def __init__(self, eng, pages, table, lens, begin):
        self.eng, self.pages, self.table, self.lens, self.begin = eng, pages, table, lens, begin


def decoding(kind, n_q, n_kv, hd, prompts, spare, group=64):
    """An engine with a head, its layers' projections in 4 bits, its prompts' pages in a pool of 4-bit pages, and the batch's arrays with room
    for `spare` tokens."""
    import torch
    import paper_2410_03065_amd as cake
    shape = si.ModelShape("q4-serving", 2, 256, n_q, n_kv, hd, 512, 997, kind)
    eng = cake.Engine(shape, None, max_tokens=256, max_chunk=256, page_tokens=PT, with_head=True, seed=4)
    per = [(n + spare + PT - 1) // PT for n in prompts]
    pool = eng.new_q4_pool(sum(per) + 2, PT)
    order = np.random.default_rng(6).permutation(sum(per) + 2)[:sum(per)].astype(np.int32)
    table, at = np.full((len(prompts), max(per)), -1, np.int32), 0
    page = cake.q4_page_bytes(shape, PT)
    ids = [np.random.default_rng([n, 8]).integers(0, shape.vocab, n).astype(np.int32) for n in prompts]
    for s, n in enumerate(prompts):
        table[s, :per[s]] = order[at:at + per[s]]
        at += per[s]
        eng.clear_pool()
        eng.prefill_chunk(ids[s], 0, n)
        images = eng.write_store(n, cake.STORE_INT4)                     # [pages][layers of a page]
        assert images.shape[1] == shape.n_layers * page
        for p in range(len(images)):
            pool[:, int(table[s, p])] = images[p].view(shape.n_layers, page).cuda()
    packed = [{name: eng.pack_w4(w[name], group=group, want_values=True) for name in ("wqkv", "wo", "w_gate", "w_up", "w_down")} for w in eng.layer_tensors]
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    return eng, pool, table, i32(table), i32(prompts), i32(np.arange(len(prompts) + 1)), ids, packed


def product_bound(a, packed, group, kind):
    """As the products' own tests: what float32 sums of 24 + c within a group, and of the groups, may be off."""
    w, scales = serving.w4_values(packed.codes.cpu().numpy(), packed.scales.float().cpu().numpy(), packed.k, group), packed.scales.double().cpu().numpy()
    padded = np.zeros((len(a), scales.shape[1] * group))
    padded[:, :packed.k] = np.abs(a)
    inside = 32 * padded.reshape(len(a), scales.shape[1], -1).sum(axis=2) @ np.abs(scales).T
    terms = 3 if kind == "f32" else 1
    return a @ w.T, 2.0 ** -24 * (16 * (group // 32) * terms * inside + (scales.shape[1] + 16 + terms) * (np.abs(a) @ np.abs(w).T)) + 1e-37


@pytest.mark.parametrize("kind,n_q,n_kv,hd", [("bf16", 8, 2, 64), ("bf16", 4, 1, 128), ("f32", 4, 4, 64)])
def test_tokens_one_after_another_from_a_written_store(kind, n_q, n_kv, hd):
    import torch
    import paper_2410_03065_amd as cake
    prompts = [150, 64, 1]                                               # inside a page, at its end, a single token
    eng, pool, table, d_table, lens, begin, ids, packed = decoding(kind, n_q, n_kv, hd, prompts, 4)
    s = eng.shape
    batch = eng.q4_batch(pool, d_table, lens, begin, n_rows=3, page_tokens=PT, max_rows=1, max_len=256)
    rope = cake.rope(s.rope_theta, hd)
    freq, magnitude = serving.rope_frequencies(s.rope_theta, hd)
    u = torch.tensor([0.2, 0.9, 0.5], device="cuda")
    k, p = torch.tensor([0, 50, 0], dtype=torch.int32, device="cuda"), torch.tensor([0.9, 0.8, 1.0], device="cuda")
    tokens = torch.tensor([int(i[-1]) for i in ids], device="cuda")
    lens.sub_(1)                                                         # the prompts' last tokens again, as the first rows
    half = 2.0 ** -8 if kind == "bf16" else 2.0 ** -24

    def checked(got, a, w):
        want, bound = product_bound(a.double().cpu().numpy(), w, 64, kind)
        assert (np.abs(got.double().cpu().numpy() - want) <= bound).all()
        return got
    for step in range(4):
        lens.add_(1)
        host_lens = lens.cpu().numpy()
        x = eng.embed[tokens.long()].float()
        for layer, w in enumerate(eng.layer_tensors):
            w4 = {name: pair[0] for name, pair in packed[layer].items()}
            h = eng.op_rmsnorm(x, w["attn_norm"])
            qkv = checked(eng.op_gemm_w4(h, w4["wqkv"]), h, w4["wqkv"])
            pages = serving.Pages(pool.shape[1], n_kv, PT, hd, 1, 4).take(pool[layer].cpu().numpy())
            q = eng.op_append_q4(qkv, layer, batch, rope)
            want_q, _ = serving.append(pages, qkv.cpu().numpy(), table, host_lens, np.arange(4), n_q, freq, magnitude, "pairs")
            np.testing.assert_array_equal(pool[layer].cpu().numpy(), pages.bytes())
            got_q = q.double().cpu().numpy()
            assert (np.abs(got_q - want_q) <= half * np.abs(want_q) + 2.0 ** -24 * np.abs(want_q) + 1e-9).all()
            o = eng.op_attention_q4(q, layer, batch)
            of = serving.attention(pages, got_q, table, host_lens, np.arange(4))
            got = o.double().cpu().numpy().reshape(of[0].shape)
            assert (np.abs(got - of[0]) <= bound_of(Pool(eng, pages, table, host_lens, np.arange(4)), q, *of)).all()
            before = x.double().cpu().numpy()
            x = eng.op_gemm_w4_residual(o, w4["wo"], x)
            want, bound = product_bound(o.double().cpu().numpy(), w4["wo"], 64, kind)
            want = want + before
            assert (np.abs(x.double().cpu().numpy() - want) <= bound + 2.0 ** -24 * (np.abs(want) + np.abs(before))).all()
            h = eng.op_rmsnorm(x, w["ffn_norm"])
            act = eng.op_gemm_w4_swiglu(h, w4["w_gate"], w4["w_up"])
            (g, dg), (up, du) = (product_bound(h.double().cpu().numpy(), w4[name], 64, kind) for name in ("w_gate", "w_up"))
            want = serving.silu_product(g, up)
            bound = half * np.abs(want) + 1.1 * dg * (np.abs(up) + du) + np.abs(g) * du + 2.0 ** -20 * np.abs(want) * (1 + np.abs(g) / 16) + 1e-37
            assert (np.abs(act.double().cpu().numpy() - want) <= bound).all()
            x = eng.op_gemm_w4_residual(act, w4["w_down"], x)
        logits = eng.op_gemm(eng.op_rmsnorm(x, eng.final_norm), eng.lm_head) * 20
        tokens, logprobs = eng.op_sample(logits, u, top_k=k, top_p=p)
        want_t, want_lp = serving.sample(logits.cpu().numpy(), u.cpu().numpy(), None, k.cpu().numpy(), p.cpu().numpy())
        np.testing.assert_array_equal(tokens.cpu().numpy(), want_t)
        assert (np.abs(logprobs.double().cpu().numpy() - want_lp) <= 2.0 ** -24 * np.abs(want_lp) + 1e-7).all()
    assert lens.tolist() == [n + 3 for n in prompts]


def test_packed_weights_stand_for_what_the_products_use():
    """The product with packed weights is the bf16 product with the values that packing returns, but for what rounding those to bf16 changed."""
    eng, _, _, _, _, _, _, packed = decoding("bf16", 8, 2, 64, [5], 1)
    import torch
    h = torch.randn((70, 256), device="cuda").bfloat16()
    for name in ("wqkv", "w_gate"):
        w, values = packed[1][name]
        a, v = h.double().cpu().numpy(), values.double().cpu().numpy()
        want, bound = product_bound(a, w, 64, "bf16")
        got = eng.op_gemm_w4(h, w).double().cpu().numpy()
        assert (np.abs(got - want) <= bound).all() and (np.abs(got - a @ v.T) <= bound + 2.0 ** -8 * np.abs(a) @ np.abs(v).T * 1.01).all()


def test_a_chunk_of_drafted_tokens_leaves_what_single_tokens_leave():
    """Five tokens appended in one call or one at a time: the same pages (a scale per token), and the same attention up to its roundings."""
    import torch
    import paper_2410_03065_amd as cake
    eng, pool, table, d_table, lens, _, _, _ = decoding("bf16", 8, 2, 64, [150, 60], 6)
    rope = cake.rope(10000.0, 64)
    qkv = torch.randn((10, 12 * 64), device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    one, many = pool.clone(), pool.clone()
    batch = eng.q4_batch(many, d_table, lens + 5, i32([0, 5, 10]), n_rows=10, page_tokens=PT, max_rows=5, max_len=192)
    q = eng.op_append_q4(qkv, 0, batch, rope)
    together = eng.op_attention_q4(q, 0, batch)
    apart = torch.empty_like(together)
    for i in range(5):
        b = eng.q4_batch(one, d_table, lens + i + 1, i32([0, 1, 2]), n_rows=2, page_tokens=PT, max_rows=1, max_len=192)
        rows = [i, 5 + i]
        q1 = eng.op_append_q4(qkv[rows].contiguous(), 0, b, rope)
        assert torch.equal(q1, q[:, rows])
        apart[rows] = eng.op_attention_q4(q1, 0, b)
    assert torch.equal(one, many)
    pages = serving.Pages(pool.shape[1], 2, PT, 64, 1, 4).take(many[0].cpu().numpy())
    begin, host = np.array([0, 5, 10]), (lens + 5).cpu().numpy()
    of = serving.attention(pages, q.double().cpu().numpy(), table, host, begin)
    bound = bound_of(Pool(eng, pages, table, host, begin), q, *of)
    for got in (together, apart):
        assert (np.abs(got.double().cpu().numpy().reshape(of[0].shape) - of[0]) <= bound).all()


@pytest.mark.parametrize("rows", [1, 40])
def test_steps_replayed_from_a_graph(rows):
    """Products, append, attention, sampling and the lengths' advance in one graph, replayed beside eager work of the program: every replay leaves
    what the same step leaves when it is called.  Two such graphs share the context's workspace."""
    import torch
    import paper_2410_03065_amd as cake
    eng, pool, _, d_table, lens, _, _, packed = decoding("bf16", 8, 2, 64, [150, 60, 41], 9 * rows)
    rope = cake.rope(10000.0, 64)
    w = {name: pair[0] for name, pair in packed[1].items()}
    h, u = torch.zeros((3 * rows, 256), device="cuda", dtype=torch.bfloat16), torch.rand(3 * rows, device="cuda")
    begin = torch.arange(0, 3 * rows + 1, rows, dtype=torch.int32, device="cuda")
    p = torch.full((3 * rows,), 0.9, device="cuda")

    def step(pool, lens):
        batch = eng.q4_batch(pool, d_table, lens, begin, n_rows=3 * rows, page_tokens=PT, max_rows=rows, max_len=150 + 9 * rows)
        lens.add_(rows)
        o = eng.op_attention_q4(eng.op_append_q4(eng.op_gemm_w4(h, w["wqkv"]), 1, batch, rope), 1, batch, window=100, sinks=4)
        x = eng.op_gemm_w4_residual(o, w["wo"], h.float())
        x = eng.op_gemm_w4_residual(eng.op_gemm_w4_swiglu(x.bfloat16(), w["w_gate"], w["w_up"]), w["w_down"], x)
        return eng.op_sample(x, u, top_p=p)[0], x
    other, other_lens = pool.clone(), lens.clone()
    step(pool.clone(), lens.clone())
    second_pool, second_lens = pool.clone(), lens.clone()
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(pool, lens)
    with torch.cuda.graph(second):
        got2 = step(second_pool, second_lens)
    for seed in range(8):
        h.copy_(torch.from_numpy(np.random.default_rng(seed).standard_normal(h.shape).astype(np.float32)))
        u.uniform_()
        graph.replay()
        second.replay()
        tokens, x = got[0].clone(), got[1].clone()
        want = step(other, other_lens)
        torch.cuda.synchronize()
        assert torch.equal(tokens, want[0]) and torch.equal(x, want[1]) and torch.equal(pool, other) and torch.equal(lens, other_lens)
        assert torch.equal(got2[0], tokens) and torch.equal(second_pool, pool)


def test_batches_of_another_kind_are_refused():
    import torch
    import paper_2410_03065_amd as cake
    eng, pool, _, d_table, lens, begin, _, packed = decoding("bf16", 8, 2, 64, [150, 60, 1], 1)
    b4 = eng.q4_batch(pool, d_table, lens, begin, n_rows=3, page_tokens=PT)
    q, qkv = torch.zeros((8, 3, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((3, 12 * 64), device="cuda")
    b8 = eng.q8_batch(eng.new_q8_pool(9, PT), d_table, lens, begin, n_rows=3, page_tokens=PT)
    for call in (lambda: eng.op_attention_q8(q, 0, b4), lambda: eng.op_attention_q4(q, 0, b8), lambda: eng.op_append_q4(qkv, 0, b8, cake.rope(10000.0, 64)),
                 lambda: eng.op_append_q8(qkv, 0, b4, cake.rope(10000.0, 64))):
        with pytest.raises(cake.CakeError) as e:
            call()
        assert e.value.code == cake.E_INVAL
