"""cake_op_attention_q8 against the definition in 64 bits: head layouts and sizes, ragged batches, lengths from none to many
pages, windows and sinks, scale blocks, rows that see nothing, what the device arrays may hold by mistake, streams and graphs."""
import numpy as np
import pytest

from oracle import serving
from q8_helpers import Batch, attention_bound, engine

pytestmark = pytest.mark.gpu


def run(b, window=0, sinks=0, seed=0, q8=None, out=None):
    import torch
    s = b.eng.shape
    q = torch.from_numpy((np.random.default_rng([seed, 5]).standard_normal((s.n_q, b.rows, s.head_dim)) * 1.5).astype(np.float32)).cuda().to(b.eng.tdtype)
    got = b.eng.op_attention_q8(q, b.layer, q8 or b.q8, window=window, sinks=sinks, out=out)
    return q, got


def check(b, window=0, sinks=0, seed=0, q8=None):
    import torch
    s = b.eng.shape
    out = torch.full((b.rows, s.n_q * s.head_dim), 77.0, dtype=b.eng.tdtype, device="cuda")
    q, got = run(b, window, sinks, seed, q8, out)
    got = got.double().cpu().numpy().reshape(b.rows, s.n_q, s.head_dim)
    want, size, mass, reach = serving.attention(b.pages, q.double().cpu().numpy(), b.table, b.lens, b.begin, window, sinks)
    nobody = np.isnan(want)
    assert (got[nobody] == 77.0).all()
    bound = attention_bound(s.dtype, s.head_dim, want, size, mass, reach, int(max(b.lens.max(), 1)))
    off = np.abs(got - want)[~nobody]
    assert np.isfinite(got).all() and (off <= bound[~nobody]).all(), (off / bound[~nobody]).max()
    return got


HEADS = [("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("bf16", 4, 4, 128), ("f32", 4, 2, 64), ("f32", 4, 1, 128), ("bf16", 16, 1, 64), ("bf16", 24, 1, 128),
         ("bf16", 15, 3, 128)]


@pytest.mark.parametrize("kind,n_q,n_kv,hd", HEADS)
@pytest.mark.parametrize("block", [1, 4, 16])
def test_single_tokens(kind, n_q, n_kv, hd, block):
    lens = [1, 2, 31, 32, 33, 63, 64, 65, 127, 129, 500]
    check(Batch(engine(n_q, n_kv, hd, kind), lens, [1] * len(lens), block=block, seed=block))


@pytest.mark.parametrize("kind,n_q,n_kv,hd", HEADS)
def test_rows_of_prompts_and_single_tokens_mixed(kind, n_q, n_kv, hd):
    check(Batch(engine(n_q, n_kv, hd, kind), [200, 70, 1, 130, 64, 333], [7, 70, 1, 33, 1, 150], pt=128, block=4, lead=3, tail=5))


@pytest.mark.parametrize("kind,n_q,n_kv,hd", [HEADS[0], HEADS[3], ("bf16", 8, 2, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 0), (32, 2), (64, 40), (100, 64), (33, 500), (1000, 4), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("rows", [1, 3, 90])
def test_windows_and_sinks(kind, n_q, n_kv, hd, window, sinks, rows):
    lens = [rows, rows + 1, 300, 411]
    check(Batch(engine(n_q, n_kv, hd, kind), lens, [rows] * 4, pt=64), window, sinks)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_sequences_without_rows_or_tokens_and_rows_without_tokens(kind):
    b = Batch(engine(8, 2, 128, kind), [0, 70, 5, 0, 90], [2, 0, 9, 0, 1], lead=1, tail=2)
    got = check(b)
    assert (got[1:3] == 0).all()                         # an empty sequence's rows
    assert (got[3:7] == 0).all() and (got[7] != 0).any()   # nine rows of five tokens: the first four see nothing


def test_long_sequences_in_many_ranges():
    b = Batch(engine(8, 2, 128, "bf16"), [9000, 40, 20011], [1, 1, 1], pt=256, block=64)
    check(b)
    b = Batch(engine(4, 4, 64, "f32"), [9001, 6100], [2, 1], pt=64)
    check(b)
    check(b, window=3000, sinks=100)


@pytest.mark.parametrize("rows,length", [(128, 128), (300, 301), (257, 2000), (64, 5000)])
@pytest.mark.parametrize("hd,n_q,n_kv", [(128, 8, 2), (64, 4, 4), (128, 10, 2)])
def test_prompt_chunks(rows, length, hd, n_q, n_kv):
    check(Batch(engine(n_q, n_kv, hd, "bf16"), [length, 130], [rows, 65], pt=64, block=16), seed=rows)
    check(Batch(engine(n_q, n_kv, hd, "bf16"), [length], [rows], pt=256), window=200, sinks=5)


@pytest.mark.parametrize("hints", [dict(max_rows=1), dict(max_rows=1, max_len=1), dict(max_rows=0, max_len=0), dict(max_len=64), dict(max_rows=500)])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_results_do_not_need_the_hints(hints, kind):
    b = Batch(engine(8, 2, 128, kind), [700, 90, 300], [80, 1, 40])
    check(b, q8=b.describe(**hints))
    check(b, window=100, sinks=3, q8=b.describe(**hints))


def test_another_layer():
    b = Batch(engine(8, 2, 128, "bf16", n_layers=3), [100, 65], [1, 2], layers=3, layer=2)
    check(b)


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_memory_behind_the_last_token_and_hidden_keys_do_not_matter(rows, kind):
    import torch
    b = Batch(engine(8, 2, 128, kind), [150, 100], [rows, 1], pt=64)
    want = run(b, 40, 2)[1].clone()
    p = b.pages_now()
    for s, n in enumerate(b.lens):
        last = b.table[s, n // 64]
        p.scales[last, :, :, n % 64:] = np.nan
        p.codes[last, :, :, n % 64:] = -128
        for j in range(2, n - int(b.new[s]) - 40 + 1):
            p.scales[b.table[s, j // 64], :, :, j % 64] = np.inf
    b.pool[0] = torch.from_numpy(p.bytes())
    assert torch.equal(run(b, 40, 2)[1], want)


@pytest.mark.parametrize("rows", [1, 40])
def test_a_nan_is_seen_by_those_who_see_its_key(rows):
    import torch
    b = Batch(engine(4, 2, 64, "bf16"), [300], [rows], pt=64)
    p = b.pages_now()
    for which, at in ((0, 280), (1, 290)):
        p.scales[b.table[0, at // 64], which, :, at % 64] = np.nan
    b.pool[0] = torch.from_numpy(p.bytes())
    got = run(b)[1].float().cpu().numpy()
    for i in range(rows):
        pos = 300 - rows + i
        assert np.isnan(got[i]).all() if pos >= 280 else np.isfinite(got[i]).all()


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_pages_outside_the_pool_and_lengths_beyond_the_table_are_not_followed(rows, kind):
    import torch
    b = Batch(engine(8, 2, 128, kind), [300, 290, 100], [rows] * 3, pt=64)
    want = run(b)[1].clone()
    for bad in (-1, b.n_pages, 2 ** 31 - 1, -2 ** 31):
        b.d_table[0, 1] = bad
        got = run(b)[1]
        assert torch.isnan(got[:rows]).all() and torch.equal(got[rows:], want[rows:])
    b.d_table[0, 1] = int(b.table[0, 1])
    for bad in (b.table.shape[1] * 64 + 1, 2 ** 31 - 1):
        b.d_lens[1] = bad
        got = run(b)[1]
        assert torch.isnan(got[rows:2 * rows]).all() and torch.equal(got[2 * rows:], want[2 * rows:])
    b.d_lens[1] = -5
    assert (run(b)[1][rows:2 * rows] == 0).all()


def test_scores_far_apart_and_equal():
    """Weights that vanish beside the largest, and a long run of equal ones."""
    import torch
    b = Batch(engine(4, 4, 64, "bf16"), [5000, 700], [1, 1], pt=64)
    s = b.eng.shape
    q = torch.zeros((4, 2, 64), device="cuda", dtype=torch.bfloat16)
    q[:, 1] = 60.0
    got = b.eng.op_attention_q8(q, 0, b.q8).double().cpu().numpy().reshape(2, 4, 64)
    want, size, mass, reach = serving.attention(b.pages, q.double().cpu().numpy(), b.table, b.lens, b.begin)
    assert (np.abs(got - want) <= attention_bound("bf16", s.head_dim, want, size, mass, reach, 5000)).all()


def test_scales_of_very_different_size():
    """Values whose scales change by many orders within a sequence, in both directions."""
    import torch
    for order in (1, -1):
        b = Batch(engine(8, 2, 128, "bf16"), [700, 700], [1, 200], pt=64)
        factor = np.exp(np.linspace(-60, 60, 64 * b.table.shape[1]))[::order].astype(np.float32)
        for s in range(2):
            for i, page in enumerate(b.table[s]):
                if page >= 0:
                    b.pages.scales[page, 1] *= factor[64 * i:64 * i + 64]
        b.pool[0] = torch.from_numpy(b.pages.bytes())
        check(b)


def test_the_same_result_in_any_batch_and_again():
    import torch
    eng = engine(8, 2, 128, "bf16")
    b = Batch(eng, [700, 90, 301], [2, 1, 60])
    first = run(b)[1].clone()
    for _ in range(3):
        assert torch.equal(run(b)[1], first)


def test_graph_replays_with_other_contents_beside_eager_calls():
    import torch
    eng = engine(8, 2, 128, "bf16")
    b = Batch(eng, [2000, 90, 301], [1, 1, 1])
    c = Batch(eng, [64, 640, 1000], [3, 1, 40], seed=4)
    q, out = run(b)
    other = run(c)[1].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eng.op_attention_q8(q, 0, b.q8, out=out)
    for lens in ([2000, 90, 301], [1, 64, 65], [1999, 17, 300]):
        b.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        assert torch.equal(run(c)[1], other)
        graph.replay()
        got = out.clone()
        want = eng.op_attention_q8(q, 0, b.q8)
        assert torch.equal(got, want)


def test_two_graphs_of_one_context_in_turn():
    import torch
    eng = engine(8, 2, 128, "bf16")
    made = []
    for seed, lens in ((1, [3000, 70]), (2, [100, 2500])):
        b = Batch(eng, lens, [1, 1], seed=seed)
        q, out = run(b, seed=seed)
        want = out.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            eng.op_attention_q8(q, 0, b.q8, out=out)
        made.append((graph, out, want, b, q))
    for _ in range(3):
        for graph, out, want, _, _ in made:
            out.zero_()
            graph.replay()
            assert torch.equal(out, want)


def test_on_another_stream_and_on_the_callers_stream():
    import torch
    b = Batch(engine(8, 2, 128, "bf16"), [900, 90], [1, 20])
    want = run(b)[1].clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.zeros(1 << 26, device="cuda")
        for _ in range(10):
            big.add_(1)                      # keeps this stream busy: the operands below are late
        q, got = run(b)
        got = got + 0
    side.synchronize()
    assert torch.equal(got, want)
    own = engine(8, 2, 128, "bf16", compute_stream=torch.cuda.current_stream())
    assert own.compute_stream.cuda_stream == torch.cuda.current_stream().cuda_stream
    b2 = Batch(own, [900, 90], [1, 20])
    assert torch.equal(run(b2)[1], want)


def test_refusals():
    import torch
    import paper_2410_03065_amd as cake
    eng = engine(8, 2, 128, "bf16")
    b = Batch(eng, [100, 65], [1, 2])
    q, out = run(b)

    def refused(f):
        with pytest.raises(cake.CakeError) as e:
            f()
        assert e.value.code == cake.E_INVAL
    refused(lambda: eng.op_attention_q8(q, 1, b.q8))
    refused(lambda: eng.op_attention_q8(q, -1, b.q8))
    refused(lambda: eng.op_attention_q8(q, 0, b.q8, window=-1))
    refused(lambda: eng.op_attention_q8(q, 0, b.q8, sinks=-1))
    refused(lambda: eng.op_attention_q8(q.float(), 0, b.q8))
    refused(lambda: eng.op_attention_q8(q.transpose(0, 1), 0, b.q8))
    refused(lambda: eng.op_attention_q8(q[:, :2], 0, b.q8))
    refused(lambda: eng.op_attention_q8(q.cpu(), 0, b.q8))
    refused(lambda: b.describe(page_tokens=96))
    refused(lambda: b.describe(scale_tokens=3))
    refused(lambda: eng.q8_batch(b.pool[:, :, :-1].contiguous(), b.d_table, b.d_lens, b.d_begin, n_rows=3, page_tokens=64))
    refused(lambda: eng.q8_batch(b.pool, b.d_table.long(), b.d_lens, b.d_begin, n_rows=3, page_tokens=64))
    refused(lambda: eng.q8_batch(b.pool, b.d_table, b.d_lens[:1], b.d_begin, n_rows=3, page_tokens=64))
    import ctypes
    for field, value in (("n_seqs", -1), ("n_rows", -1), ("pages_per_seq", 0), ("pages_per_seq", 2 ** 31 - 1), ("n_physical_pages", 0), ("max_rows", -1),
                         ("max_len", -1), ("pool", None), ("pool", b.pool.data_ptr() + 8), ("seq_len", None), ("scale_tokens", 128), ("page_tokens", 32)):
        bad = cake.Q8Batch.from_buffer_copy(b.q8)
        setattr(bad, field, value)
        assert eng.lib.cake_op_attention_q8(eng.ctx, q.data_ptr(), out.data_ptr(), 0, 0, 0, ctypes.byref(bad)) == cake.E_INVAL, field
    for args in ((None, out.data_ptr()), (q.data_ptr(), None), (q.data_ptr() + 2, out.data_ptr()), (q.data_ptr(), out.data_ptr() + 8)):
        assert eng.lib.cake_op_attention_q8(eng.ctx, *args, 0, 0, 0, ctypes.byref(b.q8)) == cake.E_INVAL
    assert eng.lib.cake_op_attention_q8(eng.ctx, q.data_ptr(), out.data_ptr(), 0, 0, 0, None) == cake.E_INVAL


def test_batches_of_nothing():
    import torch
    eng = engine(8, 2, 128, "bf16")
    b = Batch(eng, [100], [1])
    q = torch.empty((8, 0, 128), dtype=torch.bfloat16, device="cuda")
    assert eng.op_attention_q8(q, 0, b.describe(n_rows=0)).numel() == 0
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    q8 = eng.q8_batch(b.pool, b.d_table[:0].contiguous(), none[:0].contiguous(), none, n_rows=2, page_tokens=64)
    out = torch.full((2, 1024), 5.0, dtype=torch.bfloat16, device="cuda")
    eng.op_attention_q8(torch.zeros((8, 2, 128), dtype=torch.bfloat16, device="cuda"), 0, q8, out=out)
    assert (out == 5).all()
