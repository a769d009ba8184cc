"""cake_op_attention_q8 where it chooses between tiles of 16, 32, 128 and 256 rows (token, query head of the group): every side of the
choice, and in the large tiles what the device arrays may hold by mistake, hidden keys, NaN, hints, windows and graphs."""
import numpy as np
import pytest

from q8_helpers import Batch, engine
from test_gpu_q8_attention import check, run

pytestmark = pytest.mark.gpu
# groups of 4: (head size, tokens): 112 rows in a tile of 128, 256 in a tile of 256, 540 in tiles of 128
LARGE = [(128, 28), (128, 64), (64, 135)]


@pytest.mark.parametrize("hd,rows", [(128, r) for r in (4, 5, 8, 9, 24, 25, 32, 33, 44, 47, 48, 64, 65, 96, 128, 129)] + [(64, r) for r in (8, 9, 127, 128, 140)])
def test_both_sides_of_each_choice(hd, rows):
    b = Batch(engine(8, 2, hd, "bf16"), [rows + 200, rows], [rows, max(rows - 3, 1)], pt=64, block=16, lead=1, tail=2, seed=rows)
    check(b, seed=rows)
    check(b, window=90, sinks=3, seed=rows)


@pytest.mark.parametrize("hd,rows", LARGE)
def test_windows_and_sinks(hd, rows):
    for window, sinks in ((1, 0), (1, 1), (5, 0), (64, 40), (33, 500), (1000, 4), (2 ** 31 - 1, 2 ** 31 - 1)):
        check(Batch(engine(8, 2, hd, "bf16"), [rows, rows + 1, 300, 411], [rows] * 4, pt=64), window, sinks)


@pytest.mark.parametrize("hd,rows", LARGE)
@pytest.mark.parametrize("hints", [dict(max_rows=1), dict(max_len=1), dict(max_rows=0, max_len=0), dict(max_rows=500)])
def test_results_do_not_need_the_hints(hd, rows, hints):
    b = Batch(engine(8, 2, hd, "bf16"), [900, 90, 300], [rows, 1, rows - 3])
    check(b, q8=b.describe(**hints))


@pytest.mark.parametrize("hd,rows", LARGE)
def test_rows_without_tokens_and_sequences_without_rows(hd, rows):
    b = Batch(engine(8, 2, hd, "bf16"), [0, 70, 5, 0, 600], [2, 0, 9, 0, rows], lead=1, tail=2)
    got = check(b)
    assert (got[1:3] == 0).all() and (got[3:7] == 0).all() and (got[7] != 0).any()


@pytest.mark.parametrize("hd,rows", LARGE)
def test_memory_behind_the_last_token_and_hidden_keys_do_not_matter(hd, rows):
    import torch
    b = Batch(engine(8, 2, hd, "bf16"), [350, 100], [rows, 1], pt=64)
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


@pytest.mark.parametrize("hd,rows", LARGE)
def test_a_nan_is_seen_by_those_who_see_its_key(hd, rows):
    import torch
    b = Batch(engine(8, 2, hd, "bf16"), [300], [rows], pt=64)
    p = b.pages_now()
    for which, at in ((0, 280), (1, 290)):
        p.scales[b.table[0, at // 64], which, :, at % 64] = np.nan
    b.pool[0] = torch.from_numpy(p.bytes())
    got = run(b)[1].float().cpu().numpy()
    for i in range(rows):
        assert np.isnan(got[i]).all() if 300 - rows + i >= 280 else np.isfinite(got[i]).all()


@pytest.mark.parametrize("hd,rows", LARGE)
def test_pages_outside_the_pool_and_lengths_beyond_the_table_are_not_followed(hd, rows):
    import torch
    b = Batch(engine(8, 2, hd, "bf16"), [300, 290, 200], [rows] * 3, pt=64)
    want = run(b)[1].clone()
    for bad in (-1, b.n_pages, 2 ** 31 - 1, -2 ** 31):
        b.d_table[0, 1] = bad
        got = run(b)[1]
        assert torch.equal(got[rows:], want[rows:])
        sees = 300 - rows + np.arange(rows) >= 64
        assert torch.isnan(got[:rows][torch.from_numpy(sees).cuda()]).all()
    b.d_table[0, 1] = int(b.table[0, 1])
    for bad in (b.table.shape[1] * 64 + 1, 2 ** 31 - 1):
        b.d_lens[1] = bad
        got = run(b)[1]
        assert torch.isnan(got[rows:2 * rows]).all() and torch.equal(got[2 * rows:], want[2 * rows:])
    b.d_lens[1] = -5
    assert (run(b)[1][rows:2 * rows] == 0).all()


@pytest.mark.parametrize("hd,rows", LARGE)
def test_graph_replays_with_other_contents(hd, rows):
    import torch
    b = Batch(engine(8, 2, hd, "bf16"), [900, 290], [rows, rows - 1], pt=64)
    q, out = run(b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.eng.op_attention_q8(q, 0, b.q8, out=out)
    for seed in range(4):
        q.copy_(torch.from_numpy(np.random.default_rng(seed).standard_normal(q.shape).astype(np.float32)))
        b.d_lens[0] = 900 - 70 * seed
        out.zero_()
        graph.replay()
        got = out.clone()
        assert torch.equal(got, b.eng.op_attention_q8(q, 0, b.q8))


@pytest.mark.parametrize("kind,n_kv,hd,seqs", [("bf16", 8, 64, 64), ("bf16", 8, 64, 65), ("bf16", 2, 128, 300), ("f32", 4, 64, 140)])
def test_many_short_sequences(kind, n_kv, hd, seqs):
    """Short sequences undivided on eight waves, or, where there are many, on four."""
    lens = np.random.default_rng(seqs).integers(1, 260, seqs)
    lens[:3] = 0, 256, 257
    b = Batch(engine(2 * n_kv, n_kv, hd, kind), lens, [1] * seqs, pt=64, seed=seqs)
    check(b)
    check(b, window=40, sinks=3)


@pytest.mark.parametrize("keys", [250, 600, 700, 1400])
def test_few_sequences_on_both_sides_of_the_division(keys):
    for seqs in (1, 4, 16):
        check(Batch(engine(8, 2, 128, "bf16"), [keys] * (seqs - 1) + [keys - 7], [1] * seqs, pt=64, seed=keys))


@pytest.mark.parametrize("rows", [1, 30, 70])
def test_pages_of_an_odd_number_of_steps(rows):
    b = Batch(engine(8, 2, 128, "bf16"), [500, 193, 192, 70 + rows], [rows, rows, 1, rows], pt=192, block=16)
    check(b)
    check(b, window=100, sinks=5)
