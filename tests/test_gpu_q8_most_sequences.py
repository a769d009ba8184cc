"""The batch calls over as many sequences as they take, and one more."""
import ctypes

import numpy as np
import pytest

from oracle import serving
from q8_helpers import Batch, attention_bound, engine

pytestmark = pytest.mark.gpu
MOST, KV = 1 << 22, 4


@pytest.mark.parametrize("kind,rows", [("bf16", 1), ("bf16", 40), ("bf16", 600), ("f32", 3)])      # tiles of 16 and 128 rows
@pytest.mark.parametrize("block", [1, 16])
def test_the_last_of_as_many_sequences_as_there_may_be(kind, rows, block):
    import torch
    import paper_2410_03065_amd as cake
    n = MOST // KV
    eng = engine(4, KV, 64, kind)
    one = Batch(eng, [rows + 70], [rows], block=block)
    table = torch.full((n, one.table.shape[1]), -1, dtype=torch.int32, device="cuda")
    table[-1] = one.d_table[0]
    lens, begin = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    lens[-1], begin[-1] = rows + 70, rows
    many = eng.q8_batch(one.pool, table, lens, begin, n_rows=rows, page_tokens=64, scale_tokens=block, max_rows=rows, max_len=rows + 70)
    rng = np.random.default_rng(rows)
    qkv = rng.standard_normal((rows, 12 * 64)).astype(np.float32)
    q = eng.op_append_q8(torch.from_numpy(qkv).cuda(), 0, many, cake.rope(10000.0, 64))
    freq, magnitude = serving.rope_frequencies(10000.0, 64)
    serving.append(one.pages, qkv, one.table, one.lens, one.begin, 4, freq, magnitude, "pairs")
    got = one.pages_now()
    np.testing.assert_array_equal(got.scales, one.pages.scales)
    np.testing.assert_array_equal(got.codes, one.pages.codes)
    out = eng.op_attention_q8(q, 0, many).double().cpu().numpy().reshape(rows, 4, 64)
    want, size, mass, reach = serving.attention(one.pages, q.double().cpu().numpy(), one.table, one.lens, one.begin)
    assert (np.abs(out - want) <= attention_bound(kind, 64, want, size, mass, reach, rows + 70)).all()


def test_more_sequences_are_refused():
    """Before a launch that would be too large: nothing of these arrays is read."""
    import torch
    import paper_2410_03065_amd as cake
    eng = engine(4, KV, 64, "bf16")
    b = Batch(eng, [70], [1])
    q, out, qkv = (torch.zeros(n, dtype=t, device="cuda") for n, t in ((4 * 64, torch.bfloat16), (4 * 64, torch.bfloat16), (12 * 64, torch.float32)))
    bad = cake.Q8Batch.from_buffer_copy(b.q8)
    bad.n_seqs = MOST // KV + 1
    assert eng.lib.cake_op_attention_q8(eng.ctx, q.data_ptr(), out.data_ptr(), 0, 0, 0, ctypes.byref(bad)) == cake.E_INVAL
    assert eng.lib.cake_op_append_q8(eng.ctx, qkv.data_ptr(), q.data_ptr(), None, 0, ctypes.byref(cake.rope(10000.0, 64)), ctypes.byref(bad)) == cake.E_INVAL
