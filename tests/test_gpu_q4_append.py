"""cake_op_append_q4 against the definition: codes and scales bit for bit, queries to their rounding; layouts, partial and
scaled rotation, blocks that already hold tokens, and what may not be written."""
import numpy as np
import pytest

from oracle import serving
from q8_helpers import Batch as AnyBatch, engine

pytestmark = pytest.mark.gpu


def Batch(*args, **kw):
    return AnyBatch(*args, bits=4, **kw)


def qkv_of(b, seed=0):
    s = b.eng.shape
    rng = np.random.default_rng([seed, 17])
    return (rng.standard_normal((b.rows, (s.n_q + 2 * s.n_kv) * s.head_dim)) * np.exp(0.5 * rng.standard_normal((b.rows, 1)))).astype(np.float32)


def check(b, qkv=None, theta=10000.0, dim=None, layout="pairs", scaling=None, q8=None):
    import torch
    import paper_2410_03065_amd as cake
    s = b.eng.shape
    dim = dim or s.head_dim
    qkv = qkv_of(b) if qkv is None else qkv
    rope = cake.rope(theta, dim, layout=layout, scaling=scaling)
    q = torch.full((s.n_q, b.rows, s.head_dim), 77.0, dtype=b.eng.tdtype, device="cuda")
    _, values = b.eng.op_append_q4(torch.from_numpy(qkv).cuda(), b.layer, q8 or b.q8, rope, q=q, want_values=True)
    q, values = q.double().cpu().numpy(), values.double().cpu().numpy()
    freq, magnitude = serving.rope_frequencies(theta, dim, scaling)
    want_q, want_v = serving.append(b.pages, qkv, b.table, b.lens, b.begin, s.n_q, freq, magnitude, layout)
    got = b.pages_now()
    np.testing.assert_array_equal(got.scales, b.pages.scales)
    seen = ~np.isnan(np.repeat(got.scales, b.block, axis=3))[..., None]       # codes under a NaN scale mean nothing
    np.testing.assert_array_equal(np.where(seen, got.codes, 0), np.where(seen, b.pages.codes, 0))
    # half a step of the result's type; float32: and the 64-bit arithmetic before it
    half = 2.0 ** -8 if s.dtype == "bf16" else 2.0 ** -24
    nobody = np.isnan(want_q)
    assert (q[nobody] == 77.0).all()
    live = ~nobody.all(axis=(0, 2))
    assert (np.abs(q - want_q)[~nobody] <= (half * np.abs(want_q) + 2.0 ** -24 * np.abs(want_q) + 1e-9)[~nobody]).all()
    np.testing.assert_array_equal(np.isnan(values[live]), np.isnan(want_v[live]))
    ok = live[:, None, None] & ~np.isnan(want_v)
    assert (np.abs(values - want_v)[ok] <= (half * np.abs(want_v) + 1e-40)[ok]).all()
    return q, values


HEADS = [("bf16", 8, 2, 128), ("f32", 4, 4, 64), ("bf16", 12, 4, 64), ("f32", 10, 2, 128), ("bf16", 16, 1, 128)]


@pytest.mark.parametrize("kind,n_q,n_kv,hd", HEADS)
@pytest.mark.parametrize("block", [1, 4, 16, 64])
@pytest.mark.parametrize("layout", ["pairs", "halves"])
def test_ragged_batches(kind, n_q, n_kv, hd, block, layout):
    lens, new = [1, 64, 65, 130, 200, 77, 16, 33], [1, 64, 1, 3, 150, 0, 15, 33]
    check(Batch(engine(n_q, n_kv, hd, kind), lens, new, pt=256 if block == 64 else 64, block=block, lead=2, tail=3, seed=block), layout=layout)


@pytest.mark.parametrize("dim", [2, 6, 16, 48, 50, 64])
@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("hd", [64, 128])
def test_part_of_the_head(dim, layout, hd):
    check(Batch(engine(4, 2, hd, "f32"), [40, 300], [5, 33], block=4), dim=dim, layout=layout)


@pytest.mark.parametrize("scaling", [("linear", 4.0), ("bands", 8.0, 1.0, 4.0, 8192), ("ramp", 16.0, 4096, 32.0, 1.0)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_scaled_rotation_at_far_positions(scaling, kind):
    b = Batch(engine(4, 2, 128, kind), [100000, 70001], [3, 20], pt=256, block=16)
    check(b, theta=500000.0, scaling=scaling, layout="halves")
    check(Batch(engine(4, 2, 64, kind), [131071], [2], pt=256), scaling=scaling)


@pytest.mark.parametrize("block", [1, 16, 64])
def test_token_by_token_equals_its_own_definition(block):
    """A block filled by many calls: every step's codes and scales, older codes moved to a larger scale among them."""
    eng = engine(4, 4, 64, "bf16")
    b = Batch(eng, [61, 5], [1, 1], block=block)
    rng = np.random.default_rng(8)
    for step in range(12):
        b.lens = b.lens + 1
        b.d_lens.add_(1)
        check(b, qkv=(rng.standard_normal((2, 12 * 64)) * 1.3 ** step).astype(np.float32))


@pytest.mark.parametrize("block", [1, 8])
def test_zeros_infinities_and_nan(block):
    b = Batch(engine(4, 2, 64, "f32"), [70, 40, 64], [10, 3, 1], block=block)
    x = qkv_of(b).reshape(14, 8, 64)
    x[0, 4:] = 0
    x[3, 4, 5] = np.inf
    x[6, 7, 9] = np.nan
    x[8, 6, 0] = -np.inf
    x[10:13] = 0                       # a whole sequence of zeros
    x[13, 4:] = 1e-44                  # smallest numbers
    with np.errstate(invalid="ignore"):
        check(b, qkv=x.reshape(14, -1))


def test_rows_without_tokens_bad_pages_and_lengths_beyond_the_table_write_nothing():
    import torch
    b = Batch(engine(4, 2, 64, "bf16"), [3, 100, 90, 0], [5, 30, 2, 2], block=4)
    b.table[1, 1] = b.n_pages
    b.d_table[1, 1] = b.n_pages
    check(b)
    for bad in (-1, 2 ** 31 - 1, -2 ** 31):
        b.table[1, 1] = bad
        b.d_table[1, 1] = bad
        check(b)
    before = b.pool.clone()
    b.lens[:], b.begin[:] = [2 ** 31 - 1, 2 ** 30, 64 * b.table.shape[1] + 2, 2 ** 31 - 1], [0, 5, 35, 37, 39]
    b.d_lens.copy_(torch.from_numpy(b.lens.astype(np.int32)))
    import paper_2410_03065_amd as cake
    _, values = b.eng.op_append_q4(torch.from_numpy(qkv_of(b)).cuda(), 0, b.q8, cake.rope(10000.0, 64), want_values=True)
    assert torch.isnan(values).all() and torch.equal(b.pool, before)


@pytest.mark.parametrize("hints", [dict(max_rows=1), dict(max_rows=0), dict(max_rows=300)])
def test_results_do_not_need_the_hints(hints):
    b = Batch(engine(8, 2, 128, "bf16"), [300, 90], [200, 1], block=16)
    check(b, q8=b.describe(**hints))


def test_another_layer_leaves_the_others():
    import torch
    b = Batch(engine(8, 2, 128, "bf16", n_layers=3), [100, 65], [1, 2], layers=3, layer=1)
    b.pool[0], b.pool[2] = 9, 9
    check(b)
    assert (b.pool[0] == 9).all() and (b.pool[2] == 9).all()


def test_pages_past_32_bits():
    """A page whose bytes begin beyond 2^32: append there and attend to it."""
    import torch
    eng = engine(8, 8, 128, "bf16", n_layers=1)
    import paper_2410_03065_amd as cake
    page = cake.q4_page_bytes(eng.shape, 256)
    n = (1 << 32) // page + 40
    pool = torch.zeros((1, n, page), dtype=torch.uint8, device="cuda")
    b = Batch(eng, [300, 77], [2, 1], pt=256)
    used = b.table.max() + 1
    shift = n - used
    pool[0, shift:] = b.pool[0, :used]
    small = b.q8
    b_table = b.d_table + shift
    far = eng.q4_batch(pool, b_table, b.d_lens, b.d_begin, n_rows=b.rows, page_tokens=256)
    rope = cake.rope(10000.0, 128)
    x = torch.from_numpy(qkv_of(b)).cuda()
    q1, q2 = eng.op_append_q4(x, 0, small, rope), eng.op_append_q4(x, 0, far, rope)
    assert torch.equal(q1, q2) and torch.equal(pool[0, shift:], b.pool[0, :used])
    same_hints = b.describe(max_rows=far.max_rows, max_len=far.max_len)      # they choose the ranges, and those the order of the sums
    assert torch.equal(eng.op_attention_q4(q1, 0, same_hints), eng.op_attention_q4(q1, 0, far))


def test_graph_replays():
    import torch
    import paper_2410_03065_amd as cake
    eng = engine(8, 2, 128, "bf16")
    rope = cake.rope(10000.0, 128)
    b, c = (Batch(eng, [100, 65, 31], [1, 2, 1], block=4, seed=1) for _ in range(2))
    x = torch.from_numpy(qkv_of(b)).cuda()
    q = torch.empty((8, 4, 128), dtype=torch.bfloat16, device="cuda")
    before = b.pool.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eng.op_append_q4(x, 0, b.q8, rope, q=q)
    assert torch.equal(b.pool, before)
    for step in range(4):
        x.copy_(torch.from_numpy(qkv_of(b, step)))
        graph.replay()
        want = eng.op_append_q4(x, 0, c.q8, rope)
        assert torch.equal(q, want) and torch.equal(b.pool, c.pool)
        b.d_lens.add_(1), c.d_lens.add_(1)


def test_refusals():
    import ctypes
    import torch
    import paper_2410_03065_amd as cake
    eng = engine(8, 2, 64, "bf16")
    b = Batch(eng, [100, 65], [1, 2])
    x, rope = torch.from_numpy(qkv_of(b)).cuda(), cake.rope(10000.0, 64)
    q = eng.op_append_q4(x, 0, b.q8, rope)
    with pytest.raises(cake.CakeError):
        eng.op_append_q4(x, 0, b.q8, cake.rope(10000.0, 128))       # more than the head has
    for bad in (x.double(), x[:, ::2], x[:2], x.cpu()):
        with pytest.raises(cake.CakeError):
            eng.op_append_q4(bad, 0, b.q8, rope)
    with pytest.raises(cake.CakeError):
        eng.op_append_q4(x, 0, b.q8, rope, q=q.float())
    for layer in (-1, 1):
        with pytest.raises(cake.CakeError):
            eng.op_append_q4(x, layer, b.q8, rope)
    call = lambda *a: eng.lib.cake_op_append_q4(eng.ctx, *a)  # noqa: E731
    r, d = ctypes.byref(rope), ctypes.byref(b.q8)
    for args in ((None, q.data_ptr(), None, 0, r, d), (x.data_ptr(), None, None, 0, r, d), (x.data_ptr() + 4, q.data_ptr(), None, 0, r, d),
                 (x.data_ptr(), q.data_ptr() + 2, None, 0, r, d), (x.data_ptr(), q.data_ptr(), q.data_ptr() + 8, 0, r, d),
                 (x.data_ptr(), q.data_ptr(), None, 0, None, d), (x.data_ptr(), q.data_ptr(), None, 0, r, None)):
        assert call(*args) == cake.E_INVAL
    for field, value in (("rotary_dim", 0), ("rotary_dim", 3), ("layout", 2)):
        bad = cake.Rope.from_buffer_copy(rope)
        setattr(bad, field, value)
        assert call(x.data_ptr(), q.data_ptr(), None, 0, ctypes.byref(bad), d) == cake.E_INVAL


@pytest.mark.parametrize("block", [1, 16, 64])
def test_pages_of_192_tokens(block):
    check(Batch(engine(8, 4, 64, "bf16"), [500, 193, 192, 64], [300, 1, 2, 64], pt=192, block=block))
