"""Sizes and positions that the C ABI's 32 bits do not hold are refused by the binding: cut off, they would be others (2^32 + 5 a window of 5).
The tensors have no memory; nothing is called."""
import pytest

import synth_inputs as si
import paper_2410_03065_amd as cake
from test_q4_host import engine_on

FAR = 1 << 32


class Lib:
    def __getattr__(self, name):
        return lambda *a: pytest.fail("%s was called" % name)


def engine():
    import torch
    eng = engine_on(0)
    eng.torch, eng.tdtype, eng.dev, eng.lib, eng.shape = torch, torch.bfloat16, torch.device("meta"), Lib(), si.LLAMA3_8B
    eng._q8_model = eng._q4_model = eng._w4_model = "here"
    return eng


def refused(f):
    with pytest.raises(cake.CakeError, match="does not fit 32 bits") as e:
        f()
    assert e.value.code == cake.E_INVAL


def empty(*shape, dtype=None):
    import torch
    return torch.empty(shape, dtype=dtype or torch.bfloat16, device="meta")


def test_weights():
    import torch
    eng = engine()
    for n, k in ((1, FAR + 8), (FAR + 5, 8), (1, (1 << 31))):
        refused(lambda: eng.pack_w4(empty(n, k)))
        refused(lambda: eng.w4(empty(n, (k + 31) // 32 * 16, dtype=torch.uint8), empty(n, -(-k // 128)), k))


def test_rows():
    eng, w = engine(), cake.W4(None, None, 16, 8, 32)
    w.model = "here"
    for rows in (FAR, FAR + 5, 1 << 31):
        a = empty(rows, 8)
        refused(lambda: eng.op_gemm_w4(a, w))
        refused(lambda: eng.op_gemm_w4_residual(a, w, a))
        refused(lambda: eng.op_gemm_w4_swiglu(a, w, w))


@pytest.mark.parametrize("x", [FAR, FAR + 5, 1 << 31, -(1 << 31) - 1, -FAR])
def test_batch_calls(x):
    eng, b = engine(), cake.Q8Batch()
    b.model = "here"
    for op in (eng.op_attention_q8, eng.op_attention_q4):
        refused(lambda: op(None, 0, b, window=x))
        refused(lambda: op(None, 0, b, sinks=x))
        refused(lambda: op(None, x, b))
    for op in (eng.op_append_q8, eng.op_append_q4):
        refused(lambda: op(None, x, b, None))


@pytest.mark.parametrize("name", ["n_rows", "page_tokens", "scale_tokens", "max_rows", "max_len"])
def test_descriptions(name):
    import torch
    eng = engine()
    page = cake.q4_page_bytes(eng.shape, 64)
    pool, table = empty(eng.shape.n_layers, 3, page, dtype=torch.uint8), empty(2, 4, dtype=torch.int32)
    args = dict(dict(n_rows=1, page_tokens=64, scale_tokens=1, max_rows=0, max_len=0), **{name: FAR + {"page_tokens": 64, "scale_tokens": 1}.get(name, 5)})
    refused(lambda: eng.q4_batch(pool, table, table, table, **args))
