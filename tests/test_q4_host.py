"""CPU tests of what the calls in 4 bits decide on the host: page sizes, refusals that need no context or no library, the oracle's own bytes."""
import ctypes

import numpy as np
import pytest

import synth_inputs as si
from oracle import serving
from oracle import store as ostore
import paper_2410_03065_amd as cake


@pytest.mark.parametrize("shape", [si.TINY, si.LLAMA3_8B, si.LLAMA2_70B])
@pytest.mark.parametrize("pt", [64, 256])
def test_pages_with_a_scale_per_token_have_the_size_of_a_layer_of_the_int4_store(shape, pt):
    lib = cake.load_library()
    image = lib.cake_store_image_bytes(ctypes.byref(cake.model_desc(shape)), pt, cake.STORE_INT4)
    assert cake.q4_page_bytes(shape, pt) * shape.n_layers == image
    for block in (4, 16, 64):
        assert cake.q4_page_bytes(shape, pt, block) == serving.Pages(1, shape.n_kv, pt, shape.head_dim, block, bits=4).bytes().size


@pytest.mark.parametrize("pt,block", [(0, 1), (100, 1), (-64, 1), (64, 0), (64, 2), (64, 3), (64, 128), (64, -1)])
def test_pages_that_are_refused(pt, block):
    with pytest.raises(cake.CakeError):
        cake.q4_page_bytes(si.LLAMA3_8B, pt, block)


def test_scale_sections_off_16_bytes_are_refused():
    one = si.LLAMA3_8B.with_(n_q=8, n_kv=1)
    with pytest.raises(cake.CakeError):
        cake.q4_page_bytes(one, 64, 64)
    assert cake.q4_page_bytes(one, 256, 64) == 2 * (256 * 64 + 16)


def test_struct_sizes_match_the_header_layout():
    assert ctypes.sizeof(cake.W4) == 32


def test_calls_without_a_context_are_refused():
    lib = cake.load_library()
    assert lib.cake_op_append_q4(None, None, None, None, 0, None, None) == cake.E_INVAL
    assert lib.cake_op_attention_q4(None, None, None, 0, 0, 0, None) == cake.E_INVAL
    assert lib.cake_op_pack_w4(None, None, None, None, None, 1, 8, 32) == cake.E_INVAL
    assert lib.cake_op_gemm_w4(None, None, None, None, 1) == cake.E_INVAL
    assert lib.cake_op_gemm_w4_residual(None, None, None, None, 1) == cake.E_INVAL
    assert lib.cake_op_gemm_w4_swiglu(None, None, None, None, None, 1) == cake.E_INVAL


def engine_on(device, model=(2, 8, 128), kind="bf16"):
    eng = cake.Engine.__new__(cake.Engine)
    eng._dev_index, eng._q8_model = device, (*model, device)
    eng._q4_model, eng._w4_model = eng._q8_model + ("4 bits",), (kind, device)
    return eng


def test_batches_of_other_codes_are_refused_both_ways():
    eng, eight, four = engine_on(0), cake.Q8Batch(), cake.Q8Batch()
    eight.model, four.model = eng._q8_model, eng._q4_model
    assert eng._batch(eight, eng._q8_model) is eight and eng._batch(four, eng._q4_model) is four
    for batch, model in ((four, eng._q8_model), (eight, eng._q4_model)):
        with pytest.raises(cake.CakeError) as e:
            eng._batch(batch, model)
        assert e.value.code == cake.E_INVAL
    with pytest.raises(cake.CakeError):
        engine_on(1)._batch(four, engine_on(1)._q4_model)


def test_projections_of_another_type_or_device_are_refused():
    w = cake.W4()
    w.model = engine_on(0)._w4_model
    assert engine_on(0)._w4(w) is w
    for other in (engine_on(1), engine_on(0, kind="f32")):
        with pytest.raises(cake.CakeError) as e:
            other._w4(w)
        assert e.value.code == cake.E_INVAL


def test_oracle_pages_are_the_int4_store_image():
    """The oracle's own two descriptions of the same bytes agree: a scale per token is the store's format."""
    rng = np.random.default_rng(3)
    n_kv, pt, hd = 2, 64, 64
    x = rng.standard_normal((2, 1, n_kv, pt, hd)).astype(np.float32)
    pages = serving.Pages(1, n_kv, pt, hd, 1, bits=4).fill(x[0], 0).fill(x[1], 1)
    from oracle import transformer as otf
    cache = otf.KVCache(1, pt, n_kv, hd)
    cache.k[0], cache.v[0] = x[0, 0].transpose(1, 0, 2), x[1, 0].transpose(1, 0, 2)
    image = ostore.pack_store_int4(cache, pt)
    np.testing.assert_array_equal(np.asarray(image).reshape(1, -1).view(np.uint8), pages.bytes())
    again = serving.Pages(1, n_kv, pt, hd, 1, bits=4).take(pages.bytes())
    np.testing.assert_array_equal(again.codes, pages.codes)


def test_oracle_packs_a_row_by_hand():
    """Two groups of 32 and one of 8: scales 14 / 7, 0.7 / 7 and 0; halves to even; the first code of a byte in its low half."""
    w = np.zeros((1, 72), np.float32)
    w[0, :6] = [14, -14, 3, 5, -1, 9]               # / 2: 7 -7 1.5 2.5 -0.5 4.5
    w[0, 32] = 0.7
    raw, scales, values = serving.pack_w4(w, 32, "f32")
    assert raw.shape == (1, 48) and raw[0, :4].tolist() == [0x97, 0x22, 0x40, 0x00] and raw[0, 16] == 7
    np.testing.assert_array_equal(scales, np.array([[2, np.float32(0.7) / np.float32(7), 0]], np.float32))
    assert values[0, :6].tolist() == [14, -14, 4, 4, 0, 8] and (values[0, 33:] == 0).all()
    assert serving.round_to(np.float32([1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8]), "bf16").tolist() == [1.0, 1 + 2.0 ** -6]


@pytest.mark.parametrize("codes", [np.arange(-8, 8)])
def test_oracle_nibbles_there_and_back(codes):
    assert serving.one_each(serving.two_a_byte(codes)).tolist() == codes.tolist()
