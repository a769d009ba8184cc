"""CPU tests of what the 8-bit batch calls decide on the host: page sizes, rotary descriptions, refusals that need no context."""
import ctypes

import numpy as np
import pytest

import synth_inputs as si
from oracle import serving
from oracle import store as ostore
import paper_2410_03065_amd as cake


def test_struct_sizes_match_the_header_layout():
    assert ctypes.sizeof(cake.Q8Batch) == 64
    assert ctypes.sizeof(cake.RopeDesc) == 48
    assert ctypes.sizeof(cake.Rope) == 528


@pytest.mark.parametrize("shape", [si.TINY, si.LLAMA3_8B, si.LLAMA2_70B])
@pytest.mark.parametrize("pt", [64, 256])
def test_pages_with_a_scale_per_token_have_the_size_of_a_layer_of_the_int8_store(shape, pt):
    lib = cake.load_library()
    image = lib.cake_store_image_bytes(ctypes.byref(cake.model_desc(shape)), pt, cake.STORE_INT8)
    assert cake.q8_page_bytes(shape, pt) * shape.n_layers == image
    for block in (4, 16, 64):
        pages = serving.Pages(1, shape.n_kv, pt, shape.head_dim, block)
        assert cake.q8_page_bytes(shape, pt, block) == pages.bytes().size


@pytest.mark.parametrize("pt,block", [(0, 1), (100, 1), (-64, 1), (64, 0), (64, 2), (64, 3), (64, 128), (64, -1)])
def test_pages_that_are_refused(pt, block):
    with pytest.raises(cake.CakeError):
        cake.q8_page_bytes(si.LLAMA3_8B, pt, block)


def test_scale_sections_off_16_bytes_are_refused():
    one = si.LLAMA3_8B.with_(n_q=8, n_kv=1)
    with pytest.raises(cake.CakeError):
        cake.q8_page_bytes(one, 64, 64)
    assert cake.q8_page_bytes(one, 256, 64) == 2 * (256 * 128 + 16)


@pytest.mark.parametrize("scaling", [None, ("linear", 4.0), ("bands", 8.0, 1.0, 4.0, 8192), ("ramp", 16.0, 4096, 32.0, 1.0), ("ramp", 1.0, 100, 32.0, 1.0)])
@pytest.mark.parametrize("theta,dim", [(10000.0, 64), (500000.0, 128), (10000.0, 48), (10000.0, 2), (1.5, 6)])
def test_rotary_frequencies(scaling, theta, dim):
    r = cake.rope(theta, dim, layout="halves", scaling=scaling)
    freq, magnitude = serving.rope_frequencies(theta, dim, scaling)
    np.testing.assert_allclose(np.array(r.freq[:dim // 2]), freq, rtol=1e-14)      # a few roundings in 64 bits
    assert not any(r.freq[dim // 2:])
    assert abs(r.magnitude - magnitude) < 1e-14 and r.rotary_dim == dim and r.layout == 1


@pytest.mark.parametrize("change", [dict(rotary_dim=0), dict(rotary_dim=3), dict(rotary_dim=130), dict(layout=2), dict(scaling=4), dict(theta=1.0),
                                    dict(theta=float("nan")), dict(theta=float("inf")), dict(factor=0.5), dict(factor=float("nan")), dict(low=0.0),
                                    dict(high=1.0), dict(original_tokens=0)])
def test_rotary_descriptions_that_are_refused(change):
    good = dict(theta=10000.0, factor=2.0, low=1.0, high=4.0, rotary_dim=64, layout=0, scaling=2, original_tokens=4096)
    out, lib = cake.Rope(), cake.load_library()
    assert lib.cake_rope_init(ctypes.byref(out), ctypes.byref(cake.RopeDesc(**good))) == cake.OK
    assert lib.cake_rope_init(ctypes.byref(out), ctypes.byref(cake.RopeDesc(**dict(good, **change)))) == cake.E_INVAL
    assert lib.cake_rope_init(None, ctypes.byref(cake.RopeDesc(**good))) == cake.E_INVAL


def test_calls_without_a_context_are_refused():
    lib = cake.load_library()
    assert lib.cake_op_append_q8(None, None, None, None, 0, None, None) == cake.E_INVAL
    assert lib.cake_op_attention_q8(None, None, None, 0, 0, 0, None) == cake.E_INVAL
    assert lib.cake_op_sample(None, None, 1, 1, 1, None, None, None, None, None, None, None) == cake.E_INVAL


def test_oracle_pages_are_the_int8_store_image():
    """The oracle's own two descriptions of the same bytes agree: a scale per token is the store's format."""
    rng = np.random.default_rng(3)
    n_kv, pt, hd = 2, 64, 64
    x = rng.standard_normal((2, 1, n_kv, pt, hd)).astype(np.float32)
    pages = serving.Pages(1, n_kv, pt, hd, 1).fill(x[0], 0).fill(x[1], 1)
    from oracle import transformer as otf
    cache = otf.KVCache(1, pt, n_kv, hd)
    cache.k[0], cache.v[0] = x[0, 0].transpose(1, 0, 2), x[1, 0].transpose(1, 0, 2)
    image = ostore.pack_store_int8(cache, pt)
    np.testing.assert_array_equal(np.asarray(image).reshape(1, -1).view(np.uint8), pages.bytes())
