"""cake_op_append_q8's scales and codes are correctly rounded float32 quotients: values at and beside the middle between two codes, where a scale
that is one unit off (largest magnitude times 1 / 127) gives another code."""
import numpy as np
import pytest

from q8_helpers import Batch, engine

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("block", [1, 16])
def test_values_between_two_codes(kind, hd, block):
    import torch
    import paper_2410_03065_amd as cake
    n_q, n_kv, rows = 4, 2, 512
    eng = engine(n_q, n_kv, hd, kind)
    b = Batch(eng, [rows], [rows], block=block)
    rng = np.random.default_rng([hd, block])
    most = rng.uniform(0.5, 2, (rows // block, 1, 2 * n_kv)).astype(np.float32)
    scale = most / np.float32(127)
    assert (scale != most * (np.float32(1) / np.float32(127))).any()
    code = rng.integers(-126, 126, (rows // block, block, 2 * n_kv, hd))
    x = ((code + np.float32(0.5)) * scale[..., None]).astype(np.float32)
    x = np.where(rng.random(x.shape) < 0.5, x, np.nextafter(x, np.where(rng.random(x.shape) < 0.5, np.float32(9), np.float32(-9)))).astype(np.float32)
    x[:, 0, :, 0] = most[:, 0]                                   # the block's largest magnitude
    qkv = np.concatenate([np.zeros((rows, n_q, hd), np.float32), x.reshape(rows, 2 * n_kv, hd)], axis=1)
    still = cake.rope(10000.0, 2)
    still.freq[0] = 0.0                                          # an angle of 0 leaves every key as it is
    _, values = eng.op_append_q8(torch.from_numpy(qkv.reshape(rows, -1)).cuda(), 0, b.q8, still, want_values=True)
    want = np.clip(np.rint(x / scale[..., None]), -127, 127).astype(np.float32)
    got = b.pages_now()
    codes = got.codes[b.table[0, :rows // 64]].transpose(0, 3, 1, 2, 4).reshape(rows // block, block, 2 * n_kv, hd)
    scales = got.scales[b.table[0, :rows // 64]].transpose(0, 3, 1, 2).reshape(rows // block, 1, 2 * n_kv)
    np.testing.assert_array_equal(scales, scale)
    np.testing.assert_array_equal(codes, want)
    stands = torch.from_numpy((want * scale[..., None]).reshape(rows, 2 * n_kv, hd)).to(eng.tdtype)
    assert torch.equal(values.cpu(), stands)
