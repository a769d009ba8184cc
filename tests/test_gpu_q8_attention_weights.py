"""How many bits of a weight times its value's scale cake_op_attention_q8 keeps: values that nearly cancel, whose difference is small
enough for a bfloat16 result to show them."""
import numpy as np
import pytest

from oracle import serving
from q8_helpers import Batch, engine

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,n_q,n_kv,hd,rows", [("bf16", 8, 2, 128, 1), ("bf16", 8, 8, 64, 1), ("bf16", 8, 2, 128, 8), ("bf16", 8, 2, 64, 8), ("bf16", 8, 2, 128, 20),
                                                   ("bf16", 8, 2, 128, 28), ("bf16", 8, 2, 128, 64), ("bf16", 4, 4, 64, 520), ("f32", 8, 2, 128, 3), ("f32", 4, 4, 64, 40)])
@pytest.mark.parametrize("block,length", [(1, 2), (4, 8), (1, 64), (16, 2048)])
def test_values_that_nearly_cancel(kind, n_q, n_kv, hd, rows, block, length):
    """Queries of zero weigh all keys alike, so a weight times its scale is the scale.  Codes are 127 in one half of the blocks and
    -127 in the other, whose scales are larger by 2^-9 to 2^-6.  A result is then off by half a step of its own and, of the sum of
    magnitudes, by what a weight loses: two bfloat16 terms 2^-16 (2^-8 of 2^-8), half precision 2^-11 (from 97 rows of a KV head on, heads
    of 64 from 512), three terms 2^-24; the few sums of float32 in between add (keys / 32 + 64) 2^-24."""
    import torch
    seqs = 6
    lens = [rows - 1 + length + i * 2 * block for i in range(seqs)]
    b = Batch(engine(n_q, n_kv, hd, kind), lens, [rows] * seqs, pt=64, block=block, seed=rows)
    rng = np.random.default_rng([rows, length])
    scales = b.pages.scales[:, 1]
    scales[:] = rng.uniform(1, 2, scales.shape[:2] + (1,)).astype(np.float32)
    sign = np.arange(scales.shape[2]) % 2
    scales *= np.where(sign == 1, 1 + 2.0 ** rng.uniform(-9, -6, scales.shape), 1).astype(np.float32)
    b.pages.codes[:, 1] = np.where(np.repeat(sign, block) == 1, -127, 127)[:, None]
    b.pool[0] = torch.from_numpy(b.pages.bytes())
    q = torch.zeros((n_q, b.rows, hd), dtype=b.eng.tdtype, device="cuda")
    got = b.eng.op_attention_q8(q, 0, b.q8).double().cpu().numpy().reshape(b.rows, n_q, hd)
    want, size, _, _ = serving.attention(b.pages, q.double().cpu().numpy(), b.table, b.lens, b.begin)
    group_rows = rows * n_q // n_kv
    many = kind == "bf16" and group_rows >= (97 if hd == 128 else 512)
    kept = 2.0 ** -24 if kind == "f32" else 2.0 ** -11 if many else 2.0 ** -16
    bound = (2.0 ** -24 if kind == "f32" else 2.0 ** -8) * np.abs(want) + size * (kept + (max(lens) / 32 + 64) * 2.0 ** -24)
    assert (np.abs(got - want) <= bound).all(), (np.abs(got - want) / bound).max()
