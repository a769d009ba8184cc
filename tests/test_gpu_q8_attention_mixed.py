"""cake_op_attention_q8 over ragged batches that a launch is not sized for: a chunk beside single tokens, whose keys are divided by the
tiles that the batch can fill, and both sides of the rounds of undivided sequences."""
import pytest

from q8_helpers import Batch, engine
from test_gpu_q8_attention import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd,rows", [(128, 30), (128, 64), (128, 200), (64, 130)])        # groups of 4: tiles of 128 and 256 rows
@pytest.mark.parametrize("tokens", [1, 3, 20])
def test_a_chunk_beside_single_tokens(hd, rows, tokens):
    lens = [3000] + [2900 - 140 * i for i in range(tokens)]
    b = Batch(engine(8, 2, hd, "bf16"), lens, [rows] + [1] * tokens, pt=64, lead=2, tail=300, seed=rows)
    check(b)
    check(b, window=700, sinks=5)
    check(b, q8=b.describe(max_rows=0, max_len=0))


@pytest.mark.parametrize("kind,n_kv,hd", [("bf16", 8, 64), ("bf16", 8, 128), ("f32", 8, 64)])
@pytest.mark.parametrize("seqs", [31, 32, 33, 48, 64, 65])
@pytest.mark.parametrize("keys", [350, 1400])
def test_both_sides_of_the_rounds(kind, n_kv, hd, seqs, keys):
    lens = [keys - 5 * (i % 7) for i in range(seqs)]
    check(Batch(engine(n_kv, n_kv, hd, kind), lens, [1] * seqs, pt=64, block=16, seed=seqs))
