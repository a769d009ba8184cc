"""cake_op_attention_q8 where all of a row's scores are far below zero and a window hides the first keys that its tile reads: a row
that has seen nothing yet takes its reference from its first visible keys, however low they are."""
import numpy as np
import pytest

from oracle import serving
from q8_helpers import Batch, attention_bound, engine

pytestmark = pytest.mark.gpu
# groups of 4: (head size, tokens): 4, 20, 112 rows in a tile of 16, 32, 128; 256 in a tile of 256; 540 in tiles of 128
TILES = [(128, 1), (128, 5), (128, 28), (128, 64), (64, 1), (64, 135)]


def lens_of(rows, window):
    """The first key that a sequence's first row sees at several places of its 64, the last among them."""
    least = rows + window
    return [least + (place - least + rows + window - 1) % 64 for place in (63, 62, 40, 1, 0)]


def with_scores(b, level):
    """Keys whose score with a query of minus ones is -level[key] (level > 0): codes of 127, the scale sets it."""
    import torch
    hd = b.eng.shape.head_dim
    for s, pages in enumerate(b.table):
        for i, page in enumerate(pages):
            if page >= 0:
                b.pages.codes[page, 0] = 127
                b.pages.scales[page, 0] = (level[64 * i:64 * i + 64] / (127 * np.sqrt(hd))).astype(np.float32)
    b.pool[b.layer] = torch.from_numpy(b.pages.bytes())
    return torch.full((b.eng.shape.n_q, b.rows, hd), -1.0, dtype=b.eng.tdtype, device="cuda")


def check(b, q, window, sinks):
    s = b.eng.shape
    got = b.eng.op_attention_q8(q, b.layer, b.q8, window=window, sinks=sinks).double().cpu().numpy().reshape(b.rows, s.n_q, s.head_dim)
    want, size, mass, reach = serving.attention(b.pages, q.double().cpu().numpy(), b.table, b.lens, b.begin, window, sinks)
    bound = attention_bound(s.dtype, s.head_dim, want, size, mass, reach, int(b.lens.max()))
    assert np.isfinite(got).all() and (np.abs(got - want) <= bound).all(), np.nanmax(np.abs(got - want) / bound)


@pytest.mark.parametrize("hd,rows", TILES)
@pytest.mark.parametrize("window", [20, 100, 1000])      # one range of keys; two; several
@pytest.mark.parametrize("level", [100.0, 1000.0, 2e4])
def test_all_scores_equal_and_low(hd, rows, window, level):
    b = Batch(engine(8, 2, hd, "bf16"), lens_of(rows, window), [rows] * 5, pt=64)
    q = with_scores(b, np.full(64 * b.table.shape[1], level))
    check(b, q, window, 0)
    check(b, q, window, 3)


@pytest.mark.parametrize("kind,hd,rows", [("bf16",) + t for t in TILES] + [("f32", 128, 1), ("f32", 64, 40)])
@pytest.mark.parametrize("window", [20, 100])
def test_scores_of_every_depth(kind, hd, rows, window):
    """Each key at its own depth: references move up by hundreds, also from a first visible key far below the next."""
    b = Batch(engine(8, 2, hd, kind), lens_of(rows, window), [rows] * 5, pt=64, seed=rows)
    level = np.random.default_rng(rows).uniform(60, 700, 64 * b.table.shape[1])
    level[::7] *= 8
    q = with_scores(b, level)
    check(b, q, window, 0)
    check(b, q, window, 2)
