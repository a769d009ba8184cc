"""What the tests of the batch calls share: a small engine and a ragged batch with scattered pages of 8 (or 4) bits."""
import numpy as np

import synth_inputs as si
from oracle import serving


def engine(n_q, n_kv, hd, kind, **kw):
    import paper_2410_03065_amd as cake
    shape = si.ModelShape("q8", kw.pop("n_layers", 1), 64, n_q, n_kv, hd, 64, 64, kind)
    return cake.Engine(shape, None, max_tokens=256, max_chunk=256, page_tokens=64, **kw)


class Batch:
    """Sequences of `lens` tokens of which the last `new` are rows of the batch; `lead` rows before and `tail` rows behind
    belong to nobody.  The pool holds random values in every page."""

    def __init__(self, eng, lens, new, pt=64, block=1, lead=0, tail=0, seed=0, extra_pages=2, layers=1, layer=0, bits=8):
        import torch
        s, rng = eng.shape, np.random.default_rng([seed, 11])
        self.eng, self.lens, self.layer, self.bits = eng, np.asarray(lens), layer, bits
        self.begin = lead + np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
        self.rows = int(self.begin[-1]) + tail
        per = np.maximum(-(-self.lens // pt), 0)
        width, used = int(max(per.max(), 1)) + 1, int(per.sum())
        self.n_pages = used + extra_pages
        order = rng.permutation(self.n_pages)[:used]
        self.table = np.full((len(lens), width), -7, np.int32)
        at = 0
        for i, n in enumerate(per):
            self.table[i, :n] = order[at:at + n]
            at += n
        dims = (self.n_pages, s.n_kv, pt, s.head_dim)
        self.pages = serving.Pages(self.n_pages, s.n_kv, pt, s.head_dim, block, bits)
        for which in (0, 1):
            self.pages.fill(rng.standard_normal(dims) * np.exp(0.5 * rng.standard_normal(dims[:3] + (1,))), which)
        self.pool = torch.zeros((layers, self.n_pages, self.pages.bytes().shape[1]), dtype=torch.uint8, device="cuda")
        self.pool[layer] = torch.from_numpy(self.pages.bytes())
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
        self.d_table, self.d_lens, self.d_begin = i32(self.table), i32(self.lens), i32(self.begin)
        self.pt, self.block, self.new = pt, block, np.asarray(new)
        self.q8 = self.describe()

    def describe(self, **kw):
        return (self.eng.q8_batch if self.bits == 8 else self.eng.q4_batch)(self.pool, self.d_table, self.d_lens, self.d_begin, **dict(dict(
            n_rows=self.rows, page_tokens=self.pt, scale_tokens=self.block, max_rows=int(self.new.max()), max_len=int(self.lens.max())), **kw))

    def pages_now(self):
        s = self.eng.shape
        return serving.Pages(self.n_pages, s.n_kv, self.pt, s.head_dim, self.block, self.bits).take(self.pool[self.layer].cpu().numpy())


def attention_bound(kind, hd, want, size, mass, reach, most_keys):
    """How far an output may be from the exact one.  A score is a float32 sum of head_dim exact products, times a scale: off
    by at most (hd + 8) 2^-24 of the sum of magnitudes, which changes a weight by a factor e^x.  bf16: weight times scale keeps 11
    bits (off by half a step, 2^-11 of it), but no finer than half a step of 2^-24 in units of which the scale is 2^E and the row's
    largest weight 2^6 or more; E is the exponent of the largest scale of the key's 64 tokens or up to 3 more.  So each key adds at
    most 2^-25 2^3 / 2^6 of its code times that largest scale, divided by a sum of 1 or more (of the largest weight).  float32: 24
    bits.  Sums of n terms in float32 by 32 keys a step, and half a step of the result's type."""
    score = (hd + 8) * 2.0 ** -24 * reach[..., None]
    weights = 2.0 ** -11 if kind == "bf16" else 2.0 ** -22
    sums = (most_keys / 32 + 64) * 2.0 ** -24
    floor = 2.0 ** -28 * mass if kind == "bf16" else 0.0
    return (2.0 ** -8 if kind == "bf16" else 2.0 ** -24) * np.abs(want) + size * (2 * np.expm1(score) + weights + sums) + floor + 1e-30
