"""Generating tokens for a batch from an 8-bit paged KV cache, as timed cases: one decoder layer's append and attention, and
the choice of the next token.

A case is a dict of plain values, `op` among them:

    append     Engine.op_append_q8: q and k of a ragged batch's new tokens rotated (adjacent pairs or halves of the first
               `rotary` elements of a head, optionally scaled for long contexts), k and v quantised into the pages with one
               scale for `block` tokens of a KV head
    attention  Engine.op_attention_q8: the new tokens' queries against those pages, causal, optionally a sliding window
               with a few first tokens that stay visible
    sample     Engine.op_sample: the next token of each row of logits by temperature, top-k, top-p and min-p from a given
               random number, and its log-probability among the tokens that were kept

`own` false: the same in elementary torch operations.  Head layouts, chunk sizes and vocabularies are those of the
repository's workloads (`synth_inputs.SHAPES`) and of a generic small bf16 model with heads of 64.

A layer page holds, for K and then for V, int8 codes [kv_head][token][head_dim] and float32 scales
[kv_head][token / block]; value = code * scale, scale = largest magnitude of the block / 127.
"""
import math

import numpy as np
import torch

own = False

#: (query heads, KV heads, head dimension, element type, rotary base)
HEADS = {
    "tiny": (4, 4, 64, "f32", 10000.0),
    "7b": (32, 32, 128, "bf16", 10000.0),
    "8b": (32, 8, 128, "bf16", 500000.0),
    "70b": (64, 8, 128, "bf16", 10000.0),
    "small": (32, 8, 64, "bf16", 500000.0),
}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one request's single token early in its answer: the smallest call, all latency
        {"name": "attention_one", "op": "attention", "heads": "8b", "seqs": 1, "rows": 1, "len": 701, "low": 701, "page": 256, "block": 1, "window": 0, "sinks": 0},
        # a serving step: 64 requests of uneven length, one token each
        {"name": "attention_batch", "op": "attention", "heads": "8b", "seqs": 64, "rows": 1, "len": 8191, "low": 500, "page": 256, "block": 64, "window": 0, "sinks": 0},
        # long answers of a multi-head model under a sliding window with four first tokens visible
        {"name": "attention_window", "op": "attention", "heads": "7b", "seqs": 24, "rows": 1, "len": 32000, "low": 20000, "page": 256, "block": 1, "window": 4096, "sinks": 4},
        # a chunk of a long prompt, computed against the cache before it
        {"name": "attention_chunk", "op": "attention", "heads": "8b", "seqs": 1, "rows": 1024, "len": 16384, "low": 16384, "page": 256, "block": 1, "window": 0, "sinks": 0},
        # several drafted tokens of each request checked in one step, heads of 64, odd lengths
        {"name": "attention_draft", "op": "attention", "heads": "small", "seqs": 33, "rows": 5, "len": 4099, "low": 37, "page": 128, "block": 16, "window": 0, "sinks": 0},
        # the float32 model: prompts' pieces and single tokens mixed in one ragged batch
        {"name": "attention_f32", "op": "attention", "heads": "tiny", "seqs": 7, "rows": 97, "len": 2048, "low": 130, "page": 128, "block": 1, "window": 512, "sinks": 2},
        # the new tokens of a serving step, rotation scaled by wavelength bands
        {"name": "append_step", "op": "append", "heads": "8b", "seqs": 64, "rows": 1, "len": 60000, "low": 500, "page": 256, "block": 1, "rotary": 128, "layout": "pairs", "scaling": "bands"},
        # a long prompt's chunks, two requests in one call, halves layout
        {"name": "append_chunk", "op": "append", "heads": "70b", "seqs": 2, "rows": 2048, "len": 72000, "low": 30000, "page": 256, "block": 64, "rotary": 128, "layout": "halves", "scaling": "linear"},
        # the float32 model, part of the head rotated, blocks that already hold tokens
        {"name": "append_f32", "op": "append", "heads": "tiny", "seqs": 9, "rows": 41, "len": 2048, "low": 60, "page": 128, "block": 16, "rotary": 48, "layout": "halves", "scaling": "ramp"},
        # the next token of one request
        {"name": "sample_one", "op": "sample", "rows": 1, "vocab": 32000, "filters": "all"},
        # a serving step's tokens over a large vocabulary, every request with its own settings
        {"name": "sample_batch", "op": "sample", "rows": 64, "vocab": 128256, "filters": "mixed"},
        # many samples of a few prompts, temperature only
        {"name": "sample_plain", "op": "sample", "rows": 256, "vocab": 32003, "filters": "none"},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "append", "sample"])
    if op == "sample":
        rows = _log_int(rng, 1, 256)
        return {"op": op, "rows": rows, "vocab": _log_int(rng, 1000, min(128256, 8200000 // rows)), "filters": rng.choice(["all", "mixed", "none"])}
    heads = rng.choice(sorted(HEADS))
    n_q, n_kv, hd, _, _ = HEADS[heads]
    page, block = rng.choice([64, 128, 256]), rng.choice([1, 1, 4, 16, 64])
    seqs = _log_int(rng, 1, 64)
    if op == "append":
        rows = _log_int(rng, 1, max(1, 4096 // seqs))
        length = max(rows, _log_int(rng, 1, min(60000, 16000000 // (seqs * n_kv))))
        return {"op": op, "heads": heads, "seqs": seqs, "rows": rows, "len": length, "low": max(rows, length // 3), "page": page, "block": block,
                "rotary": rng.choice([hd, hd, hd // 2, hd - 16]), "layout": rng.choice(["pairs", "halves"]), "scaling": rng.choice(["none", "linear", "bands", "ramp"])}
    rows = rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 9, 1024)])
    rows = min(rows, math.isqrt(500000000 // (seqs * n_q)))
    most = min(32000, 4000000 // (seqs * n_kv * hd // 128), 500000000 // (rows * seqs * n_q))   # cache and pairs at most the listed ones'
    length = max(rows, _log_int(rng, 1, max(2, most)))
    window = rng.choice([0, 0, _log_int(rng, 16, 4096)])
    return {"op": op, "heads": heads, "seqs": seqs, "rows": rows, "len": length, "low": max(min(rows, length), length // 4), "page": page, "block": block,
            "window": window, "sinks": rng.choice([0, 1, 4, 70]) if window else 0}


# ------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _lengths(case):
    """Tokens of each sequence and how many of them are this call's, spread over the case's range; the first has the most."""
    n, rows = case["seqs"], case["rows"]
    r = np.random.default_rng([n, rows, case["len"]])
    lens = r.integers(case["low"], case["len"] + 1, n)
    lens[0] = case["len"]
    new = np.full(n, rows) if rows <= 8 else r.integers(1, rows + 1, n)
    new[0] = rows
    return lens.astype(np.int64), np.minimum(new, lens).astype(np.int64)


def rotary_frequencies(rotary, theta, scaling):
    """(radians per position of each pair, factor on cosine and sine) of the four scalings, in 64 bits."""
    i = np.arange(rotary // 2, dtype=np.float64)
    f = theta ** (-2.0 * i / rotary)
    if scaling == "linear":
        return f / 4.0, 1.0
    if scaling == "bands":       # short wavelengths as they are, long ones at an eighth, a ramp in between
        turns = 8192.0 * f / (2 * math.pi)
        keep = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return f * (keep + (1 - keep) / 8.0), 1.0
    if scaling == "ramp":        # by the pair's index, between the pairs that turn 32 times and once in 4096 tokens
        at = [rotary * math.log(4096.0 / (turns * 2 * math.pi)) / (2 * math.log(theta)) for turns in (32.0, 1.0)]
        low, high = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rotary - 1)
        part = np.clip((i - low) / max(high - low, 1e-3), 0.0, 1.0)
        return f / 16.0 * part + f * (1 - part), 0.1 * math.log(16.0) + 1.0
    return f, 1.0


def _rotary_spec(scaling):
    return {"none": None, "linear": ("linear", 4.0), "bands": ("bands", 8.0, 1.0, 4.0, 8192), "ramp": ("ramp", 16.0, 4096, 32.0, 1.0)}[scaling]


def _page_bytes(case):
    _, n_kv, hd, _, _ = HEADS[case["heads"]]
    return 2 * n_kv * (case["page"] * hd + case["page"] // case["block"] * 4)


def _views(pool, case):
    """The codes [page][kv_head][token][head_dim] and scales [page][kv_head][block] of K and of V in the pool."""
    _, n_kv, hd, _, _ = HEADS[case["heads"]]
    pages, page, blocks = pool.shape[0], case["page"], case["page"] // case["block"]
    codes, scales, got = n_kv * page * hd, n_kv * blocks * 4, []
    for at in (0, codes + scales):
        got.append(pool[:, at:at + codes].view(torch.int8).unflatten(1, (n_kv, page, hd)))
        got.append(pool[:, at + codes:at + codes + scales].view(torch.float32).unflatten(1, (n_kv, blocks)))
    return got


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "sample":
        rows, vocab = case["rows"], case["vocab"]
        logits = torch.randn((rows, vocab), generator=g, device="cuda") * 2.2
        favoured = torch.randint(0, vocab, (rows, 24), generator=g, device="cuda")
        logits.scatter_add_(1, favoured, torch.rand((rows, 24), generator=g, device="cuda") * 8.0 + 3.0)
        r = np.random.default_rng([seed, 3])
        temperature = r.uniform(0.5, 1.2, rows)
        top_k, top_p, min_p = np.zeros(rows), np.ones(rows), np.zeros(rows)
        if case["filters"] != "none":
            on = np.ones((3, rows), bool) if case["filters"] == "all" else r.random((3, rows)) < 0.6
            top_k[on[0]] = r.integers(20, 200, on[0].sum())
            top_p[on[1]] = r.uniform(0.7, 0.98, on[1].sum())
            min_p[on[2]] = r.uniform(0.001, 0.05, on[2].sum())
            if case["filters"] == "mixed":
                temperature[r.random(rows) < 0.1] = 0.0          # some requests ask for the likeliest token
        f32 = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()  # noqa: E731
        return {"case": case, "logits": logits, "temperature": f32(temperature), "top_k": torch.from_numpy(top_k.astype(np.int32)).cuda(),
                "top_p": f32(top_p), "min_p": f32(min_p), "u": f32(np.minimum(r.random(rows), 1 - 2.0 ** -24))}
    n_q, n_kv, hd, kind, theta = HEADS[case["heads"]]
    page, block = case["page"], case["block"]
    lens, new = _lengths(case)
    per = (lens + page - 1) // page
    used, width = int(per.sum()), int(per.max())
    order = np.random.default_rng([seed, 5]).permutation(used + 3)[:used]
    table, at = np.full((case["seqs"], width), -1, np.int32), 0
    for s, n in enumerate(per):
        table[s, :n] = order[at:at + n]
        at += n
    begin = np.concatenate([[0], np.cumsum(new)])
    pool = torch.empty((used + 3, _page_bytes(case)), dtype=torch.uint8, device="cuda")
    for codes, scales in zip(*[iter(_views(pool, case))] * 2):
        for p in range(0, used + 3, 64):                         # a cache of values of uneven size, 64 pages at a time
            x = torch.randn(codes[p:p + 64].shape, generator=g, device="cuda")
            x *= torch.exp(0.4 * torch.randn((*x.shape[:3], 1), generator=g, device="cuda"))
            x = x.unflatten(2, (page // block, block))
            s = x.abs().amax(dim=(3, 4)) / 127.0
            codes[p:p + 64] = torch.round(x / s[..., None, None]).flatten(2, 3).to(torch.int8)
            scales[p:p + 64] = s
    i32 = lambda a: torch.from_numpy(a.astype(np.int32)).cuda()  # noqa: E731
    state = {"case": case, "pool": pool, "table": torch.from_numpy(table).cuda(), "lens": i32(lens), "begin": i32(begin), "rows": int(begin[-1]),
             "max_rows": int(new.max()), "max_len": int(lens.max())}
    if case["op"] == "append":
        state["qkv"] = torch.randn((state["rows"], (n_q + 2 * n_kv) * hd), generator=g, device="cuda")
        state["qkv"] *= torch.exp(0.4 * torch.randn((state["rows"], 1), generator=g, device="cuda"))
        f, magnitude = rotary_frequencies(case["rotary"], theta, case["scaling"])
        state["frequencies"], state["magnitude"] = torch.from_numpy(f).cuda(), magnitude
    else:
        state["q"] = (torch.randn((n_q, state["rows"], hd), generator=g, device="cuda") * 1.5).to(DTYPES[kind])
    return state


# ------------------------------------------------------------------------------------------------- the framework's calls
_kept = {}


def _engine(heads):
    """An engine of these heads on torch's current stream: what a serving program makes once and keeps."""
    if heads not in _kept:
        import paper_2410_03065_amd as cake
        import synth_inputs as si
        n_q, n_kv, hd, kind, theta = HEADS[heads]
        shape = si.ModelShape("operators-" + heads, 1, 512, n_q, n_kv, hd, 512, 256, kind, rope_theta=theta)
        _kept[heads] = cake.Engine(shape, None, max_tokens=1024, max_chunk=1024, page_tokens=64, compute_stream=torch.cuda.current_stream())
    return _kept[heads]


def _rope(case):
    key = (case["heads"], case["rotary"], case["layout"], case["scaling"])
    if key not in _kept:
        import paper_2410_03065_amd as cake
        _kept[key] = cake.rope(HEADS[case["heads"]][4], case["rotary"], layout=case["layout"], scaling=_rotary_spec(case["scaling"]))
    return _kept[key]


def _run_own(state):
    case = state["case"]
    if case["op"] == "sample":
        tokens, logprobs = _engine("8b").op_sample(state["logits"], state["u"], temperature=state["temperature"], top_k=state["top_k"],
                                                   top_p=state["top_p"], min_p=state["min_p"])
        return {"tokens": tokens, "logprobs": logprobs}
    engine = _engine(case["heads"])
    if "batch" not in state:         # the descriptor of the batch's buffers, kept from step to step like them
        state["batch"] = engine.q8_batch(state["pool"], state["table"], state["lens"], state["begin"], n_rows=state["rows"], page_tokens=case["page"],
                                         scale_tokens=case["block"], max_rows=state["max_rows"], max_len=state["max_len"])
    if case["op"] == "attention":
        return engine.op_attention_q8(state["q"], 0, state["batch"], window=case["window"], sinks=case["sinks"])
    q, values = engine.op_append_q8(state["qkv"], 0, state["batch"], _rope(case), want_values=True)
    return _append_outputs(state, q, values)


def _append_outputs(state, q, values):
    """q [query head][row][head_dim]; values [row][K then V heads][head_dim], what the pages hold of the new tokens; where a
    block is longer than a token, also all scales (a block that got tokens may have a new one)."""
    got = {"q": q, "values": values}
    if state["case"]["block"] > 1:
        _, got["k_scales"], _, got["v_scales"] = _views(state["pool"], state["case"])
    return got


# ------------------------------------------------------------------------------------------------- the plain forms
def _rows_of(state):
    """For each row of the batch its sequence, its number among that sequence's rows, and its position."""
    row = torch.arange(state["rows"], device="cuda")
    begin = state["begin"].long()
    seq = torch.searchsorted(begin, row, right=True) - 1
    mine = row - begin[seq]
    new = begin[1:] - begin[:-1]
    return seq, mine, (state["lens"].long() - new)[seq] + mine


def _plain_attention(state):
    case = state["case"]
    n_q, n_kv, hd, kind, _ = HEADS[case["heads"]]
    page, block, window, sinks, group = case["page"], case["block"], case["window"], case["sinks"], n_q // n_kv
    k_codes, k_scales, v_codes, v_scales = _views(state["pool"], case)
    lens, begin = state["lens"].long(), state["begin"].long()
    new = begin[1:] - begin[:-1]
    most = state["max_rows"]
    # keys that some row of the sequence sees: the first `sinks`, and the window before its first row onwards
    if window:
        first = (lens - new - window + 1).clamp(min=0)
        slot = torch.arange(sinks + min(state["max_len"], window + most), device="cuda")
        at = torch.where(slot < sinks, slot, first[:, None] + slot - sinks)
        there = torch.where(slot < sinks, (slot < first[:, None]) & (slot < lens[:, None]), at < lens[:, None])
    else:
        at = torch.arange(state["max_len"], device="cuda").expand(case["seqs"], -1)
        there = at < lens[:, None]
    at = torch.where(there, at, torch.zeros_like(at))
    phys = torch.gather(state["table"].long(), 1, at // page).clamp(min=0)
    keys = k_codes[phys, :, at % page].float() * k_scales[phys, :, at % page // block][..., None]       # [seq][key][kv_head][head_dim]
    values = v_codes[phys, :, at % page].float() * v_scales[phys, :, at % page // block][..., None]
    number = torch.arange(most, device="cuda")
    row = (begin[:-1, None] + number).clamp(max=state["rows"] - 1)
    q = state["q"].float()[:, row].permute(1, 0, 2, 3).reshape(case["seqs"], n_kv, group * most, hd)    # [seq][kv_head][head in group, row]
    scores = torch.matmul(q, keys.permute(0, 2, 3, 1).contiguous()) / math.sqrt(hd)
    pos = (lens - new)[:, None] + number
    seen = there[:, None, :] & (at[:, None, :] <= pos[:, :, None])
    if window:
        seen &= (pos[:, :, None] - at[:, None, :] < window) | (at[:, None, :] < sinks)
    scores = scores.unflatten(2, (group, most)).masked_fill_(~seen[:, None, None], -math.inf).flatten(2, 3)
    top = scores.amax(dim=3, keepdim=True)
    p = torch.exp(scores - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(dim=3, keepdim=True)
    out = torch.matmul(p, values.permute(0, 2, 1, 3).contiguous()) / torch.where(total == 0, torch.ones_like(total), total)
    seq, mine, _ = _rows_of(state)
    out = out.unflatten(2, (group, most))[seq, :, :, mine]                                              # [row][kv_head][group][head_dim]
    return out.reshape(state["rows"], n_q * hd).to(DTYPES[kind])


def _rotate(x, cos, sin, rotary, layout):
    """x [row][head][head_dim] in 64 bits, cos and sin [row][1][pair]."""
    y = x.clone()
    a, b = (x[..., 0:rotary:2], x[..., 1:rotary:2]) if layout == "pairs" else (x[..., :rotary // 2], x[..., rotary // 2:rotary])
    if layout == "pairs":
        y[..., 0:rotary:2], y[..., 1:rotary:2] = a * cos - b * sin, a * sin + b * cos
    else:
        y[..., :rotary // 2], y[..., rotary // 2:rotary] = a * cos - b * sin, a * sin + b * cos
    return y


def _quantise(x, codes, scales, phys, off, state, holds, old_pos, old_phys):
    """x [row][kv_head][head_dim] float32 into the pages; returns the values that they then stand for."""
    block = state["case"]["block"]
    size = x.abs().amax(dim=2) / 127.0
    if block == 1:
        scale = size
        scales[phys, :, off] = scale
    else:
        blocks = scales.shape[2]
        where = (phys * scales.shape[1])[:, None] * blocks + torch.arange(scales.shape[1], device="cuda") * blocks + (off // block)[:, None]
        before = scales.contiguous().flatten()
        had = torch.where(holds[:, None], before[where], torch.zeros_like(size))    # of a block that held tokens before this call
        after = torch.zeros_like(before)
        after.scatter_reduce_(0, where.flatten(), torch.maximum(size, had).flatten(), "amax", include_self=True)
        scale = after[where]
        # those blocks' older tokens: [sequence][block - 1] positions, -1 where there is none
        there = old_pos >= 0
        slot = (old_pos.clamp(min=0) % state["case"]["page"])
        index = (old_phys * scales.shape[1])[..., None] * blocks + torch.arange(scales.shape[1], device="cuda") * blocks + (slot // block)[..., None]
        new_scale = after[index]
        ratio = torch.where(new_scale > 0, before[index] / new_scale, torch.ones_like(new_scale))
        older = codes[old_phys, :, slot].float()
        moved = torch.round(older * ratio[..., None]).clamp(-127, 127)
        keep = there[..., None, None]
        flat_phys, flat_slot, flat = old_phys[there], slot[there], torch.where(keep, moved, older)[there]
        codes[flat_phys, :, flat_slot] = flat.to(torch.int8)
        scales[phys, :, off // block] = scale
    code = torch.where(scale[..., None] > 0, torch.round(x / scale[..., None]), torch.zeros_like(x)).clamp(-127, 127)
    codes[phys, :, off] = code.to(torch.int8)
    return code * scale[..., None]


def _plain_append(state):
    case = state["case"]
    n_q, n_kv, hd, kind, _ = HEADS[case["heads"]]
    page, block = case["page"], case["block"]
    seq, mine, pos = _rows_of(state)
    angle = pos.double()[:, None, None] * state["frequencies"]
    cos, sin = torch.cos(angle) * state["magnitude"], torch.sin(angle) * state["magnitude"]
    x = state["qkv"].unflatten(1, (n_q + 2 * n_kv, hd))
    turned = _rotate(x[:, :n_q + n_kv].double(), cos, sin, case["rotary"], case["layout"]).float()
    q = turned[:, :n_q].transpose(0, 1).to(DTYPES[kind]).contiguous()
    phys = state["table"].long()[seq, pos // page]
    lens, begin = state["lens"].long(), state["begin"].long()
    start = lens - (begin[1:] - begin[:-1])                                    # the first new position of each sequence
    holds = (pos // block * block) < start[seq]
    old = (start // block * block)[:, None] + torch.arange(max(block - 1, 1), device="cuda")
    old = torch.where(old < start[:, None], old, torch.full_like(old, -1))
    old_phys = torch.gather(state["table"].long(), 1, old.clamp(min=0) // page).clamp(min=0)
    k_codes, k_scales, v_codes, v_scales = _views(state["pool"], case)
    k = _quantise(turned[:, n_q:], k_codes, k_scales, phys, pos % page, state, holds, old, old_phys)
    v = _quantise(x[:, n_q + n_kv:], v_codes, v_scales, phys, pos % page, state, holds, old, old_phys)
    return _append_outputs(state, q, torch.cat([k, v], dim=1).to(DTYPES[kind]))


def _plain_sample(state):
    logits = state["logits"].double()
    rows, vocab = logits.shape
    greedy = state["temperature"] <= 0
    t = torch.where(greedy, torch.ones_like(state["temperature"]), state["temperature"]).double()[:, None]
    value, index = torch.sort(logits, dim=1, descending=True, stable=True)     # equal ones by their id
    w = torch.exp((value - value[:, :1]) / t)
    k = torch.where(state["top_k"] > 0, state["top_k"], torch.full_like(state["top_k"], vocab)).long()[:, None]
    w = torch.where(torch.arange(vocab, device="cuda") < k, w, torch.zeros_like(w))
    reached = torch.cumsum(w, dim=1)
    before = torch.cat([torch.zeros_like(reached[:, :1]), reached[:, :-1]], dim=1)
    p = state["top_p"].double()[:, None]
    keep = (p >= 1) | (before < p * reached[:, -1:])
    keep &= w >= state["min_p"].double()[:, None]
    kept = torch.zeros_like(w).scatter_(1, index, w * keep)
    reached = torch.cumsum(kept, dim=1)
    total = reached[:, -1:]
    token = (reached <= state["u"].double()[:, None] * total).sum(dim=1).clamp(max=vocab - 1)
    token = torch.where(greedy, index[:, 0], token)
    logprob = torch.log(kept.gather(1, token[:, None]) / total)[:, 0]
    return {"tokens": token.int(), "logprobs": torch.where(greedy, torch.zeros_like(logprob), logprob).float()}


def run(state):
    if own:
        return _run_own(state)
    return {"attention": _plain_attention, "append": _plain_append, "sample": _plain_sample}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------- sizes
def work(case):
    if case["op"] == "sample":
        return {"bytes": 4.0 * case["rows"] * case["vocab"] + 28.0 * case["rows"], "flops": 0.0}
    n_q, n_kv, hd, kind, _ = HEADS[case["heads"]]
    e = 4 if kind == "f32" else 2
    lens, new = _lengths(case)
    rows = float(new.sum())
    if case["op"] == "append":
        out = n_q * hd * e + 2 * n_kv * hd * (1 + e) + 2 * n_kv * 4.0 / case["block"]
        return {"bytes": rows * ((n_q + 2 * n_kv) * hd * 4 + out), "flops": rows * (n_q + n_kv) * case["rotary"] * 3.0}
    keys = pairs = 0.0
    for n, r in zip(lens, new):
        pos = np.arange(n - r, n, dtype=np.float64)
        if case["window"]:
            first = max(0, n - r - case["window"] + 1)
            keys += n - first + min(case["sinks"], first)
            pairs += np.sum(np.minimum(pos + 1, case["window"]) + np.minimum(case["sinks"], np.maximum(0, pos + 1 - case["window"])))
        else:
            keys += n
            pairs += np.sum(pos + 1)
    return {"bytes": keys * n_kv * 2 * (hd + 4.0 / case["block"]) + 2 * rows * n_q * hd * e, "flops": 4.0 * hd * n_q * pairs}


# ------------------------------------------------------------------------------------------------- definitions in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    return {"attention": _exact_attention, "append": _exact_append, "sample": _exact_sample}[case["op"]](state)


def _exact_attention(state):
    case = state["case"]
    n_q, n_kv, hd, _, _ = HEADS[case["heads"]]
    kc, ks, vc, vs = _views(state["pool"], case)
    lens, begin, table = state["lens"].tolist(), state["begin"].tolist(), state["table"].long()
    out = torch.zeros((state["rows"], n_q, hd), dtype=torch.float64, device="cuda")
    for s, n in enumerate(lens):
        pages = table[s, :(n + case["page"] - 1) // case["page"]]
        rows = begin[s + 1] - begin[s]
        pos, key = torch.arange(n - rows, n, device="cuda")[:, None], torch.arange(n, device="cuda")
        hidden = key > pos
        if case["window"]:
            hidden = hidden | ((key <= pos - case["window"]) & (key >= case["sinks"]))
        for h in range(n_kv):
            k, v = ((c[pages, h].double() * sc[pages, h].double().repeat_interleave(case["block"], dim=1)[..., None]).reshape(-1, hd)[:n] for c, sc in ((kc, ks), (vc, vs)))
            for i in range(h * (n_q // n_kv), (h + 1) * (n_q // n_kv)):
                a = (state["q"][i, begin[s]:begin[s + 1]].double() @ k.T) * hd ** -0.5
                out[begin[s]:begin[s + 1], i] = torch.softmax(a.masked_fill(hidden, -math.inf), dim=1) @ v
    return out.flatten(1, 2)


def _exact_append(state):
    """The rotation in 64 bits.  The scales and codes are defined on float32 values: the rotated key is rounded to float32,
    scale = largest magnitude / 127 and value / scale are float32 quotients, halves round to even."""
    case = state["case"]
    n_q, n_kv, hd, _, theta = HEADS[case["heads"]]
    page, block = case["page"], case["block"]
    _, ks, _, vs = (a.cpu().numpy().copy() for a in _views(state["pool"], case))
    lens, begin, table = state["lens"].tolist(), state["begin"].tolist(), state["table"].tolist()
    x = state["qkv"].cpu().numpy().reshape(state["rows"], n_q + 2 * n_kv, hd).astype(np.float64)
    pos = np.concatenate([np.arange(n - (e - b), n) for n, b, e in zip(lens, begin, begin[1:])])
    f, magnitude = rotary_frequencies(case["rotary"], theta, case["scaling"])
    z = magnitude * np.exp(1j * (pos[:, None] * f))[:, None]
    half = case["rotary"] // 2
    i, j = (2 * np.arange(half), 2 * np.arange(half) + 1) if case["layout"] == "pairs" else (np.arange(half), np.arange(half) + half)
    turned = (x[:, :n_q + n_kv][..., i] + 1j * x[:, :n_q + n_kv][..., j]) * z
    x[:, :n_q + n_kv][..., i], x[:, :n_q + n_kv][..., j] = turned.real, turned.imag
    q = x[:, :n_q].transpose(1, 0, 2).copy()
    kv, values = x[:, n_q:].astype(np.float32), np.zeros((state["rows"], 2 * n_kv, hd))
    size = np.abs(kv).max(axis=2) / np.float32(127)
    for s, n in enumerate(lens):
        start, stop = n - (begin[s + 1] - begin[s]), n
        for b in range(start // block, (stop - 1) // block + 1):
            lo, hi = max(start, b * block), min(stop, (b + 1) * block)
            r = slice(begin[s] + lo - start, begin[s] + hi - start)
            phys, slot = table[s][b * block // page], b * block % page // block
            scale = size[r].max(axis=0)
            if b * block < start:
                scale = np.maximum(scale, np.concatenate([ks[phys, :, slot], vs[phys, :, slot]]))
            ks[phys, :, slot], vs[phys, :, slot] = scale[:n_kv], scale[n_kv:]
            values[r] = np.clip(np.rint(kv[r] / scale[:, None]), -127, 127).astype(np.float64) * scale[:, None].astype(np.float64)
    got = {"q": torch.from_numpy(q), "values": torch.from_numpy(values)}
    if block > 1:
        got["k_scales"], got["v_scales"] = torch.from_numpy(ks.astype(np.float64)), torch.from_numpy(vs.astype(np.float64))
    return got


def _exact_sample(state):
    logits = state["logits"].cpu().numpy().astype(np.float64)
    t, k, p, low, u = (state[n].cpu().numpy().astype(np.float64) for n in ("temperature", "top_k", "top_p", "min_p", "u"))
    tokens, logprobs = np.zeros(len(logits), np.int32), np.zeros(len(logits))
    for r, row in enumerate(logits):
        if t[r] <= 0:
            tokens[r] = int(np.argmax(row))
            continue
        order = np.argsort(-row, kind="stable")
        if k[r] > 0:
            order = order[:int(k[r])]
        w = np.exp((row[order] - row[order[0]]) / t[r])
        n = len(order)
        if p[r] < 1:
            n = 1 + int(np.count_nonzero(np.cumsum(w)[:-1] < p[r] * np.sum(w)))
        n = min(n, int(np.count_nonzero(w >= low[r])))
        ids = np.sort(order[:n])
        mass = np.cumsum(np.exp((row[ids] - row[order[0]]) / t[r]))
        at = int(np.searchsorted(mass, u[r] * mass[-1], side="right"))
        tokens[r], logprobs[r] = ids[at], (row[ids[at]] - row[order[0]]) / t[r] - math.log(mass[-1])
    return {"tokens": torch.from_numpy(tokens), "logprobs": torch.from_numpy(logprobs)}
