"""Decoding a batch from a paged cache in 8 or 4 bits, in 64 bits: the definitions that the calls of include/cake.h state
(cake_op_append_q8, cake_op_attention_q8, their q4 forms, cake_op_sample, cake_op_pack_w4, the cake_op_gemm_w4 products), written from their
formulas with NumPy, a sequence, a head and a row at a time."""
from __future__ import annotations

import math

import numpy as np


def rope_frequencies(theta, rotary_dim, scaling=None):
    """(frequencies of the pairs, magnitude).  scaling: None, ("linear", factor), ("bands", factor, low, high, tokens),
    ("ramp", factor, tokens, high, low)."""
    freq, magnitude = [], 1.0
    for i in range(rotary_dim // 2):
        f = theta ** (-2.0 * i / rotary_dim)
        if scaling is None:
            freq.append(f)
        elif scaling[0] == "linear":
            freq.append(f / scaling[1])
        elif scaling[0] == "bands":
            _, factor, low, high, tokens = scaling
            turns = tokens * f / (2 * math.pi)
            share = min(max((turns - low) / (high - low), 0.0), 1.0)
            freq.append(share * f + (1 - share) * f / factor)
        else:
            _, factor, tokens, high, low = scaling

            def number(turns):     # the pair that turns so often: tokens * theta^(-2 i / dim) = 2 pi turns
                return rotary_dim * math.log(tokens / (2 * math.pi * turns)) / (2 * math.log(theta))
            a, b = max(math.floor(number(high)), 0), min(math.ceil(number(low)), rotary_dim - 1)
            scaled = min(max((i - a) / max(b - a, 1e-3), 0.0), 1.0)
            freq.append(scaled * f / factor + (1 - scaled) * f)
            magnitude = 0.1 * math.log(factor) + 1
    return np.array(freq), magnitude


def rotate(x, pos, freq, magnitude, layout):
    """x [heads][hd] float64 at one position."""
    y = x.copy()
    n = len(freq)
    c, s = np.cos(pos * freq) * magnitude, np.sin(pos * freq) * magnitude
    i, j = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if layout == "pairs" else (np.arange(n), np.arange(n, 2 * n))
    y[:, i] = x[:, i] * c - x[:, j] * s
    y[:, j] = x[:, i] * s + x[:, j] * c
    return y


class Pages:
    """The 8-bit pages of one layer, in the layout of the pool: codes int8 [page][K|V][head][token][hd], scales float32
    [page][K|V][head][token / block].  bits=4: of 4-bit pages, whose bytes hold two codes each (self.codes: one each, as for 8)."""

    def __init__(self, n_pages, n_kv, page_tokens, hd, block, bits=8):
        self.pt, self.block, self.n_kv, self.hd, self.bits = page_tokens, block, n_kv, hd, bits
        self.top = 127 if bits == 8 else 7
        self.codes = np.zeros((n_pages, 2, n_kv, page_tokens, hd), np.int8)
        self.scales = np.zeros((n_pages, 2, n_kv, page_tokens // block), np.float32)

    def bytes(self):
        n = len(self.codes)
        raw = (lambda c: c) if self.bits == 8 else two_a_byte
        return np.concatenate([np.concatenate([raw(self.codes[:, w].reshape(n, -1)).view(np.uint8), self.scales[:, w].reshape(n, -1).view(np.uint8)], axis=1)
                               for w in (0, 1)], axis=1)

    def take(self, raw):
        """From the pool's bytes [page][page bytes]."""
        at, n = 0, len(raw)
        raw = np.ascontiguousarray(raw)
        for w in (0, 1):
            c = self.n_kv * self.pt * self.hd * self.bits // 8
            codes = raw[:, at:at + c].view(np.int8) if self.bits == 8 else one_each(raw[:, at:at + c])
            self.codes[:, w] = codes.reshape(n, self.n_kv, self.pt, self.hd)
            at += c
            c = self.n_kv * (self.pt // self.block) * 4
            self.scales[:, w] = np.ascontiguousarray(raw[:, at:at + c]).view(np.float32).reshape(n, self.n_kv, -1)
            at += c
        return self

    def fill(self, x, which):
        """Whole pages from values x [page][head][token][hd]."""
        n = len(x)
        b = x.astype(np.float32).reshape(n, self.n_kv, self.pt // self.block, self.block * self.hd)
        s = np.abs(b).max(axis=3) / np.float32(self.top)
        self.scales[:, which] = s
        self.codes[:, which] = quantise(b, s[..., None], self.top).reshape(n, self.n_kv, self.pt, self.hd)
        return self

    def values(self, which, pages, n):
        """float64 [head][token][hd] of the first n tokens of a sequence on `pages`."""
        c = self.codes[pages, which].astype(np.float64) * np.repeat(self.scales[pages, which], self.block, axis=2)[..., None].astype(np.float64)
        return c.transpose(1, 0, 2, 3).reshape(self.n_kv, -1, self.hd)[:, :n]


def quantise(x, scale, top=127):
    """float32 in, whole numbers out."""
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.clip(np.rint(x / scale), -top, top)
    return np.where(scale > 0, c, 0)


def two_a_byte(codes):
    """Whole numbers from -8 to 7, [..., 2n] -> uint8 [..., n], the first of two in the low half."""
    c = np.asarray(codes).astype(np.int64) % 16
    return (c[..., 0::2] + 16 * c[..., 1::2]).astype(np.uint8)


def one_each(raw):
    """The codes of bytes [..., n] -> int8 [..., 2n]."""
    b = np.asarray(raw).astype(np.int64)
    both = np.stack([b % 16, b // 16], axis=-1).reshape(*b.shape[:-1], -1)
    return np.where(both > 7, both - 16, both).astype(np.int8)


def append(pages, qkv, table, lens, begin, n_q, freq, magnitude, layout):
    """Appends to `pages`; returns (q [n_q][rows][hd] float64, values [rows][2 n_kv][hd] float64); rows of no sequence: NaN."""
    n_kv, hd, pt, block = pages.n_kv, pages.hd, pages.pt, pages.block
    rows = len(qkv)
    x = qkv.reshape(rows, n_q + 2 * n_kv, hd)
    q, values = np.full((n_q, rows, hd), np.nan), np.full((rows, 2 * n_kv, hd), np.nan)
    for s in range(len(lens)):
        n = begin[s + 1] - begin[s]
        new = {}
        for i in range(n):
            pos = lens[s] - n + i
            if pos < 0:
                continue
            r = rotate(x[begin[s] + i, :n_q + n_kv].astype(np.float64), pos, freq, magnitude, layout)
            q[:, begin[s] + i] = r[:n_q]
            new.setdefault(pos // block, []).append((pos, begin[s] + i, np.stack([r[n_q:].astype(np.float32), x[begin[s] + i, n_q + n_kv:].astype(np.float32)])))
        for b, items in new.items():
            if b * block // pt >= table.shape[1]:
                continue
            page, slot = table[s, b * block // pt], b * block % pt // block
            if page < 0 or page >= len(pages.codes):
                continue
            top = np.max([np.abs(v).max(axis=2) for _, _, v in items], axis=0)
            scale = np.where(np.isfinite(top), top / np.float32(pages.top), np.float32(np.nan)).astype(np.float32)
            older = items[0][0] - b * block
            if older > 0:
                had = pages.scales[page, :, :, slot].copy()
                scale = np.where(np.isnan(scale) | np.isnan(had), np.float32(np.nan), np.maximum(scale, had))
                with np.errstate(divide="ignore", invalid="ignore"):
                    ratio = np.where(scale > 0, had / scale, np.float32(1)).astype(np.float32)
                at = slice(b * block % pt, b * block % pt + older)
                moved = np.clip(np.rint(pages.codes[page, :, :, at].astype(np.float32) * ratio[..., None, None]), -pages.top, pages.top)
                pages.codes[page, :, :, at] = np.where(ratio[..., None, None] < 1, moved, pages.codes[page, :, :, at])
            pages.scales[page, :, :, slot] = scale
            for pos, row, v in items:
                c = quantise(v, scale[..., None], pages.top)
                pages.codes[page, :, :, pos % pt] = c
                values[row] = (c * scale[..., None].astype(np.float64)).reshape(2 * n_kv, hd)
    return q, values


def attention(pages, q, table, lens, begin, window=0, sinks=0):
    """q [n_q][rows][hd] -> (out [rows][n_q][hd], the same with magnitudes of the values, the magnitudes of the codes times the
    largest scale of their 64 tokens summed without weights, the largest sum of magnitudes of a row's scores), float64.  Rows of no sequence: NaN."""
    n_q, rows, hd = q.shape
    group = n_q // pages.n_kv
    out, size, mass, reach = np.full((rows, n_q, hd), np.nan), np.zeros((rows, n_q, hd)), np.zeros((rows, n_q, hd)), np.zeros((rows, n_q))
    for s in range(len(lens)):
        n = begin[s + 1] - begin[s]
        if n <= 0:
            continue
        used = (max(lens[s], 1) + pages.pt - 1) // pages.pt
        k, v = pages.values(0, table[s, :used], lens[s]), pages.values(1, table[s, :used], lens[s])
        key = np.arange(lens[s])
        scale = np.repeat(pages.scales[table[s, :used], 1], pages.block, axis=2).transpose(1, 0, 2).reshape(pages.n_kv, -1)[:, :lens[s]].astype(np.float64)
        pad = np.zeros((pages.n_kv, -lens[s] % 64))
        most = np.repeat(np.concatenate([scale, pad], axis=1).reshape(pages.n_kv, -1, 64).max(axis=2), 64, axis=1)[:, :lens[s]] if lens[s] else scale
        for i in range(n):
            pos = lens[s] - n + i
            seen = key <= pos
            if window > 0:
                seen &= (pos - key < window) | (key < sinks)
            for h in range(n_q):
                if not seen.any():
                    out[begin[s] + i, h] = 0
                    continue
                kk, vv = k[h // group][seen], v[h // group][seen]
                x = q[h, begin[s] + i].astype(np.float64)
                z = kk @ x / math.sqrt(hd)
                p = np.exp(z - z.max())
                p /= p.sum()
                r = begin[s] + i
                out[r, h], size[r, h], mass[r, h] = p @ vv, p @ np.abs(vv), (np.abs(vv) * (most / scale)[h // group][seen][:, None]).sum(axis=0)
                reach[r, h] = (np.abs(kk) @ np.abs(x)).max() / math.sqrt(hd)
    return out, size, mass, reach


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """(tokens, log-probabilities) of float32 logits [rows][vocab]."""
    tokens, logprobs = [], []
    for r, row in enumerate(np.asarray(logits, np.float64)):
        t = 1.0 if temperature is None else float(temperature[r])
        k = 0 if top_k is None else int(top_k[r])
        p = 1.0 if top_p is None else float(top_p[r])
        low = 0.0 if min_p is None else float(min_p[r])
        x = np.where(np.isnan(row), -np.inf, row)
        order = np.argsort(-x, kind="stable")          # equal logits by id
        best = x[order[0]]
        if best == -np.inf:
            tokens.append(-1), logprobs.append(-np.inf)
            continue
        if not t > 0:
            tokens.append(int(order[0])), logprobs.append(0.0)
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            z = np.where(x == best, 0.0, (x - best) / t)
        z = np.where(np.isneginf(x), -np.inf, z)
        w = np.exp(z)
        w[w < 2.0 ** -45] = 0
        if 0 < k < len(order):
            order = order[:k]
        if p < 1:
            before = np.concatenate([[0], np.cumsum(w[order])[:-1]])
            order = order[(before < p * w[order].sum()) | (np.arange(len(order)) == 0)]
        if low > 0:
            order = order[w[order] >= min(low, 1.0)]
        ids = np.sort(order)
        run = np.cumsum(w[ids])
        at = int(np.searchsorted(run, (0.0 if np.isnan(u[r]) else float(u[r])) * run[-1], side="right"))
        if at >= len(ids) or w[ids[at]] == 0:          # u = 1
            at = int(np.nonzero(w[ids])[0][-1])
        tokens.append(int(ids[at]))
        logprobs.append(z[ids[at]] - math.log(run[-1]))
    return np.array(tokens, np.int32), np.array(logprobs)


def round_to(x, kind):
    """float32 values rounded to the model's element type ("f32" or "bf16"), as float32."""
    x = np.asarray(x, np.float32)
    if kind == "f32":
        return x
    bits = x.view(np.uint32).astype(np.uint64)
    up = ((bits + 0x7FFF + ((bits >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), np.float32(np.nan), up)


def pack_w4(w, group, kind):
    """(codes as bytes [N][(K + 31) // 32 * 16], scales [N][groups] float32, values [N][K] float64) of weights [N][K]."""
    w = np.asarray(w, np.float32)
    N, K = w.shape
    codes, scales = np.zeros((N, (K + 31) // 32 * 32)), []
    for k in range(0, K, group):
        part = w[:, k:k + group]
        top = np.abs(part).max(axis=1)
        with np.errstate(invalid="ignore"):
            s = round_to(np.where(np.isfinite(top), top / np.float32(7), np.float32(np.nan)), kind)
        codes[:, k:k + part.shape[1]] = quantise(part, s[:, None], 7)
        scales.append(s)
    raw, scales = two_a_byte(codes), np.stack(scales, axis=1)
    return raw, scales, w4_values(raw, scales, K, group)


def w4_values(raw, scales, K, group):
    """The weights [N][K], float64, that bytes and scales stand for."""
    return one_each(raw)[:, :K].astype(np.float64) * np.repeat(np.asarray(scales, np.float64), group, axis=1)[:, :K]


def silu_product(gate, up):
    return gate / (1 + np.exp(-gate)) * up
