"""Attention over a 4-bit store in 64 bits, with what a kernel may be off by, row by row and head by head, from the arithmetic that it is
documented to use.  In a score (units of the scale, angles aside, for every token j):

  query     turned in fp32 and split into two fp16 terms: 2^-22 of each channel and 2^-25 of the row's largest power of two (the low term's
            last place; as much again where fp16 rows are scaled ahead of it).  Own keys of bf16 calls meet two bf16 terms: 2^-16
  turn      two products and the softmax scale's factor, 2^-24 each: 2^-22 together; cos and sin: the fraction of a revolution in fp32 (2^-26,
            times 2 pi) and the instructions' own 2^-22.9 (measured over all fractions): 2^-22.  Without a turn they are 1 and 0: the factor's
            rounding and the product's, 2^-23
  sum       chained matrix instructions: 2^-23.5 of the sum of magnitudes at the most (measured against 64 bits): 2^-23
A probability is off by its score's and by the weighted mean of all scores' (the row sum), by exp2's last place (2^-23), the rounding of its
argument, and the sums' roundings.  For the product with v it is rounded to fp16 (2^-11, and 2^-33 of the row's largest: half the step below 2^-22 of it); own blocks: two terms."""

from __future__ import annotations

import numpy as np

from paper_2502_11101_amd import binding as cf
from tests import q4_reference as R

HALF = cf.CF_ROPE_HALF
SPLIT = {"bf16": 2.0 ** -16, "f16": 2.0 ** -22}          # two terms of the type


def pairs(x, pairing):
    """x [..., 128] as the two channels of its 64 slices."""
    return (x[..., :64], x[..., 64:]) if pairing == "half" else (x[..., 0::2], x[..., 1::2])


def turn(x, positions, rope_base, pairing):
    a, b = pairs(x, pairing)
    angle = positions * rope_base ** (-2.0 * np.arange(64) / 128)
    c, s = np.cos(angle), np.sin(angle)
    u, w = a * c - b * s, a * s + b * c
    out = np.empty_like(x)
    out_a, out_b = pairs(out, pairing)
    out_a[...], out_b[...] = u, w
    return out


def spread(x, pairing):
    """Every channel's magnitude and its partner's, added."""
    x = np.abs(x)
    out = np.empty_like(x)
    a, b = pairs(x, pairing)
    out_a, out_b = pairs(out, pairing)
    out_a[...] = out_b[...] = a + b
    return out


def attention(q, q_pos, k_store, v_store, k_self, v_self, segs, n_kv_heads, rope_base, pairing="half", scale=None, dtype="bf16", query=None):
    """(out, mass, out bound, mass bound): out [rows, heads, 128] ahead of its own rounding, mass per entry.  `query`: what to replace a segment's
    turned queries by (own: bool), to see what another arithmetic would give."""
    q = np.asarray(q, dtype=np.float64)
    rows, hq, _ = q.shape
    group = hq // n_kv_heads
    scale = 1.0 / np.sqrt(128) if scale is None else float(np.float32(scale))
    unit = 2.0 ** np.floor(np.log2(np.maximum(np.abs(q).max(-1), 1e-300)))             # [rows, heads]
    scores, off, values, entry, own_of = [], [], [], [], []
    for i, g in enumerate(segs):
        own = g.kind == 2
        k, v = ((k_self, v_self) if own else (k_store, v_store))
        k = np.asarray(k[g.tok_offset:g.tok_offset + g.len], dtype=np.float64)
        v = np.asarray(v[g.tok_offset:g.tok_offset + g.len], dtype=np.float64)
        delta = g.new_start - g.stored_start - q_pos
        turned = turn(q, -delta, rope_base, pairing)
        used = turned if query is None else query(turned, unit, own)
        take = lambda x, y: np.matmul(x.transpose(1, 0, 2), np.repeat(y, group, axis=1).transpose(1, 2, 0)) * scale      # noqa: E731
        size = take(np.abs(turned), np.abs(k))
        s = take(used, k)
        low = 0.0 if own and dtype == "bf16" else 2.0 ** -25 * (3 if dtype == "f16" else 1)
        e = size * ((SPLIT[dtype] if own else 2.0 ** -22) + (2.0 ** -22 if delta else 2.0 ** -23) + 2.0 ** -23)
        e += low * unit.T[..., None] * np.repeat(np.abs(k).sum(-1), group, axis=1).T[:, None] * scale
        if delta:
            e += 2.0 ** -22 * take(spread(q, pairing), np.abs(k))
        if own:
            s = np.where(np.arange(g.len) <= np.arange(rows)[:, None], s, -np.inf)
        scores.append(s)
        off.append(e)
        values.append(np.repeat(v, group, axis=1))
        entry.append(np.full(g.len, i))
        own_of.append(np.full(g.len, own))
    s, e, v = np.concatenate(scores, -1), np.concatenate(off, -1), np.concatenate(values).transpose(1, 0, 2)      # [heads, rows, n], [heads, n, 128]
    entry, own_of = np.concatenate(entry), np.concatenate(own_of)
    top = s.max(-1, keepdims=True)
    p = np.exp(s - top)
    p /= p.sum(-1, keepdims=True)
    n = s.shape[-1]
    sums = 2.0 ** -24 * (n / 32 + 64)
    x = np.where(p > 0, (top - np.where(np.isfinite(s), s, top)) * 1.4427, 0.0) + 16
    d = e + x * 2.0 ** -24 + 2.0 ** -23 + sums
    mean = (p * d).sum(-1, keepdims=True)
    dp = p * np.expm1(d + mean)
    rounding = np.where(own_of, SPLIT[dtype], 2.0 ** -11) * p + np.where(own_of & (dtype == "bf16"), 0.0, 2.0 ** -33) * p.max(-1, keepdims=True)
    out = np.matmul(p, v).transpose(1, 0, 2)
    out_off = np.matmul(dp + rounding + sums * p, np.abs(v)).transpose(1, 0, 2)
    mass, mass_off = np.zeros(len(segs)), np.zeros(len(segs))
    np.add.at(mass, entry, p.sum((0, 1)))
    np.add.at(mass_off, entry, (dp + 2.0 ** -17 * p).sum((0, 1)))                        # up to 128 sums of masses
    return out, mass, out_off, mass_off


def factor(scale):
    """Of the softmax scale (times log2 e) between 1 and 2, which the kernels turn the query with."""
    x = float(np.float32(np.float32(scale) * np.float32(1.44269504)))
    return x / 2.0 ** np.floor(np.log2(x))


def rounded_query(terms, bits, factor=1.0):
    """What a query of that many terms of `bits` bits stands for, scaled by its row's power of two (see `query` above)."""
    def query(turned, unit, own):
        rest = turned / unit[..., None] * factor
        total = np.zeros_like(rest)
        for _ in range(terms):
            m, e = np.frexp(rest)
            term = np.ldexp(np.rint(np.ldexp(m, bits)), e - bits)
            total, rest = total + term, rest - term
        return total * unit[..., None] / factor
    return query


def single_tokens(rng, heads, n, dtype, q_rows=1, loud=3.0):
    """Inputs whose masses tell how well scores are known: `n` entries of one token each, loud queries."""
    host = R.random_store(rng, n, heads, dtype)
    return host, rng.standard_normal((q_rows, heads, 128)) * loud


def one_channel(rng, n, dtype, q_rows=1):
    """The same with one head, whose queries are all alike and have one channel: nothing averages out, and few products are added up."""
    host = R.random_store(rng, n, 1, dtype)
    q = np.zeros((q_rows, 1, 128))
    q[:, :, 5] = 93.0                                    # (a loud channel of the keys)
    return host, q
