"""Plain NumPy definitions of the 4-bit cache store, in 64 bits, that the GPU tests compare with: the format, its writer, the
bounds on what attention over it may be off by, and a scheduler step of a cache in blocks, request by request."""

from __future__ import annotations

import numpy as np

from oracle import cachefocus_oracle as orc
from paper_2502_11101_amd import binding as cf

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E_RANGE = {"bf16": (-125, 125), "f16": (-23, 13)}
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}       # of a rounding to the type, relative to the value


def decode(codes, scales):
    """Values [..., 128] of codes [..., 64] and scale bytes [..., 4]."""
    nibble = np.stack([codes & 15, codes >> 4], axis=-1).reshape(*codes.shape[:-1], 128)
    value = np.where(nibble & 8, -1.0, 1.0) * MAGNITUDES[nibble & 7]
    s = np.repeat(np.asarray(scales, dtype=np.int64), 32, axis=-1)
    return np.where(s == 255, np.nan, value * 2.0 ** (s - 127.0))


def encode(x, dtype):
    """(codes, scales, clear) of values [..., 128]; clear: whether a value is further than 2^-20 of itself from a border between codes, so
    that a rotation's last bit cannot have moved it."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(*x.shape[:-1], 4, 32)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        top = np.abs(g).max(-1)
        bad = ~np.isfinite(top)
        safe = np.where(bad | (top == 0), 1.0, top)
        e = np.ceil(np.log2(safe / 7.0))
        e = np.where(safe > 7.0 * 2.0 ** e, e + 1, e)
        e = np.where(safe <= 7.0 * 2.0 ** (e - 1), e - 1, e)
        e = np.where(top == 0, -1000, e).clip(*E_RANGE[dtype])
        y = np.where(bad[..., None], 0.0, np.abs(g) / 2.0 ** e[..., None])
    borders = (MAGNITUDES[:-1] + MAGNITUDES[1:]) / 2
    code = np.zeros(g.shape, dtype=np.uint8)
    for i, b in enumerate(borders):                      # a tie goes to the even index
        code += (y > b) | ((y == b) & (i % 2 == 1))
    near = (np.abs(y[..., None] - borders) < 2.0 ** -20 * borders).any(-1)
    near |= (np.abs(safe / 2.0 ** e - 7.0) < 1e-5)[..., None] | (np.abs(safe / 2.0 ** e - 3.5) < 1e-5)[..., None]
    code |= np.signbit(g).astype(np.uint8) << 3
    code = np.where(bad[..., None], 0, code).reshape(*x.shape[:-1], 64, 2)
    scales = np.where(bad, 255, e + 127).astype(np.uint8)
    return (code[..., 0] | code[..., 1] << 4).astype(np.uint8), scales, ~near.reshape(x.shape)


def turned(x, shift, rope_base, pairing="half"):
    """Rows [n][heads][128] turned by shift[n] positions."""
    out = np.empty(x.shape, dtype=np.float64)
    for i, s in enumerate(np.broadcast_to(shift, (x.shape[0],))):
        out[i:i + 1] = orc.rotate(np.asarray(x[i:i + 1], dtype=np.float64), int(s), rope_base, pairing) if s else x[i:i + 1]
    return out


def random_store(rng, n_tokens, heads, dtype, loud=True):
    """codes and scales of keys and values [token][head][.], with loud channels among the keys, as trained models have."""
    out = {}
    for x in "kv":
        v = rng.standard_normal((n_tokens, heads, 128))
        if loud and x == "k":
            v[..., 5::43] *= 4
        out[x + "_codes"], out[x + "_scales"], _ = encode(v, dtype)
    return out


def attention(q, q_pos, k_store, v_store, k_self, v_self, segs, n_kv_heads, rope_base, pairing="half", scale=None):
    """(out, mass, out bound, mass bound) of one query whose rows carry local positions: the oracle's result, and what a kernel may be
    off by before its output's own rounding, from the arithmetic it is documented to use.
      score    the query enters with 15 bits: off by 2^-15 * sum |q_c k_c|, twice that with fp32's sums and angles
      p        rounded to fp16 for the product with v (own blocks: 15 bits or more): 2^-11; and by the score's error
    so |d out| <= (2^-11 + 2 * ds) * sum p |v| and |d mass| <= 2 * ds * mass, each twice (row sums) and with 1e-6 for fp32 sums."""
    args = (q_pos, k_store, v_store, k_self, v_self, segs, n_kv_heads, rope_base, pairing)
    q = np.asarray(q, dtype=np.float64)
    out, mass = orc.prefill_attention(q, 0, *args, scale=scale)
    absolute = lambda x: None if x is None else np.abs(x)
    with_abs = (q_pos, k_store, absolute(v_store), k_self, absolute(v_self), segs, n_kv_heads, rope_base, pairing)
    spread, _ = orc.prefill_attention(q, 0, *with_abs, scale=scale)
    reach = 0.0                                          # the largest sum |q_c k_c| * scale (a turn keeps norms: times 2 for the pairs)
    for k in (k_store, k_self):
        if k is not None and len(k):
            group = q.shape[1] // n_kv_heads
            for h in range(q.shape[1]):
                reach = max(reach, (np.abs(q[:, h]) @ np.abs(np.asarray(k[:, h // group], dtype=np.float64)).T).max())
    ds = 2.0 ** -14 * 2 * reach * (1.0 / np.sqrt(128) if scale is None else scale)
    return out, mass, 2 * (2.0 ** -11 + 2 * ds) * spread, (4 * ds + 1e-6) * np.asarray(mass)


class Blocks:
    """A scheduler step of a cache in blocks, by the words of its definition."""

    def __init__(self, table_stride, block, n_blocks, first_token, seg_stride, base_stride=0, max_new=1 << 30, q_stored=0):
        self.table_stride, self.block, self.n_blocks, self.first = table_stride, block, n_blocks, first_token
        self.seg_stride, self.base_stride, self.max_new, self.q_stored = seg_stride, base_stride, max_new, q_stored

    def step(self, cached, fresh, table, free, n_free, position, base=None):
        """-> dict of what is written, and flags.  table, free: arrays, copied; base: list of lists of entries."""
        B, block = len(cached), self.block
        table, stack, flags = np.array(table), [int(x) for x in free[:n_free]], 0
        free_out = np.array(free)
        lost = [c < 0 or -(-c // block) > self.table_stride for c in cached]
        have = [0 if lost[b] else -(-cached[b] // block) for b in range(B)]
        rows = [max(f, 0) for f in fresh]
        bad = [lost[b] or (fresh[b] >= 0 and -(-(cached[b] + rows[b]) // block) > self.table_stride) for b in range(B)]
        for b in range(B):
            if fresh[b] < 0:
                stack += [int(x) for x in table[b, :have[b]]]
        room, taken, n_stack = len(stack), 0, len(stack)
        want = [0 if fresh[b] < 0 or bad[b] else -(-(cached[b] + rows[b]) // block) - have[b] for b in range(B)]
        served, new_ids = [], []
        for b in range(B):
            ok = not bad[b] and (want[b] == 0 or sum(want[:b + 1]) <= room)
            served.append(ok)
            ids = []
            for i in range(want[b] if ok else 0):
                ids.append(stack[n_stack - 1 - (sum(want[:b]) + i)])
            taken += len(ids)
            new_ids.append(ids)
            if bad[b]:
                flags |= cf.CF_FLAG_BAD_INDEX
            elif not ok:
                flags |= cf.CF_FLAG_NO_BLOCKS
        left = room - taken
        for at in range(n_free, left):
            free_out[at] = stack[at]
        out = dict(table=table, free=free_out, next_n_free=left, q_off=[0], q_new=[], slots=[], shift=[], n_seg=[], next_len=[], segs=[])
        good = lambda x: 0 <= x < self.n_blocks
        for b in range(B):
            table[b, have[b]:have[b] + len(new_ids[b])] = new_ids[b]
            ids = [int(x) for x in table[b, :have[b] + len(new_ids[b])]]
            if not all(good(x) for x in new_ids[b]) or (fresh[b] < 0 and not all(good(x) for x in ids)):
                flags |= cf.CF_FLAG_BAD_INDEX
            leaves = fresh[b] < 0
            q_new = position[b] + (0 if leaves or lost[b] else cached[b])
            out["q_new"].append(q_new)
            out["next_len"].append(0 if leaves else cached[b] + rows[b] if served[b] else cached[b])
            for r in range(rows[b]):
                t = cached[b] + r
                ok = served[b] and good(ids[t // block])
                if served[b] and not ok:
                    flags |= cf.CF_FLAG_BAD_INDEX
                out["slots"].append(self.first + ids[t // block] * block + t % block if ok else -1)
                out["shift"].append(q_new - self.q_stored)
            entries = []
            if not leaves:
                if base is not None and not lost[b]:
                    entries += [tuple(e) for e in base[b]]
                j = 0
                while j < have[b]:
                    k = j + 1
                    while k < have[b] and ids[k] == ids[k - 1] + 1:
                        k += 1
                    n, pos = min(k * block, cached[b]) - j * block, position[b] + j * block
                    if ids[j] >= 0 and ids[j] + (k - j) <= self.n_blocks:
                        entries.append((self.first + ids[j] * block, n, pos, pos, cf.CF_SEG_PREFIX, -1))
                    else:
                        entries.append((0, 0, pos, pos, cf.CF_SEG_PREFIX, -1))
                        flags |= cf.CF_FLAG_BAD_INDEX
                    j = k
                if rows[b] and not lost[b]:
                    entries.append((out["q_off"][-1], rows[b], self.q_stored, q_new, cf.CF_SEG_SELF, -1))
            if len(entries) > self.seg_stride:
                flags |= cf.CF_FLAG_BAD_SEGMENT
                entries = []
                out["n_seg"].append(0)
            else:
                out["n_seg"].append(len(entries))
            out["segs"].append(entries)
            out["q_off"].append(out["q_off"][-1] + rows[b])
        if out["q_off"][-1] > self.max_new:
            flags |= cf.CF_FLAG_BAD_INDEX
        out["flags"] = flags
        return out
