"""The 4-bit cache store's operators, as cases that can be timed and compared with their plain forms.

A server that keeps its Context KV Cache Store in 4 bits calls, one `kind` each:

  tables    one scheduler step of a block-wise cache: requests grow, start and leave; block tables, slots of the new
            tokens and segment tables come out (cf_block_tables)
  store     fresh keys and values go to their slots in 4 bits (cf_quantize_cache) and are read back as a 16-bit run
            (cf_assemble_cache_q4): what is held in 4 bits is compared as the values it stands for
  assemble  a query's surviving documents, held in 4 bits, moved and gathered into a 16-bit decode cache
            (cf_assemble_cache_q4)
  decode    one new token per request over its cache in 4 bits, outputs only (cf_prefill_attention_q4)
  layer     a layer's query pre-fill over documents in 4 bits, with their attention mass (cf_prefill_attention_q4)

The 4-bit format, per token and kv head of 128 channels: four groups of 32 channels, each with a scale byte `s` that
stands for 2^(s - 127) (255: every value of the group is NaN) and 16 bytes of codes, the lower four bits first.  A code
is a sign bit and the index of a magnitude in 0, 0.5, 1, 1.5, 2, 3, 4, 6.  The scale of a group with largest magnitude A
is the smallest power of two with A <= 7 * scale, within the exponents at which every value is a number of the 16-bit
type; values round to the nearest magnitude, ties to the one with the even index, past 6 to 6.

With `own` false, `run` computes the same in elementary torch operations, in 32 bits (angles in 64, values next to a
rounding border in 64); with it true it makes the library's calls.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16}
D = 128                                     # channels of a head
E_RANGE = {"bf16": (-125, 125), "f16": (-23, 13)}       # exponents of a group's scale
PREFIX, DOC, SELF = 0, 1, 2                 # kinds of a table entry
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

# head geometries of workloads.CONFIGS: query heads, kv heads, rope base, positions
LLAMA2_7B = dict(hq=32, hkv=32, base=1.0e4, positions=4096)
QWEN2_7B = dict(hq=28, hkv=4, base=1.0e6, positions=32768)
QWEN2_1P5B = dict(hq=12, hkv=2, base=1.0e6, positions=32768)


def listed():
    return [
        # the step of a server with one conversation: it adds a token; once per token, latency only
        dict(name="tables_step_one", kind="tables", batch=1, lo=881, hi=881, new_lo=1, new_hi=1, leave=0.0, block=64, docs=0),
        # continuous batching at its busiest: 512 requests over shared passages, prompts admitted beside running answers, some leave
        dict(name="tables_admit_512", kind="tables", batch=512, lo=0, hi=3000, new_lo=1, new_hi=700, leave=0.05, block=64, docs=5),
        # the newest token of 64 conversations appended to the cache, grouped-query heads
        dict(name="store_append_64", kind="store", **QWEN2_7B, dtype="bf16", pairing="half", layout="head", texts=64, lo=1, hi=1,
             position=2000),
        # offline: thirty passages encoded for one layer written to the store, multi-head attention
        dict(name="store_documents", kind="store", **LLAMA2_7B, dtype="bf16", pairing="half", layout="head", texts=30, lo=160, hi=160,
             position=32),
        # Alg. 2 Phase 2 from a 4-bit store: the passages of one layer into a 16-bit decode cache
        dict(name="assemble_llama2_7b", kind="assemble", **LLAMA2_7B, dtype="bf16", pairing="half", layout="head", batch=1, prefix=32,
             docs=30, lo=160, hi=160, tq=48),
        # eight queries' passages of a model with interleaved pairs, token-major store, unequal lengths
        dict(name="assemble_interleaved_b8", kind="assemble", **QWEN2_1P5B, dtype="f16", pairing="interleaved", layout="token", batch=8,
             prefix=0, docs=8, lo=100, hi=200, tq=21),
        # one new token of one conversation over its cache: the smallest call, made once per layer and token
        dict(name="decode_one", kind="decode", **LLAMA2_7B, dtype="bf16", pairing="half", layout="head", batch=1, lo=881, hi=881, block=0),
        # continuous batching: 32 conversations of unequal length in blocks of 128 tokens
        dict(name="decode_batch_blocks", kind="decode", **QWEN2_7B, dtype="bf16", pairing="half", layout="head", batch=32, lo=1000,
             hi=5000, block=128),
        # four long conversations near the end of the positional range
        dict(name="decode_long", kind="decode", **QWEN2_7B, dtype="bf16", pairing="half", layout="head", batch=4, lo=24000, hi=31000,
             block=0),
        # interactive question answering over ten passages, multi-head attention
        dict(name="layer_llama2_7b", kind="layer", **LLAMA2_7B, dtype="bf16", pairing="half", layout="head", batch=1, prefix=32, docs=10,
             lo=160, hi=160, tq=48, spare=0),
        # a long context: fifty passages, grouped-query heads
        dict(name="layer_qwen2_7b", kind="layer", **QWEN2_7B, dtype="bf16", pairing="half", layout="head", batch=1, prefix=32, docs=50,
             lo=100, hi=200, tq=64, spare=0),
        # throughput serving: 64 queries over a store of 10 000 passages, fp16
        dict(name="layer_qwen2_1p5b_b64", kind="layer", **QWEN2_1P5B, dtype="f16", pairing="half", layout="head", batch=64, prefix=0,
             docs=20, lo=100, hi=200, tq=64, spare=8720),
    ]


def draw(rng):
    """One more case: sizes log-uniform over their ranges, no more work than the largest listed case of its kind."""
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def lengths(lo, hi):
        a = log_int(lo, hi)
        return dict(lo=a, hi=a if rng.random() < 0.3 else min(hi, int(a * rng.uniform(1.1, 2.0)) + 1))

    def cost(c):
        w = work(c)
        return w["bytes"] + w["flops"] / 300

    kind = rng.choice(["tables", "store", "assemble", "decode", "decode", "layer", "layer"])
    limit = max(cost(c) for c in listed() if c["kind"] == kind)
    while True:
        geo = dict(rng.choice([LLAMA2_7B, QWEN2_7B, QWEN2_1P5B]), dtype=rng.choice(["bf16", "bf16", "f16"]),
                   pairing=rng.choice(["half", "half", "half", "interleaved"]), layout=rng.choice(["head", "head", "token"]))
        if kind == "tables":
            c = dict(kind=kind, batch=log_int(1, 512), lo=rng.choice([0, 1, 200]), hi=log_int(300, 4000), new_lo=rng.choice([0, 1]),
                     new_hi=rng.choice([1, 1, 4, log_int(8, 700)]), leave=rng.choice([0.0, 0.0, 0.1]),
                     block=rng.choice([16, 32, 48, 64, 128, 256]), docs=rng.choice([0, 0, 5, 11]))
            c["hi"] = min(c["hi"], 200 * c["block"])
        elif kind == "store":
            c = dict(kind=kind, **geo, texts=log_int(1, 300), **(dict(lo=1, hi=1) if rng.random() < 0.4 else lengths(2, 300)),
                     position=rng.choice([0, 32, 57, 2000]))
        elif kind == "assemble":
            c = dict(kind=kind, **geo, batch=log_int(1, 32), prefix=rng.choice([0, 32, 57]), docs=log_int(1, 50), **lengths(1, 250),
                     tq=log_int(1, 100))
        elif kind == "decode":
            c = dict(kind=kind, **geo, batch=log_int(1, 64), **lengths(1, 30000), block=rng.choice([0, 0, 64, 128]))
            if c["block"]:
                c["hi"] = min(c["hi"], 250 * c["block"])
                c["lo"] = min(c["lo"], c["hi"])
        else:
            c = dict(kind=kind, **geo, batch=log_int(1, 64), prefix=rng.choice([0, 4, 32, 57]), docs=log_int(1, 56), **lengths(1, 260),
                     tq=log_int(1, 130), spare=rng.choice([0, 0, 100]))
        if kind != "tables" and c["hi"] + c.get("tq", 1) + c.get("prefix", 0) + c.get("position", 0) >= c["positions"]:
            continue
        if cost(c) <= limit:
            return c


def work(case):
    """What each path cannot do without: its inputs read once, its outputs written once; 4 * 128 flops per (query head, row, key)."""
    c = case
    mean = 0.5 * (c["lo"] + c["hi"])
    if c["kind"] == "tables":
        new = 0.5 * (c["new_lo"] + c["new_hi"])
        blocks = (mean + new) / c["block"] + 1
        entries = c["docs"] + 2 + mean / c["block"] / 4
        return {"bytes": c["batch"] * (24 + 4 * blocks + 12 * new + 32 * (entries + c["docs"])), "flops": c["batch"] * (blocks + new)}
    kv16, kv4 = 2 * c["hkv"] * D * 2, 2 * c["hkv"] * (D // 2 + D // 32)        # K and V of one token
    if c["kind"] == "store":                # read, written in 4 bits, read again, written in 16
        n = c["texts"] * mean
        return {"bytes": n * (2 * kv16 + 2 * kv4), "flops": n * 8.0 * c["hkv"] * D}
    if c["kind"] == "assemble":
        n = c["batch"] * (c["prefix"] + c["docs"] * mean)
        return {"bytes": n * (kv4 + kv16) + 2 * c["batch"] * c["tq"] * kv16, "flops": n * 3.0 * c["hkv"] * D}
    rows = 1 if c["kind"] == "decode" else c["tq"]
    cached = mean if c["kind"] == "decode" else c["prefix"] + c["docs"] * mean
    return {"bytes": c["batch"] * (cached * kv4 + rows * (kv16 + 2 * c["hq"] * D * 2)),
            "flops": 4.0 * D * c["hq"] * c["batch"] * (rows * cached + rows * (rows + 1) / 2)}


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    return globals()["_prepare_" + case["kind"]](dict(case), int(seed))


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 7919 + 13)


def _dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x).astype(dtype)).cuda()


def _normal(gen, shape, dtype, loud=True):
    """N(0, 1); of keys some channels are four times as loud, as those of trained models are."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    if loud:
        x[..., 5::43] *= 4
    return x.to(TORCH[dtype])


def _encode(x, dtype):
    """[..., 128] float64 -> codes [..., 64] and scale bytes [..., 4] of the format above."""
    g = x.reshape(*x.shape[:-1], 4, 32)
    top = g.abs().amax(-1)
    fraction, exponent = torch.frexp(top)                   # top = fraction * 2^exponent, fraction in [0.5, 1)
    lo, hi = E_RANGE[dtype]
    e = (exponent.to(torch.int32) - 3 + (fraction > 0.875)).clamp(lo, hi)
    e = torch.where(top > 0, e, lo)
    bad = ~torch.isfinite(top)
    y = torch.ldexp(g.abs(), -e[..., None])
    code = torch.zeros(y.shape, dtype=torch.uint8, device=x.device)
    code += y > 0.25
    code += y >= 0.75
    code += y > 1.25
    code += y >= 1.75
    code += y > 2.5
    code += y >= 3.5
    code += y > 5
    code |= torch.signbit(g).to(torch.uint8) << 3
    code = torch.where(bad[..., None], 0, code).reshape(*x.shape[:-1], 64, 2)
    return code[..., 0] | code[..., 1] << 4, torch.where(bad, 255, e + 127).to(torch.uint8)


def _decode(codes, scales):
    """The values that codes [..., 64] and scale bytes [..., 4] stand for, fp32 [..., 128]."""
    both = torch.stack([codes & 15, codes >> 4], dim=-1).reshape(*codes.shape[:-1], 4, 32).to(torch.int64)
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=torch.float32, device=codes.device)
    s = scales.to(torch.int32)
    values = torch.ldexp(table[both], (s - 127)[..., None])
    return torch.where((s == 255)[..., None], float("nan"), values).reshape(*codes.shape[:-1], D)


def _empty_store(c, n_tokens):
    """Codes and scales of keys and values: [tokens][kv heads][.] or, head-major, [kv heads][tokens][.]."""
    lead = (n_tokens, c["hkv"]) if c["layout"] == "token" else (c["hkv"], n_tokens)
    return {x + y: torch.zeros((*lead, n), dtype=torch.uint8, device="cuda") for x in "kv" for y, n in (("_codes", 64), ("_scales", 4))}


def _random_store(c, gen, n_tokens):
    store = _empty_store(c, n_tokens)
    for x in "kv":
        codes, scales = (store[x + y].view(-1, n) for y, n in (("_codes", 64), ("_scales", 4)))
        for at in range(0, codes.shape[0], 1 << 18):
            n = min(1 << 18, codes.shape[0] - at)
            codes[at:at + n], scales[at:at + n] = _encode(_normal(gen, (n, D), c["dtype"], x == "k").float(), c["dtype"])
    return store


ENTRY = np.dtype([("tok_offset", "<i8"), ("len", "<i4"), ("stored_start", "<i4"), ("new_start", "<i4"), ("kind", "<i4"), ("doc", "<i4"),
                  ("reserved", "<i4")])


def _table(rows, stride):
    """[batch][stride] table entries from lists of (tok_offset, len, stored, new, kind, doc)."""
    t = np.zeros((len(rows), stride), dtype=ENTRY)
    for b, entries in enumerate(rows):
        for i, e in enumerate(entries):
            t[b, i] = (*e, 0)
    return t, _dev(t.view(np.uint8).reshape(len(rows), stride, 32), np.uint8), _dev([len(e) for e in rows], np.int32)


def _documents(c, seed):
    """Per query its prefix, its documents — moved from the place they were cached at to places back to back — and its own block."""
    rng = np.random.default_rng(seed)
    b, k = c["batch"], c["docs"]
    n_docs = b * k + c.get("spare", 0)
    lens = rng.integers(c["lo"], c["hi"] + 1, size=n_docs)
    off = c["prefix"] + np.concatenate([[0], np.cumsum(lens)])
    pick = rng.permutation(n_docs)[:b * k].reshape(b, k)
    rows, q_new = [], []
    room = c["positions"] - c["tq"]
    for i in range(b):
        entries = [(0, c["prefix"], 0, 0, PREFIX, -1)] if c["prefix"] else []
        # groups of documents that fit the positional range, each from behind the prefix on
        at, ends = c["prefix"], c["prefix"]
        for slot, d in enumerate(pick[i]):
            n = int(lens[d])
            if at + n > room:
                at = c["prefix"]
            entries.append((int(off[d]), n, c["prefix"], at, DOC, slot))
            at += n
            ends = max(ends, at)
        q_new.append(ends)
        rows.append(entries + [(i * c["tq"], c["tq"], 0, ends, SELF, -1)])
    return rows, q_new, int(off[-1])


def _state(c, gen, rows, q_new, n_tokens, tq):
    """A batch's tensors and tables; every query has `tq` rows that carry local positions."""
    b = len(rows)
    stride = max(len(r) for r in rows)
    table, segs, n_seg = _table(rows, stride)
    s = dict(case=c, store=_random_store(c, gen, n_tokens), n_tokens=n_tokens, table=table, segs=segs, n_seg=n_seg, stride=stride, tq=tq,
             q=_normal(gen, (b * tq, c["hq"], D), c["dtype"]), k_self=_normal(gen, (b * tq, c["hkv"], D), c["dtype"]),
             v_self=_normal(gen, (b * tq, c["hkv"], D), c["dtype"], False), q_off=_dev(np.arange(b + 1) * tq, np.int32),
             q_new=_dev(q_new, np.int32), max_kv=max(sum(e[1] for e in r) for r in rows), max_len=max(e[1] for r in rows for e in r),
             flag=torch.zeros(1, dtype=torch.int32, device="cuda"))
    return s


def _prepare_layer(c, seed):
    rows, q_new, n_tokens = _documents(c, seed)
    s = _state(c, _gen(seed), rows, q_new, n_tokens, c["tq"])
    s["out"] = torch.zeros_like(s["q"])
    s["mass"] = torch.zeros((c["batch"], s["stride"]), dtype=torch.float32, device="cuda")
    return s


def _runs(ids):
    """(first id, number) of every run of ascending neighbours."""
    cut = np.flatnonzero(np.diff(ids) != 1) + 1
    return [(int(r[0]), len(r)) for r in np.split(ids, cut)] if len(ids) else []


def _blocks(rng, n, ids):
    """`n` of the ids, cut into runs of one to eight neighbours in a random order: what a pool hands out after a while."""
    cuts, at = [], 0
    while at < len(ids):
        cuts.append(at)
        at += int(rng.integers(1, 9))
    pieces = np.split(ids, cuts[1:])
    order = rng.permutation(len(pieces))
    return np.concatenate([pieces[i] for i in order])[:n] if n else np.zeros(0, dtype=np.int64)


def _prepare_decode(c, seed):
    rng = np.random.default_rng(seed)
    b, block = c["batch"], c["block"]
    lens = rng.integers(c["lo"], c["hi"] + 1, size=b)
    rows = []
    if block:                               # caches in blocks that lie anywhere in the store
        per = -(-lens // block)
        ids = _blocks(rng, int(per.sum()), np.arange(int(per.sum())))
        first = np.concatenate([[0], np.cumsum(per)])
        for i in range(b):
            entries, done = [], 0
            for at, n in _runs(ids[first[i]:first[i + 1]]):
                m = min(n * block, int(lens[i]) - done)
                entries.append((at * block, m, done, done, PREFIX, -1))
                done += m
            rows.append(entries)
        n_tokens = int(per.sum()) * block
    else:                                   # one run each
        off = np.concatenate([[0], np.cumsum(lens)])
        rows = [[(int(off[i]), int(lens[i]), 0, 0, PREFIX, -1)] for i in range(b)]
        n_tokens = int(off[-1])
    rows = [e + [(i, 1, 0, int(lens[i]), SELF, -1)] for i, e in enumerate(rows)]
    s = _state(c, _gen(seed), rows, [int(n) for n in lens], n_tokens, 1)
    s["out"] = torch.zeros_like(s["q"])
    return s


def _prepare_assemble(c, seed):
    rows, q_new, n_tokens = _documents(c, seed)
    s = _state(c, _gen(seed), rows, q_new, n_tokens, c["tq"])
    total = [sum(e[1] for e in r) for r in rows]
    return dict(s, **_final(c, total, c["batch"] * (c["prefix"] + c["docs"] * c["hi"] + c["tq"])))


def _final(c, total, n):
    """A 16-bit cache [kv head][token][128] with room for n tokens, for runs of these lengths, back to back."""
    at = np.concatenate([[0], np.cumsum(total)])
    zeros = lambda: torch.zeros((c["hkv"], n, D), dtype=TORCH[c["dtype"]], device="cuda")      # noqa: E731
    return dict(capacity=n, longest=int(max(total)), final_off=_dev(at[:-1], np.int64), k_final=zeros(), v_final=zeros(),
                final_len=torch.zeros(len(total), dtype=torch.int32, device="cuda"),
                final_pos=torch.zeros(n, dtype=torch.int32, device="cuda"))


def _prepare_store(c, seed):
    rng, gen = np.random.default_rng(seed), _gen(seed)
    lens = rng.integers(c["lo"], c["hi"] + 1, size=c["texts"])
    total = int(lens.sum())
    start = np.concatenate([[0], np.cumsum(lens)])
    # texts go to places of the store in another order, with gaps between them
    order = rng.permutation(c["texts"])
    place = np.zeros(c["texts"], dtype=np.int64)
    place[order] = np.cumsum(lens[order] + 3) - lens[order]
    n_tokens = total + 3 * c["texts"]
    pos = c["position"] + rng.integers(0, 7, size=c["texts"])
    pos = np.minimum(pos, c["positions"] - lens)
    slots = np.concatenate([place[i] + np.arange(lens[i]) for i in range(c["texts"])])
    rows = [[(int(place[i]), int(lens[i]), int(pos[i]), int(pos[i]), DOC, -1) for i in range(c["texts"])]]
    table, segs, n_seg = _table(rows, c["texts"])
    return dict(case=c, store=_empty_store(c, n_tokens), n_tokens=n_tokens, n=total, slots=_dev(slots, np.int64),
                shift=_dev(np.repeat(pos, lens), np.int32), k=_normal(gen, (total, c["hkv"], D), c["dtype"]),
                v=_normal(gen, (total, c["hkv"], D), c["dtype"], False), table=table, segs=segs, n_seg=n_seg, stride=c["texts"], tq=1,
                q_off=_dev([0, 0], np.int32), max_len=int(lens.max()), k_self=None, v_self=None, start=start,
                flag=torch.zeros(1, dtype=torch.int32, device="cuda"), **_final(c, [total], c["texts"] * c["hi"]))


def _prepare_tables(c, seed):
    rng = np.random.default_rng(seed)
    b, block = c["batch"], c["block"]
    cached = rng.integers(c["lo"], c["hi"] + 1, size=b)
    new = rng.integers(c["new_lo"], c["new_hi"] + 1, size=b)
    if c["new_hi"] > 4:                     # prompts are admitted beside answers that grow by a token
        new = np.where((rng.random(b) < 0.5) & (cached > 0), np.minimum(new, 1), new)
    new = np.where((rng.random(b) < c["leave"]) & (cached > 0), -1, new)
    have = -(-cached // block)
    table_stride = -(-(c["hi"] + max(c["new_hi"], 0)) // block) + 1
    n_blocks = b * table_stride + 5
    ids = _blocks(rng, n_blocks, np.arange(n_blocks))
    table = np.full((b, table_stride), -1, dtype=np.int64)
    first = np.concatenate([[0], np.cumsum(have)])
    for i in range(b):
        table[i, :have[i]] = ids[first[i]:first[i + 1]]
    free = np.zeros(n_blocks, dtype=np.int64)
    n_free = n_blocks - int(have.sum())
    free[:n_free] = ids[first[-1]:][::-1]
    # shared passages ahead of every request's own tokens, whose positions follow
    docs = c["docs"]
    base = [[(32 + 160 * int(d), 160, 32, 32 + 160 * j, DOC, j) for j, d in enumerate(rng.permutation(4 * docs)[:docs])] for _ in range(b)]
    base_np, base_segs, n_base = _table(base, max(docs, 1))
    first_token = 32 + 640 * docs
    capacity = b * c["new_hi"]
    stride = docs + -(-c["hi"] // block) + 1
    zeros = lambda shape, t: torch.zeros(shape, dtype=t, device="cuda")                  # noqa: E731
    i32, i64 = torch.int32, torch.int64
    return dict(case=c, host=dict(cached=cached, new=new, table=table, free=free, n_free=n_free, base=base_np), batch=b, block=block,
                n_blocks=n_blocks, first_token=first_token, table_stride=table_stride, seg_stride=stride, base_stride=max(docs, 1),
                capacity=capacity, cached=_dev(cached, np.int32), new=_dev(new, np.int32), table=_dev(table, np.int32),
                free=_dev(free, np.int32), n_free=_dev([n_free], np.int32), position=_dev(np.full(b, 32 + 160 * docs), np.int32),
                base_segs=base_segs if docs else None, n_base=n_base if docs else None, next_len=zeros(b, i32), next_n_free=zeros(1, i32),
                q_off=zeros(b + 1, i32), q_new=zeros(b, i32), slots=zeros(max(capacity, 1), i64), shift=zeros(max(capacity, 1), i32),
                segs=zeros((b, stride, 32), torch.uint8), n_seg=zeros(b, i32), flag=zeros(1, i32))


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["kind"]](state)


def _handle(s):
    """What a user's program keeps: the layer's geometry, the store and, for attention, a workspace."""
    if "handle" not in s:
        from paper_2502_11101_amd import binding as cf
        c = s["case"]
        strides = (c["hkv"] * D, D) if c["layout"] == "token" else (D, s["n_tokens"] * D)
        desc = cf.make_desc(c["hq"], c["hkv"], D, c["dtype"], c["base"], c["positions"],
                            cf.CF_ROPE_INTERLEAVED if c["pairing"] == "interleaved" else cf.CF_ROPE_HALF,
                            store_token_stride=strides[0], store_head_stride=strides[1])
        store = cf.make_q4_store(*(s["store"][x] for x in ("k_codes", "k_scales", "v_codes", "v_scales")), s["n_tokens"])
        ws, nbytes = None, 0
        if "out" in s:
            nbytes = cf.cf_prefill_workspace_bytes_q4(desc, c["batch"], s["tq"], s["stride"], s["max_kv"])
            ws = torch.zeros(nbytes, dtype=torch.uint8, device="cuda")
        s["handle"] = (cf, desc, store, ws, nbytes)
    return s["handle"]


def _attend(s, mass):
    cf, desc, store, ws, nbytes = _handle(s)
    cf.cf_prefill_attention_q4(desc, s["q"], s["q_off"], 0, s["q_new"], store, s["k_self"], s["v_self"], s["segs"], s["n_seg"], s["stride"],
                               s["case"]["batch"], s["tq"], s["max_kv"], s["out"], mass, None, 1, ws, nbytes, s["flag"])


def _own_layer(s):
    _attend(s, s["mass"])
    return [s["out"], s["mass"], s["flag"]]


def _own_decode(s):
    _attend(s, None)
    return [s["out"], s["flag"]]


def _gather(s, batch):
    cf, desc, store, _, _ = _handle(s)
    cf.cf_assemble_cache_q4(desc, store, s["k_self"], s["v_self"], s["q_off"], s["segs"], s["n_seg"], s["stride"], batch, s["tq"],
                            s["max_len"], s["final_off"], s["capacity"], D, s["capacity"] * D, s["k_final"], s["v_final"], s["final_len"],
                            s["final_pos"], s["flag"])
    return [s["k_final"], s["v_final"], s["final_len"], s["final_pos"], s["flag"]]


def _own_assemble(s):
    return _gather(s, s["case"]["batch"])


def _own_store(s):
    cf, desc, store, _, _ = _handle(s)
    cf.cf_quantize_cache(desc, s["k"], s["v"], s["n"], s["slots"], s["shift"], store, s["flag"])
    return _gather(s, 1)


def _own_tables(s):
    from paper_2502_11101_amd import binding as cf
    cf.cf_block_tables(s["cached"], s["new"], s["batch"], s["block"], s["n_blocks"], s["first_token"], s["table"], s["table_stride"],
                       s["free"], s["n_free"], s["position"], s["base_segs"], s["n_base"], s["base_stride"], 0, s["next_len"],
                       s["next_n_free"], s["q_off"], s["q_new"], s["slots"], s["shift"], s["capacity"], s["segs"], s["n_seg"],
                       s["seg_stride"], s["flag"])
    return _tables_out(s)


def _tables_out(s):
    # of the free list what lies below its top
    return [s["table"], s["free"], s["next_len"], s["next_n_free"], s["q_off"], s["q_new"], s["slots"], s["shift"],
            s["segs"].view(torch.int32), s["n_seg"], s["flag"]]


# ------------------------------------------------------------------------------------------------ plain forms
def _fields(segs):
    """The table entries' fields as int64 tensors [batch][stride]."""
    tok = segs.view(torch.int64)[..., 0]
    rest = segs.view(torch.int32).to(torch.int64)
    return tok, rest[..., 2], rest[..., 3], rest[..., 4], rest[..., 5]


def _theta(c, device):
    """Radians per position of the 64 two-dimensional slices, in 64 bits."""
    return c["base"] ** (-2.0 * torch.arange(64, dtype=torch.float64, device=device) / D)


def _moved(k, cos, sin, pairing):
    """Keys [..., 128] turned by the angles with these cosines and sines [..., 64]."""
    x, y = (k[..., :64], k[..., 64:]) if pairing == "half" else (k[..., 0::2], k[..., 1::2])
    u, w = x * cos - y * sin, x * sin + y * cos
    return torch.cat([u, w], dim=-1) if pairing == "half" else torch.stack([u, w], dim=-1).flatten(-2)


def _listed_tokens(s):
    """Every query's tokens in table order, padded to the longest list: which entry, which place in it, whether it is there."""
    tok, n, stored, new, kind = _fields(s["segs"])
    at = torch.arange(s["stride"], device=tok.device)
    n = torch.where(at < s["n_seg"][:, None], n, 0)
    ends = n.cumsum(1)
    j = torch.arange(s["max_kv"], device=tok.device).expand(n.shape[0], -1).contiguous()
    entry = torch.searchsorted(ends, j, right=True).clamp(max=s["stride"] - 1)
    place = j - (ends - n).gather(1, entry)
    return entry, place, j < ends[:, -1:]


def _rows_of(s, x, tok):
    """Values of the store's keys or values at tokens [...], fp32 [..., kv heads, 128]."""
    codes, scales = s["store"][x + "_codes"], s["store"][x + "_scales"]
    if s["case"]["layout"] == "head":
        codes, scales = codes.transpose(0, 1), scales.transpose(0, 1)
    return _decode(codes[tok], scales[tok])


def _keys_values(s, delta):
    """Every query's keys, moved by `delta` [batch][stride] positions, and values in table order."""
    c = s["case"]
    entry, place, there = _listed_tokens(s)
    tok, _, _, new, kind = _fields(s["segs"])
    own_block = (kind.gather(1, entry) == SELF) & there
    at = torch.where(there, tok.gather(1, entry) + place, 0)
    k, v = (_rows_of(s, x, torch.where(own_block, 0, at)) for x in "kv")
    if s["k_self"] is not None:
        pick = torch.where(own_block, at, 0)
        k = torch.where(own_block[..., None, None], s["k_self"][pick].float(), k)
        v = torch.where(own_block[..., None, None], s["v_self"][pick].float(), v)
    angle = delta.to(torch.float64)[..., None] * _theta(c, delta.device)
    index = entry[..., None].expand(-1, -1, 64)
    cos, sin = angle.cos().float().gather(1, index)[:, :, None], angle.sin().float().gather(1, index)[:, :, None]
    return _moved(k, cos, sin, c["pairing"]), v, entry, place, there, own_block, new.gather(1, entry) + place


def _plain_attention(s):
    c, tq = s["case"], s["tq"]
    b, hkv, group = c["batch"], c["hkv"], c["hq"] // c["hkv"]
    _, _, stored, new, _ = _fields(s["segs"])
    k, v, entry, place, there, own_block, _ = _keys_values(s, new - stored - s["q_new"][:, None])
    q = s["q"].float().reshape(b, tq, hkv, group, D).permute(0, 2, 3, 1, 4).reshape(b, hkv, group * tq, D)
    k, v = (x.permute(0, 2, 1, 3).contiguous() for x in (k, v))
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(D))
    row = torch.arange(tq, device=k.device).repeat(group)
    seen = there[:, None] & (~own_block[:, None] | (place[:, None] <= row[:, None]))
    scores = torch.where(seen[:, None], scores, -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    out = torch.matmul(p, v).reshape(b, hkv, group, tq, D).permute(0, 3, 1, 2, 4).reshape(b * tq, c["hq"], D)
    s["out"].copy_(out)
    return p, entry, there


def _plain_layer(s):
    p, entry, there = _plain_attention(s)
    by_token = torch.where(there, p.sum((1, 2), dtype=torch.float64), 0.0)
    mass = torch.zeros(s["mass"].shape, dtype=torch.float64, device=p.device).scatter_add_(1, entry, by_token)
    s["mass"].copy_(mass)
    return [s["out"], s["mass"], s["flag"]]


def _plain_decode(s):
    _plain_attention(s)
    return [s["out"], s["flag"]]


def _plain_gather(s):
    _, _, stored, new, _ = _fields(s["segs"])
    k, v, _, _, there, _, pos = _keys_values(dict(s, max_kv=s["longest"]), new - stored)
    k, v, pos = k[there], v[there], pos[there]
    s["k_final"][:, :len(k)] = k.transpose(0, 1)
    s["v_final"][:, :len(v)] = v.transpose(0, 1)
    s["final_len"].copy_(there.sum(1))
    s["final_pos"][:len(pos)] = pos
    return [s["k_final"], s["v_final"], s["final_len"], s["final_pos"], s["flag"]]


def _plain_assemble(s):
    return _plain_gather(s)


def _plain_store(s):
    c = s["case"]
    angle = s["shift"].to(torch.float64)[:, None] * _theta(c, s["k"].device)
    # in 64 bits up to the fp32 value that is rounded to 4 bits: next to a border an error would take another code
    k = _moved(s["k"].double(), angle.cos()[:, None], angle.sin()[:, None], c["pairing"]).float()
    for x, values in (("k", k), ("v", s["v"].float())):
        codes, scales = _encode(values, c["dtype"])
        for y, z in (("_codes", codes), ("_scales", scales)):
            to = s["store"][x + y]
            (to if c["layout"] == "token" else to.transpose(0, 1))[s["slots"]] = z
    return _plain_gather(s)


def _plain_tables(s):
    dev, b, block, stride = s["cached"].device, s["batch"], s["block"], s["table_stride"]
    i64 = torch.int64
    cached, raw_new = s["cached"].to(i64), s["new"].to(i64)
    leaves, new = raw_new < 0, raw_new.clamp(min=0)
    have = (cached + block - 1) // block
    j = torch.arange(stride, device=dev)
    held = j < have[:, None]
    # blocks of the requests that leave go on top of the free list, in order
    table, top = s["table"].to(i64), s["n_free"].to(i64)
    returned = (held & leaves[:, None]).reshape(-1)
    n_back = returned.sum()
    place = returned.cumsum(0) - 1
    stack = torch.cat([s["free"].to(i64), torch.zeros(b * stride + 1, dtype=i64, device=dev)])
    stack[torch.where(returned, top + place, len(stack) - 1)] = table.reshape(-1)
    # and the others' new ones come off it, in order, as long as they last
    want = torch.where(leaves, 0, (cached + new + block - 1) // block - have)
    before = want.cumsum(0) - want
    served = before + want <= top + n_back
    want = torch.where(served, want, 0)
    fresh = (j >= have[:, None]) & (j < (have + want)[:, None])
    i = before[:, None] + j - have[:, None]
    table = torch.where(fresh, stack[(top + n_back - 1 - i).clamp(min=0)], table)
    s["next_len"].copy_(torch.where(leaves, 0, torch.where(served, cached + new, cached)))
    n_left = top + n_back - want.sum()
    s["next_n_free"].copy_(n_left)
    at = torch.arange(s["n_blocks"], device=dev)
    s["free"].copy_(torch.where((at >= top) & (at < n_left), stack[at], s["free"]))
    # rows, positions and slots of the new tokens
    s["q_off"][1:].copy_(new.cumsum(0))
    q_new = s["position"] + torch.where(leaves, 0, cached)
    s["q_new"].copy_(q_new)
    row = torch.arange(s["capacity"], device=dev)
    of = torch.searchsorted(new.cumsum(0), row, right=True)
    used, of = of < b, of.clamp(max=b - 1)
    t = cached[of] + row - (new.cumsum(0) - new)[of]
    slot = s["first_token"] + table[of, (t // block).clamp(max=stride - 1)] * block + t % block
    s["slots"][:s["capacity"]] = torch.where(used, torch.where(served[of], slot, -1), s["slots"][:s["capacity"]])
    s["shift"][:s["capacity"]] = torch.where(used, q_new[of].to(torch.int32), s["shift"][:s["capacity"]])
    # entries: the shared passages, runs of neighbouring blocks, the own rows
    last = torch.cat([torch.full((b, 1), -7, dtype=i64, device=dev), table[:, :-1]], dim=1)
    held &= ~leaves[:, None]
    starts = held & ((j == 0) | (table != last + 1))
    run = starts.to(i64).cumsum(1) - 1
    n_run = torch.where(leaves, 0, starts.sum(1))
    n_base = torch.zeros(b, dtype=i64, device=dev) if s["n_base"] is None else s["n_base"].to(i64)
    n_base = torch.where(leaves, 0, n_base)
    wide = s["seg_stride"] + 1              # the last column takes what is not an entry
    out = torch.zeros((b, wide, 4), dtype=i64, device=dev)
    if s["base_segs"] is not None:
        k = min(s["base_stride"], s["seg_stride"])
        keep = torch.arange(k, device=dev) < n_base[:, None]
        out[:, :k] = torch.where(keep[..., None], s["base_segs"].view(i64)[:, :k], 0)
    tokens = (cached[:, None] - j * block).clamp(0, block)
    n_of = torch.zeros((b, stride + 1), dtype=i64, device=dev).scatter_add_(1, torch.where(held, run, stride), torch.where(held, tokens, 0))
    half = lambda lo, hi: (lo & 0xFFFFFFFF) | (hi << 32)                                     # noqa: E731
    pos = s["position"][:, None] + j * block
    run_len = n_of.gather(1, run.clamp(min=0))
    entry = torch.stack([s["first_token"] + table * block, half(run_len, pos), half(pos, torch.full_like(pos, PREFIX)),
                         torch.full_like(pos, half(-1, 0))], dim=-1)
    to = torch.where(starts, n_base[:, None] + run, wide - 1)
    out.scatter_(1, to[..., None].expand(-1, -1, 4), entry)
    mine = torch.stack([new.cumsum(0) - new, half(new, torch.zeros_like(new)), half(q_new.to(i64), torch.full_like(new, SELF)),
                        torch.full_like(new, half(-1, 0))], dim=-1)
    to = torch.where(new > 0, n_base + n_run, wide - 1)
    out.scatter_(1, to[:, None, None].expand(-1, 1, 4), mine[:, None])
    n_seg = n_base + n_run + (new > 0)
    real = torch.arange(wide - 1, device=dev) < n_seg[:, None]
    s["segs"].copy_(torch.where(real[..., None], out[:, :-1], s["segs"].view(i64)).view(torch.uint8))
    s["n_seg"].copy_(n_seg)
    s["table"].copy_(table)
    return _tables_out(s)


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return globals()["_exact_" + case["kind"]](s, dict(case))


def _values64(codes, scales):
    """The format's values by its definition: sign, exponent and mantissa bits of every code."""
    n = torch.stack([codes % 16, codes // 16], dim=-1).flatten(-2).to(torch.float64)
    sign, m = torch.where(n >= 8, -1.0, 1.0), n % 8
    magnitude = torch.where(m < 2, m / 2, (2 + m % 2) / 2 * 2.0 ** (torch.div(m, 2, rounding_mode="floor") - 1))
    s = scales.to(torch.float64).repeat_interleave(32, dim=-1)
    return torch.where(s == 255, math.nan, sign * magnitude * 2.0 ** (s - 127))


def _turned64(x, positions, c):
    """Vectors [n][heads][128] turned by `positions` [n] positions, as complex numbers."""
    x = x.to(torch.float64)
    z = torch.complex(x[..., :64], x[..., 64:]) if c["pairing"] == "half" else torch.view_as_complex(x.reshape(*x.shape[:-1], 64, 2))
    freq = torch.exp(-math.log(c["base"]) * torch.arange(64, dtype=torch.float64, device=x.device) / 64)
    angle = positions.to(torch.float64)[:, None] * freq
    z = z * torch.polar(torch.ones_like(angle), angle)[:, None]
    return torch.cat([z.real, z.imag], dim=-1) if c["pairing"] == "half" else torch.view_as_real(z).flatten(-2)


def _lists64(s, c, b):
    """Query b's keys (turned by their shift), values, entry numbers and, for own tokens, their row (-1: any row sees it)."""
    ks, vs, entry, row, pos = [], [], [], [], []
    for i in range(int(s["n_seg"][b])):
        e = s["table"][b, i]
        a, n = int(e["tok_offset"]), int(e["len"])
        if e["kind"] == SELF:
            k, v = s["k_self"][a:a + n], s["v_self"][a:a + n]
            row += range(n)
        else:
            part = (lambda x: x[a:a + n]) if c["layout"] == "token" else (lambda x: x[:, a:a + n].transpose(0, 1))
            k, v = (_values64(part(s["store"][x + "_codes"]), part(s["store"][x + "_scales"])) for x in "kv")
            row += [-1] * n
        ks.append(_turned64(k, torch.full((n,), int(e["new_start"]) - int(e["stored_start"]), device="cuda"), c))
        vs.append(v.to(torch.float64))
        entry += [i] * n
        pos += range(int(e["new_start"]), int(e["new_start"]) + n)
    dev = lambda x: torch.tensor(x, dtype=torch.int64, device="cuda")                          # noqa: E731
    return torch.cat(ks), torch.cat(vs), dev(entry), dev(row), dev(pos)


def _attention64(s, c):
    outs, masses = [], torch.zeros((c["batch"], s["stride"]), dtype=torch.float64, device="cuda")
    tq, group = s["tq"], c["hq"] // c["hkv"]
    for b in range(c["batch"]):
        k, v, entry, row, _ = _lists64(s, c, b)
        q = _turned64(s["q"][b * tq:(b + 1) * tq], torch.full((tq,), int(s["q_new"][b]), device="cuda"), c)
        out = torch.empty((tq, c["hq"], D), dtype=torch.float64, device="cuda")
        hidden = row[None, :] > torch.arange(tq, device="cuda")[:, None]
        for h in range(c["hq"]):
            w = (q[:, h] @ k[:, h // group].T / math.sqrt(D)).masked_fill(hidden, -math.inf).softmax(-1)
            out[:, h] = w @ v[:, h // group]
            masses[b].index_add_(0, entry, w.sum(0))
        outs.append(out)
    return torch.cat(outs), masses


def _exact_layer(s, c):
    out, mass = _attention64(s, c)
    return [out, mass, None]


def _exact_decode(s, c):
    return [_attention64(s, c)[0], None]


def _exact_assemble(s, c):
    parts = [_lists64(s, c, b) for b in range(c["batch"])]
    k, v = (_padded(torch.cat([p[i] for p in parts]), s["capacity"]).transpose(0, 1) for i in range(2))
    return [k, v, torch.tensor([len(p[2]) for p in parts], device="cuda"), _padded(torch.cat([p[4] for p in parts]), s["capacity"]), None]


def _padded(x, n):
    return torch.cat([x, torch.zeros((n - len(x), *x.shape[1:]), dtype=x.dtype, device=x.device)])


def _exact_store(s, c):
    """The nearest values of the format, found among all of them."""
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64, device="cuda")
    lo, hi = E_RANGE[c["dtype"]]

    def nearest(x):
        x = x.reshape(-1, 4, 32)
        top = x.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(top / 7)).clamp(lo, hi)
        for d in (-1, 0):                   # log2 may be a rounding off: the smallest that holds the largest value
            e = torch.where(top > 7 * 2.0 ** (e + d), (e + d + 1).clamp(lo, hi), e)
        y = (x.abs() / 2.0 ** e).unsqueeze(-1)
        far = (y - grid).abs() + torch.tensor([0, 1e-12] * 4, dtype=torch.float64, device="cuda")    # a tie: the even index
        return (torch.sign(x) * grid[far.argmin(-1)] * 2.0 ** e).reshape(-1, D)

    k = _turned64(s["k"], s["shift"], c).float().to(torch.float64)
    out = []
    for x in (k, s["v"].to(torch.float64)):
        flat = x.reshape(-1, D)
        y = torch.cat([nearest(flat[a:a + (1 << 14)]) for a in range(0, flat.shape[0], 1 << 14)])
        out.append(_padded(y.reshape(x.shape), s["capacity"]).transpose(0, 1))
    pos = np.concatenate([np.arange(e["new_start"], e["new_start"] + e["len"]) for e in s["table"][0]])
    return [*out, torch.tensor([s["n"]], device="cuda"), _padded(torch.from_numpy(pos).cuda(), s["capacity"]), None]


def _exact_tables(s, c):
    """The same step, request by request."""
    h, block = s["host"], s["block"]
    table, stack, free = h["table"].copy(), list(h["free"][:h["n_free"]]), h["free"].copy()
    q_off, q_new, n_seg, next_len = [0], [], [], []
    position = int(s["position"][0])
    entries = np.zeros((s["batch"], s["seg_stride"]), dtype=ENTRY)
    slots, shift = [], []
    for b, (old, new) in enumerate(zip(h["cached"], h["new"])):
        if new < 0:
            stack += list(table[b, :-(-old // block)])
    for b, (old, new) in enumerate(zip(h["cached"], h["new"])):
        old, rows = int(old), max(int(new), 0)
        q_off.append(q_off[-1] + rows)
        if new < 0:
            q_new.append(position)
            n_seg.append(0)
            next_len.append(0)
            continue
        have, need = -(-old // block), -(-(old + rows) // block)
        assert need - have <= len(stack)    # the pool of every case lasts
        for i in range(have, need):
            table[b, i] = stack.pop()
        q_new.append(position + old)
        next_len.append(old + rows)
        for t in range(old, old + rows):
            slots.append(s["first_token"] + int(table[b, t // block]) * block + t % block)
            shift.append(position + old)
        list_b = [tuple(e) for e in h["base"][b][:c["docs"]]]
        done = 0
        for at, n in _runs(table[b, :have]):
            m = min(n * block, old - done)
            list_b.append((s["first_token"] + at * block, m, position + done, position + done, PREFIX, -1, 0))
            done += m
        if rows:
            list_b.append((q_off[b], rows, 0, position + old, SELF, -1, 0))
        for i, e in enumerate(list_b):
            entries[b, i] = e
        n_seg.append(len(list_b))
    if len(stack) > h["n_free"]:
        free[h["n_free"]:len(stack)] = stack[h["n_free"]:]
    pad = lambda x, n: x + [0] * (n - len(x))                                                # noqa: E731
    out = [table, free, next_len, [len(stack)], q_off, q_new, pad(slots, max(s["capacity"], 1)), pad(shift, max(s["capacity"], 1)),
           entries.view(np.int32).reshape(s["batch"], s["seg_stride"], 8), n_seg]
    return [torch.from_numpy(np.asarray(x).astype(np.int64)).cuda() for x in out] + [None]
