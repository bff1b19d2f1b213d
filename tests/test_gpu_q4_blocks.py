"""Block tables, slots and segment tables of a scheduler step (cf_block_tables) against the step worked out request by request, and a
decode loop that uses them: tables, attention over the blocks, new tokens appended in 4 bits."""

import numpy as np
import pytest
import torch

from oracle import cachefocus_oracle as orc
from paper_2502_11101_amd import binding as cf
from paper_2502_11101_amd import pipeline as pl
from paper_2502_11101_amd import workloads as wl
from tests import q4_reference as R

pytestmark = pytest.mark.gpu

i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def run_step(ref, cached, fresh, table, free, n_free, position, base=None, use_position=True):
    """One call with everything that is not written preset, compared with the definition; returns the reference's result."""
    B = len(cached)
    want = ref.step(cached, fresh, table, free, n_free, position, base)
    d_table, d_free, flag = i32(table), i32(free), i32([0])
    next_len, next_free, q_off, q_new, n_seg = i32([-9] * B), i32([-9]), i32([-9] * (B + 1)), i32([-9] * B), i32([-9] * B)
    cap = min(ref.max_new, sum(max(f, 0) for f in fresh) + 5)
    slots, shift = torch.full((cap + 3,), -77, dtype=torch.int64, device="cuda"), i32([-77] * (cap + 3))
    segs = torch.full((B, ref.seg_stride, 32), 0xEE, dtype=torch.uint8, device="cuda")
    base_segs = n_base = None
    if base is not None:
        rows = [e for b in base for e in list(b) + [(0, 0, 0, 0, 0, -1)] * (ref.base_stride - len(b))]
        base_segs, n_base = cf.segments_to_device(cf.segments_array(rows)), i32([len(b) for b in base])
    args = (i32(cached), i32(fresh), B, ref.block, ref.n_blocks, ref.first, d_table, ref.table_stride, d_free, i32([n_free]),
            i32(position) if use_position else None, base_segs, n_base, ref.base_stride, ref.q_stored, next_len, next_free, q_off, q_new, slots, shift,
            cap, segs, n_seg, ref.seg_stride, flag)
    cf.cf_block_tables(*args)
    torch.cuda.synchronize()
    assert int(flag.item()) == want["flags"]
    assert next_free.item() == want["next_n_free"]
    for got, name in ((next_len, "next_len"), (q_off, "q_off"), (q_new, "q_new"), (n_seg, "n_seg")):
        assert got.tolist() == want[name], name
    assert np.array_equal(d_table.cpu().numpy(), want["table"]) and np.array_equal(d_free.cpu().numpy(), want["free"])
    n = min(len(want["slots"]), cap)
    assert slots[:n].tolist() == want["slots"][:n] and shift[:n].tolist() == want["shift"][:n]
    assert (slots[n:] == -77).all() and (shift[n:] == -77).all()
    for b in range(B):
        k = want["n_seg"][b]
        got = cf.segments_from_device(segs[b], k)
        assert [tuple(int(x) for x in e)[:6] for e in got] == want["segs"][b] and all(e["reserved"] == 0 for e in got)
        if k or want["flags"] == 0:
            assert (segs[b, k:] == 0xEE).all()
    return want


def pool(rng, B, block, cached, table_stride, spare):
    """A table of distinct blocks for the cached tokens, and the free list of the rest."""
    have = [-(-c // block) for c in cached]
    n_blocks = sum(have) + spare
    ids = rng.permutation(n_blocks)
    if rng.random() < 0.5:
        ids = np.concatenate([p for p in np.array_split(np.sort(ids), max(1, n_blocks // 4))][::-1])
    table, at = np.full((B, table_stride), -3), 0
    for b, n in enumerate(have):
        table[b, :n] = ids[at:at + n]
        at += n
    free = np.full(n_blocks, -5)
    free[:spare] = ids[at:]
    return table, free, spare, n_blocks


@pytest.mark.parametrize("seed,B,block,most,new,leave", [
    (0, 1, 16, 0, 1, 0.0), (1, 1, 64, 900, 1, 0.0), (2, 3, 1, 20, 3, 0.3), (3, 7, 48, 700, 90, 0.3), (4, 64, 32, 900, 1, 0.2),
    (5, 257, 16, 400, 40, 0.2), (6, 600, 128, 3000, 2, 0.1), (7, 5, 16, 5000, 700, 0.0), (8, 33, 7, 300, 20, 0.9), (9, 1000, 64, 200, 0, 1.0)])
def test_steps(seed, B, block, most, new, leave):
    rng = np.random.default_rng(seed)
    cached = [int(x) for x in rng.integers(0, most + 1, size=B)]
    fresh = [int(x) for x in rng.integers(0, new + 1, size=B)]
    fresh = [-int(rng.integers(1, 9)) if rng.random() < leave else f for f in fresh]
    table_stride = -(-(most + new) // block) + 1
    table, free, n_free, n_blocks = pool(rng, B, block, cached, table_stride, B * (-(-new // block) + 1))
    ref = R.Blocks(table_stride, block, n_blocks, 1000, min(table_stride + 4, 4000), base_stride=3, q_stored=2)
    base = [[(int(rng.integers(0, 900)), 100, 32, 40, cf.CF_SEG_DOC, i) for i in range(int(rng.integers(0, 4)))] for _ in range(B)]
    position = [int(x) for x in rng.integers(0, 3000, size=B)]
    want = run_step(ref, cached, fresh, table, free, n_free, position, base)
    # the next step goes on from what was written
    fresh = [0 if rng.random() < 0.5 else 1 for _ in range(B)]
    run_step(ref, want["next_len"], fresh, want["table"], want["free"], want["next_n_free"], position, base)


@pytest.mark.parametrize("spare", [0, 1, 2, 5, 300])
def test_a_pool_that_runs_short(spare):
    rng = np.random.default_rng(spare)
    for B in (3, 300):
        cached = [int(x) for x in rng.integers(0, 40, size=B)]
        fresh = [int(x) for x in rng.integers(0, 30, size=B)]
        fresh = [-1 if rng.random() < 0.1 and spare > 1 else f for f in fresh]
        table, free, n_free, n_blocks = pool(rng, B, 8, cached, 10, spare)
        run_step(R.Blocks(10, 8, n_blocks, 0, 12), cached, fresh, table, free, n_free, [0] * B, use_position=False)


def test_bad_lengths_ids_and_room():
    table = np.array([[0, 1, 2, 3], [4, 5, 0, 0], [6, 0, 0, 0], [7, 0, 0, 0]])
    free = np.array([8, 9, 10, 11] + [0] * 8)
    ref = R.Blocks(4, 4, 12, 0, 6)
    # no room in the table, a negative length, more tokens than the table holds, and a request that is fine among them
    run_step(ref, [16, 3, 4, 4], [1, 2, 0, 3], table, free, 4, [0] * 4)
    run_step(ref, [16, -3, 17, 4], [0, 2, 1, 3], table, free, 4, [0] * 4)
    run_step(ref, [16, -3, 17, 4], [0, -1, -1, 3], table, free, 4, [0] * 4)
    # ids outside the pool: held, handed out, given back
    bad = table.copy()
    bad[1, 1], bad[2, 0] = 99, -4
    run_step(ref, [16, 7, 4, 4], [0, 1, 1, 1], bad, free, 4, [0] * 4)
    run_step(ref, [16, 7, 4, 4], [0, -1, -1, 0], bad, free, 4, [0] * 4)
    wrong = free.copy()
    wrong[3] = 12
    run_step(ref, [16, 3, 4, 4], [0, 2, 1, 1], table, wrong, 4, [0] * 4)
    # more fresh tokens than there is room for, more entries than the segment table takes
    run_step(R.Blocks(4, 4, 12, 0, 6, max_new=3), [4, 3, 4, 4], [1, 2, 1, 3], table, free, 4, [0] * 4)
    run_step(R.Blocks(4, 4, 12, 0, 1), [4, 3, 4, 4], [1, 2, 0, 3], table, free, 4, [0] * 4)


def _texts(rng, n, heads, dtype):
    return wl.round_to_dtype(rng.standard_normal((n, heads, 128), dtype=np.float32), dtype)


@pytest.mark.parametrize("dtype,hq,hkv,pairing,layout,captured", [
    ("bf16", 4, 2, "half", "head", False), ("f16", 2, 2, "interleaved", "token", False), ("bf16", 14, 2, "half", "head", True)])
def test_a_serving_loop(dtype, hq, hkv, pairing, layout, captured):
    """Requests over shared documents start, grow token by token, leave and are replaced, two layers each: every step's output of every
    layer against the oracle on what the caches stand for.  `captured`: the decode step is one graph, replayed."""
    rng = np.random.default_rng(hq)
    B, block, layers, base_rope, positions = 3, 16, 2, 1.0e4, 4096
    kind = {"half": cf.CF_ROPE_HALF, "interleaved": cf.CF_ROPE_INTERLEAVED}[pairing]
    n_shared, n_blocks = 90, 12
    stores = [pl.Q4Store(hq, hkv, dtype, base_rope, positions, n_shared + n_blocks * block, layout, kind) for _ in range(layers)]
    held = []                                            # per layer: the store's values as the GPU wrote them are read back below
    for s in stores:
        s.write(pl.to_device(_texts(rng, n_shared, hkv, dtype), dtype), pl.to_device(_texts(rng, n_shared, hkv, dtype), dtype),
                torch.arange(n_shared, device="cuda"))
    base = [[(0, 10, 0, 0, cf.CF_SEG_PREFIX, -1), (10, 30, 10, 10, cf.CF_SEG_DOC, 0), (50, 40, 10, 40, cf.CF_SEG_DOC, 1)],
            [(0, 10, 0, 0, cf.CF_SEG_PREFIX, -1), (50, 40, 10, 10, cf.CF_SEG_DOC, 0)], [(0, 10, 0, 0, cf.CF_SEG_PREFIX, -1)]]
    rows = [e for b in base for e in b + [(0, 0, 0, 0, 0, -1)] * (3 - len(b))]
    start = [80, 50, 10]
    cache = pl.BlockCache(stores[0].desc, B, block, n_blocks, 60, 21, n_shared, cf.segments_to_device(cf.segments_array(rows)),
                          i32([len(b) for b in base]), 3, 80, i32(start))
    own_k = [[np.zeros((0, hkv, 128)) for _ in range(B)] for _ in range(layers)]     # what each request's cache stands for, by the reference
    own_v = [[np.zeros((0, hkv, 128)) for _ in range(B)] for _ in range(layers)]

    def values(s):
        get = lambda t: t.cpu().numpy() if layout == "token" else t.cpu().numpy().transpose(1, 0, 2)
        return R.decode(get(s.k_codes), get(s.k_scales)), R.decode(get(s.v_codes), get(s.v_scales))

    shared = [tuple(x[:n_shared] for x in values(s)) for s in stores]
    fresh_dev = i32([0] * B)
    most = B * 21
    bufs = [[torch.zeros((most, h, 128), dtype=pl.TORCH_DTYPE[dtype], device="cuda") for h in (hq, hkv, hkv, hq)] for _ in range(layers)]

    def issue():
        cache.step(fresh_dev)
        for s, (q, k, v, out) in zip(stores, bufs):
            cache.attend(s, q, k, v, out)
            cache.append(s, k, v)

    lens, graph = [0] * B, None
    plan = [[20, 3, 1], [1, 1, 1], [1, 1, 1], [1, 0, 1], [-1, 1, 16], [5, 1, 1], [1, -2, 1], [1, 7, 1]] if not captured else \
        [[20, 3, 1], [1, 1, 1]] + [[1, 1, 1], [1, 0, 1], [1, 1, 1], [1, 1, 0], [1, 1, 1], [1, 1, 1]]
    for step, fresh in enumerate(plan):
        n = [max(f, 0) for f in fresh]
        fresh_dev.copy_(i32(fresh))
        host = [(_texts(rng, sum(n), hq, dtype), _texts(rng, sum(n), hkv, dtype), _texts(rng, sum(n), hkv, dtype)) for _ in range(layers)]
        for x, b in zip(host, bufs):
            for y, t in zip(x, b):
                t[:sum(n)].copy_(pl.to_device(y, dtype))
        if captured and step >= 2:
            if graph is None:
                torch.cuda.synchronize()
                # two steps per graph: a step swaps its lengths with those it writes
                graph = []
                state = (cache.len, cache.next_len, cache.n_free, cache.next_n_free)
                for _ in range(2):
                    g = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(g):
                        issue()
                    graph.append(g)
                cache.len, cache.next_len, cache.n_free, cache.next_n_free = state
            graph[step & 1].replay()
            cache.len, cache.next_len = cache.next_len, cache.len
            cache.n_free, cache.next_n_free = cache.next_n_free, cache.n_free
        else:
            issue()
        torch.cuda.synchronize()
        assert cache.flags() == 0
        for i in range(layers):
            q, k, v = host[i]
            got = bufs[i][3][:sum(n)].double().cpu().numpy()
            at = 0
            for b in range(B):
                part = slice(at, at + n[b])
                at += n[b]
                if n[b] == 0:
                    continue
                pos = start[b] + lens[b]
                ks = np.concatenate([shared[i][0], own_k[i][b]])
                vs = np.concatenate([shared[i][1], own_v[i][b]])
                segs = [orc.Segment(*e) for e in base[b]]
                if lens[b]:
                    segs.append(orc.Segment(n_shared, lens[b], start[b], start[b], orc.KIND_PREFIX, -1))
                segs.append(orc.Segment(part.start, n[b], 0, pos, orc.KIND_SELF, -1))
                ref, _, off, _ = R.attention(q[part], pos, ks, vs, k, v, segs, hkv, base_rope, pairing)
                assert (np.abs(got[part] - ref) <= R.HALF_STEP[dtype] * np.abs(ref) + off + 1e-6).all(), (step, i, b)
                moved = R.turned(k[part], pos, base_rope, pairing).astype(np.float32)
                for cache_of, x in ((own_k, moved), (own_v, v[part])):
                    c, sc, _ = R.encode(x, dtype)
                    cache_of[i][b] = np.concatenate([cache_of[i][b], R.decode(c, sc)])
            # what is stored is what the reference stores (but for values next to a border of the format)
            stored = values(stores[i])
            table = cache.table.cpu().numpy()
            for b in range(B):
                if fresh[b] < 0:
                    own_k[i][b] = own_v[i][b] = np.zeros((0, hkv, 128))
                    continue
                m = lens[b] + n[b]
                tok = [n_shared + int(table[b, t // block]) * block + t % block for t in range(m)]
                assert np.array_equal(stored[1][tok], own_v[i][b])
                assert (stored[0][tok] == own_k[i][b]).mean() > 0.999 if m else True
                own_k[i][b] = stored[0][tok]
        lens = [0 if fresh[b] < 0 else lens[b] + n[b] for b in range(B)]
        assert cache.len.tolist() == lens
    used = sum(-(-x // block) for x in lens)
    assert cache.n_free.item() == n_blocks - used
