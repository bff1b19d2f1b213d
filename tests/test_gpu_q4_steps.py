"""Scheduler steps whose fresh tokens do not fit (cf_block_tables with max_fresh): refused requests keep what they hold, the others' tables
are those of a step without them, and the steps that follow attend to stored tokens only."""

import numpy as np
import pytest
import torch

from oracle import cachefocus_oracle as orc
from paper_2502_11101_amd import binding as cf
from paper_2502_11101_amd import pipeline as pl
from paper_2502_11101_amd import workloads as wl
from tests import q4_reference as R
from tests.test_gpu_q4_blocks import i32, pool, run_step

pytestmark = pytest.mark.gpu


def limited_step(ref, max_fresh, room, cached, fresh, table, free, n_free, position, base):
    """The step by its definition: refused requests add nothing to the plain step; rows lie where `fresh` says."""
    B = len(cached)
    rows = [max(f, 0) for f in fresh]
    ends = np.cumsum(rows)
    over = [rows[b] > 0 and (rows[b] > max_fresh or ends[b] > room) for b in range(B)]
    want = ref.step(cached, [0 if over[b] else fresh[b] for b in range(B)], table, free, n_free, position, base)
    slots, shift, at = [], [], 0
    for b in range(B):
        n = 0 if over[b] else rows[b]
        slots += [-1] * rows[b] if over[b] else want["slots"][at:at + n]
        shift += [want["q_new"][b] - ref.q_stored] * rows[b]
        at += n
        first = int(ends[b]) - rows[b]
        want["segs"][b] = [] if over[b] else [(first, *e[1:]) if e[4] == cf.CF_SEG_SELF else e for e in want["segs"][b]]
        want["n_seg"][b] = len(want["segs"][b])
    want.update(slots=slots[:room], shift=shift[:room], q_off=[0] + [min(int(e), room) for e in ends],
                flags=want["flags"] | (cf.CF_FLAG_BAD_INDEX if any(over) else 0))
    return want, over


@pytest.mark.parametrize("seed,B,most,max_fresh,share,spare", [
    (0, 1, 5, 4, 1.0, 30), (1, 6, 40, 20, 0.6, 100), (2, 6, 40, 60, 0.6, 100), (3, 300, 30, 25, 0.5, 4000), (4, 600, 9, 9, 0.9, 300),
    (5, 300, 30, 31, 0.0, 4000), (6, 513, 3, 2, 2.0, 9000), (7, 40, 30, 25, 0.7, 15)])
def test_rows_past_the_limits(seed, B, most, max_fresh, share, spare):
    """`share`: the step's room for rows, as a share of the rows that it is given."""
    rng = np.random.default_rng(seed)
    block, stride = 8, 12
    cached = [int(x) for x in rng.integers(0, 50, size=B)]
    fresh = [int(x) for x in rng.integers(0, most + 1, size=B)]
    fresh = [-1 if rng.random() < 0.1 else f for f in fresh]
    if B == 1:
        fresh = [most]
    room = int(share * sum(max(f, 0) for f in fresh))
    table, free, n_free, n_blocks = pool(rng, B, block, cached, stride, spare)
    ref = R.Blocks(stride, block, n_blocks, 500, stride + 4, base_stride=2, q_stored=3)
    base = [[(int(rng.integers(0, 400)), 100, 32, 40, cf.CF_SEG_DOC, i) for i in range(int(rng.integers(0, 3)))] for _ in range(B)]
    position = [int(x) for x in rng.integers(0, 3000, size=B)]
    want, over = limited_step(ref, max_fresh, room, cached, fresh, table, free, n_free, position, base)
    assert any(over) or share > 1
    d_table, d_free, flag = i32(table), i32(free), i32([0])
    next_len, next_free, q_off, q_new, n_seg = i32([-9] * B), i32([-9]), i32([-9] * (B + 1)), i32([-9] * B), i32([-9] * B)
    slots, shift = torch.full((room + 3,), -77, dtype=torch.int64, device="cuda"), i32([-77] * (room + 3))
    segs = torch.full((B, ref.seg_stride, 32), 0xEE, dtype=torch.uint8, device="cuda")
    rows = [e for b in base for e in list(b) + [(0, 0, 0, 0, 0, -1)] * (2 - len(b))]
    cf.cf_block_tables(i32(cached), i32(fresh), B, block, n_blocks, 500, d_table, stride, d_free, i32([n_free]), i32(position),
                       cf.segments_to_device(cf.segments_array(rows)), i32([len(b) for b in base]), 2, 3, next_len, next_free, q_off, q_new,
                       slots, shift, room, segs, n_seg, ref.seg_stride, flag, max_fresh=max_fresh)
    torch.cuda.synchronize()
    assert int(flag.item()) == want["flags"] and next_free.item() == want["next_n_free"]
    for got, name in ((next_len, "next_len"), (q_off, "q_off"), (q_new, "q_new"), (n_seg, "n_seg")):
        assert got.tolist() == want[name], name
    assert np.array_equal(d_table.cpu().numpy(), want["table"]) and np.array_equal(d_free.cpu().numpy(), want["free"])
    n = len(want["slots"])
    assert slots[:n].tolist() == want["slots"] and shift[:n].tolist() == want["shift"]
    assert (slots[n:] == -77).all() and (shift[n:] == -77).all()
    for b in range(B):
        got = cf.segments_from_device(segs[b], want["n_seg"][b])
        assert [tuple(int(x) for x in e)[:6] for e in got] == want["segs"][b]


@pytest.mark.parametrize("fresh", [[3, 9, 4], [4, 4, 9], [9, 4, 4], [30, 1, 1], [1, 1, 30]])
def test_a_cache_goes_on_after_a_step_with_too_many_rows(fresh):
    """BlockCache: requests with more than max_new rows are refused, nothing is written behind the step's buffers, and the next step's outputs
    are the attention over what is stored."""
    rng = np.random.default_rng(sum(fresh))
    B, block, heads, dtype, base_rope, max_new = 3, 4, 2, "bf16", 1.0e4, 4
    n_blocks = 12
    s = pl.Q4Store(heads, heads, dtype, base_rope, 4096, n_blocks * block)
    cache = pl.BlockCache(s.desc, B, block, n_blocks, 24, max_new)
    normal = lambda n: wl.round_to_dtype(rng.standard_normal((n, heads, 128), dtype=np.float32), dtype)
    own_k, own_v = [np.zeros((0, heads, 128))] * B, [np.zeros((0, heads, 128))] * B
    lens = [0] * B
    refused_once = False
    for step, n in enumerate(([2, 4, 1], fresh, [1, 4, 3])):
        host = [normal(cache.max_rows) for _ in range(3)]
        dev = [pl.to_device(x, dtype) for x in host]
        out = torch.full((cache.max_rows + 8, heads, 128), 55.0, dtype=torch.bfloat16, device="cuda")
        cache.dev_flag.zero_()
        cache.step(i32(n))
        cache.attend(s, *dev, out)
        cache.append(s, dev[1], dev[2])
        torch.cuda.synchronize()
        over = [n[b] > max_new or sum(n[:b + 1]) > cache.max_rows for b in range(B)]
        refused_once |= any(over)
        assert cache.flags() == (cf.CF_FLAG_BAD_INDEX if any(over) else 0)
        assert bool((out[cache.max_rows:] == 55).all())
        got, at = out.double().cpu().numpy(), 0
        codes = [x.cpu().numpy().transpose(1, 0, 2) for x in (s.k_codes, s.k_scales, s.v_codes, s.v_scales)]
        for b in range(B):
            part = slice(at, at + n[b])
            at += n[b]
            if over[b]:
                shown = range(part.start, min(part.start + max_new, part.stop, cache.max_rows))
                assert (got[shown] == 0).all()
                continue
            segs = [orc.Segment(0, lens[b], 0, 0, orc.KIND_PREFIX, -1)] if lens[b] else []
            segs.append(orc.Segment(part.start, n[b], 0, lens[b], orc.KIND_SELF, -1))
            ref, _, off, _ = R.attention(host[0][part], lens[b], own_k[b], own_v[b], host[1], host[2], segs, heads, base_rope)
            assert (np.abs(got[part] - ref) <= R.HALF_STEP[dtype] * np.abs(ref) + off + 1e-6).all(), (step, b)
            lens[b] += n[b]
            table = cache.table[b].tolist()
            tok = [table[t // block] * block + t % block for t in range(lens[b])]
            own_k[b], own_v[b] = R.decode(codes[0][tok], codes[1][tok]), R.decode(codes[2][tok], codes[3][tok])
            moved = R.turned(host[1][part], lens[b] - n[b], base_rope).astype(np.float32)
            assert np.array_equal(own_v[b][-n[b]:], R.decode(*R.encode(host[2][part], dtype)[:2]))
            assert (own_k[b][-n[b]:] == R.decode(*R.encode(moved, dtype)[:2])).mean() > 0.999
        assert cache.len.tolist() == lens
        assert cache.n_free.item() == n_blocks - sum(-(-x // block) for x in lens)
    assert refused_once


def test_the_largest_step():
    """8192 requests with room for 4095 blocks each: some hold all of them, some of those leave, and the newcomers take theirs."""
    rng = np.random.default_rng(7)
    B, stride, block = 8192, 4095, 2
    cached = [int(x) for x in rng.integers(0, 7, size=B)]
    fresh = [int(x) for x in rng.integers(0, 3, size=B)]
    for b in (0, 1, 4000, 8190, 8191):
        cached[b] = stride * block - b % 2               # full, or with room for one more token
        fresh[b] = b % 2
    for b in (1, 77, 300, 4000, 5000, 8191):
        fresh[b] = -1
    fresh[200] = 6000
    have = [-(-c // block) for c in cached]
    spare = 50                                           # far less than is taken: most comes from the requests that leave
    first = np.concatenate([[0], np.cumsum(have)])
    n_blocks = int(first[-1]) + spare
    table = np.full((B, stride), -3)
    for b in range(B):
        table[b, :have[b]] = np.arange(first[b], first[b + 1])
    free = np.full(n_blocks, -5)
    free[:spare] = first[-1] + rng.permutation(spare)
    want = run_step(R.Blocks(stride, block, n_blocks, 9, 3), cached, fresh, table, free, spare, [0] * B, use_position=False)
    assert want["flags"] == 0 and want["next_n_free"] > 0
