"""Refusals of the calls on a 4-bit cache store and of the block tables: host arguments are checked before any HIP call, so this runs
without a GPU.  And pins of the plain definitions that the GPU tests compare with."""

import ctypes as C

import numpy as np
import pytest

from paper_2502_11101_amd import binding as cf
from paper_2502_11101_amd import pipeline as pl
from tests import q4_reference as R

FAKE = 0x10000      # never dereferenced: validation fails first


def _desc(**kw):
    a = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, dtype="bf16", rope_base=1.0e4, max_positions=4096)
    a.update(kw)
    return cf.make_desc(**a)


def _store(**kw):
    a = dict(k_codes=FAKE, k_scales=FAKE, v_codes=FAKE, v_scales=FAKE, n_tokens=100)
    a.update(kw)
    return cf.make_q4_store(**a)


def _status(fn, **k):
    with pytest.raises(cf.CacheFocusError) as e:
        fn(**k, stream=0)
    assert e.value.message
    return e.value.status


INVALID, UNSUPPORTED, RANGE, WORKSPACE = cf.CF_ERR_INVALID_ARG, cf.CF_ERR_UNSUPPORTED, cf.CF_ERR_RANGE, cf.CF_ERR_WORKSPACE
BAD_DESCS = [(dict(dtype="f32"), UNSUPPORTED), (dict(head_dim=64), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED),
             (dict(store_token_stride=192, store_head_stride=12800), INVALID), (dict(store_token_stride=128, store_head_stride=12808), INVALID),
             (dict(n_q_heads=7), INVALID), (dict(rope_base=0.5), INVALID)]
BAD_STORES = [dict(k_codes=None), dict(k_scales=None), dict(v_codes=None), dict(v_scales=None), dict(n_tokens=-1), dict(k_codes=FAKE + 8),
              dict(v_scales=FAKE + 4)]


def _quantize(**kw):
    a = dict(desc=_desc(), k=FAKE, v=FAKE, n_tokens=4, slots=FAKE, shift=None, store=_store())
    a.update(kw)
    return _status(cf.cf_quantize_cache, **a)


def _attend(**kw):
    a = dict(desc=_desc(), q=FAKE, q_off=FAKE, q_stored_start=0, q_new_start=FAKE, store=_store(), k_self=FAKE, v_self=FAKE, segs=FAKE,
             n_seg=FAKE, seg_stride=4, batch=1, max_tq=8, max_kv_tokens=100, out=FAKE, mass=FAKE, score_accum=None, score_stride=0,
             workspace=FAKE, workspace_bytes=1 << 40)
    a.update(kw)
    return _status(cf.cf_prefill_attention_q4, **a)


def _assemble(**kw):
    a = dict(desc=_desc(), store=_store(), k_self=FAKE, v_self=FAKE, q_off=FAKE, segs=FAKE, n_seg=FAKE, seg_stride=4, batch=1, max_tq=8,
             max_seg_len=10, final_off=FAKE, final_capacity=100, final_token_stride=128, final_head_stride=12800, k_final=2 * FAKE,
             v_final=3 * FAKE, final_len=FAKE)
    a.update(kw)
    return _status(cf.cf_assemble_cache_q4, **a)


def _tables(**kw):
    a = dict(cached=FAKE, fresh=FAKE, batch=2, block_tokens=16, n_blocks=8, first_token=0, table=FAKE, table_stride=4, free_blocks=FAKE,
             n_free=FAKE, position=None, base_segs=None, n_base=None, base_stride=0, q_stored_start=0, next_len=2 * FAKE,
             next_n_free=2 * FAKE, q_off=FAKE, q_new_start=FAKE, slots=FAKE, shift=FAKE, max_new_tokens=8, segs=FAKE, n_seg=FAKE, seg_stride=6)
    a.update(kw)
    return _status(cf.cf_block_tables, **a)


@pytest.mark.parametrize("bad,code", BAD_DESCS)
def test_descriptors(bad, code):
    assert _quantize(desc=_desc(**bad)) == code
    assert _attend(desc=_desc(**bad)) == code
    assert _assemble(desc=_desc(**bad)) == code
    assert cf.cf_prefill_workspace_bytes_q4(_desc(**bad), 1, 8, 4, 100) == 0


@pytest.mark.parametrize("bad", BAD_STORES)
def test_stores(bad):
    assert _quantize(store=_store(**bad)) == INVALID
    assert _attend(store=_store(**bad)) == INVALID
    assert _assemble(store=_store(**bad)) == INVALID


def test_quantize_arguments():
    for kw in (dict(k=None), dict(v=None), dict(slots=None), dict(k=FAKE + 2), dict(v=FAKE + 8), dict(n_tokens=-1), dict(store=None)):
        assert _quantize(**kw) == INVALID, kw
    cf.cf_quantize_cache(_desc(), None, None, 0, None, None, _store(), stream=0)          # nothing to do


def test_attention_arguments():
    for kw in (dict(q=None), dict(q_off=None), dict(segs=None), dict(n_seg=None), dict(out=None), dict(q_new_start=None), dict(v_self=None),
               dict(out=FAKE + 2), dict(max_tq=0), dict(seg_stride=0), dict(batch=-1), dict(max_kv_tokens=-1),
               dict(score_accum=FAKE, score_stride=0), dict(mass=None, score_accum=FAKE, score_stride=4)):
        assert _attend(**kw) == INVALID, kw
    assert _attend(seg_stride=257) == UNSUPPORTED
    assert _attend(batch=70000) == UNSUPPORTED
    assert _attend(q_stored_start=4096) == RANGE and _attend(q_stored_start=-1) == RANGE
    assert _attend(workspace=None) == WORKSPACE and _attend(workspace=FAKE + 16) == WORKSPACE
    need = cf.cf_prefill_workspace_bytes_q4(_desc(), 1, 8, 4, 100)
    assert need > 0 and need % 256 == 0 and _attend(workspace_bytes=need - 1) == WORKSPACE
    assert cf.cf_prefill_workspace_bytes_q4(_desc(), 1, 8, 257, 100) == 0
    cf.cf_prefill_attention_q4(_desc(), None, None, 0, None, None, None, None, None, None, 4, 0, 8, 0, None, None, None, 0, None, 0, stream=0)


def test_assemble_arguments():
    for kw in (dict(store=None), dict(q_off=None), dict(segs=None), dict(final_off=None), dict(k_final=None), dict(final_len=None),
               dict(k_self=None), dict(k_final=FAKE), dict(v_final=2 * FAKE), dict(final_token_stride=64), dict(final_head_stride=132),
               dict(max_seg_len=0), dict(seg_stride=0), dict(max_tq=0), dict(final_capacity=-1)):
        assert _assemble(**kw) == INVALID, kw


def test_block_table_arguments():
    for kw in (dict(cached=None), dict(fresh=None), dict(table=None), dict(free_blocks=None), dict(n_free=None), dict(next_len=None),
               dict(next_n_free=None), dict(q_off=None), dict(q_new_start=None), dict(slots=None), dict(shift=None), dict(segs=None),
               dict(n_seg=None), dict(block_tokens=0), dict(n_blocks=-1), dict(first_token=-1), dict(table_stride=0), dict(seg_stride=0),
               dict(max_new_tokens=-1), dict(base_segs=FAKE), dict(n_base=FAKE), dict(base_segs=2 * FAKE, n_base=FAKE, base_stride=0),
               dict(next_len=FAKE), dict(next_n_free=FAKE), dict(segs=2 * FAKE, base_segs=2 * FAKE, n_base=FAKE, base_stride=1), dict(batch=-1)):
        assert _tables(**kw) == INVALID, kw
    assert _tables(batch=8193) == UNSUPPORTED and _tables(table_stride=4096) == UNSUPPORTED
    assert _tables(q_stored_start=-1) == RANGE


def test_a_workspace_serves_shorter_lists():
    """For every batch and row count the bytes grow with both of what they may be shorter in."""
    for hq, hkv in ((32, 32), (28, 4), (12, 2), (4, 4)):
        d = _desc(n_q_heads=hq, n_kv_heads=hkv)
        for batch in (1, 2, 7, 33, 64):
            for tq in (1, 5, 48, 200):
                last = 0
                for kv in (0, 1, 31, 100, 500, 900, 2000, 5000, 9000, 33000, 100000):
                    n = cf.cf_prefill_workspace_bytes_q4(d, batch, tq, 8, kv)
                    assert n >= last
                    last = n
                last = 0
                for stride in (1, 2, 9, 64, 65, 256):
                    n = cf.cf_prefill_workspace_bytes_q4(d, batch, tq, stride, 3000)
                    assert n >= last
                    last = n


def test_structure_matches_the_header():
    assert C.sizeof(cf.cf_q4_store) == 40


# ------------------------------------------------------------------------------------------------ the plain definitions
def test_the_format_by_hand():
    codes = np.zeros((1, 64), dtype=np.uint8)
    codes[0, :8] = [0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE]
    scales = np.array([[128, 127, 126, 255]], dtype=np.uint8)
    v = R.decode(codes, scales)[0]
    assert v[:16].tolist() == [0, 1, 2, 3, 4, 6, 8, 12, 0, -1, -2, -3, -4, -6, -8, -12]
    assert (v[16:96] == 0).all() and np.isnan(v[96:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rounding_to_the_format(dtype):
    # magnitudes and ties with the scale 1: 6.9 keeps it at 1
    x = np.zeros((1, 128))
    x[0, :14] = [6.9, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.2500001, 5.0000001, -5.0, 7.0, 0.2, -0.0]
    codes, scales, _ = R.encode(x, dtype)
    assert R.decode(codes, scales)[0, :14].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, -0.5, 6, -4, 6, 0, 0]
    assert scales[0].tolist() == [127] + [R.E_RANGE[dtype][0] + 127] * 3
    # the scale: the least power of two with top <= 7 * scale, within the range
    for top, e in ((7.0, 0), (7.0000001, 1), (3.5, -1), (3.5000001, 0), (1.0, -2), (1e-30, max(-102, R.E_RANGE[dtype][0])),
                   (3.0e38, min(R.E_RANGE[dtype][1], 126))):
        x[0, 0], x[0, 1:] = top, 0
        assert R.encode(x, dtype)[1][0, 0] == 127 + e, top
    for v in (np.inf, np.nan):
        x[0, 40] = v
        codes, scales, _ = R.encode(x, dtype)
        assert scales[0, 1] == 255 and np.isnan(R.decode(codes, scales)[0, 32:64]).all() and np.isfinite(R.decode(codes, scales)[0, :32]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_what_is_written_is_a_number_of_the_type_and_rounds_to_itself(dtype):
    import torch
    t = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    rng = np.random.default_rng(5)
    hi = 1.0e4 if dtype == "f16" else 1.0e30
    x = rng.standard_normal((64, 128)) * np.exp(rng.uniform(np.log(1e-8), np.log(hi), size=(64, 1)))
    x = torch.from_numpy(x).to(t).double().numpy()
    codes, scales, _ = R.encode(x, dtype)
    v = R.decode(codes, scales)
    assert np.array_equal(torch.from_numpy(v).to(t).double().numpy(), v)
    again = R.decode(*R.encode(v, dtype)[:2])
    assert np.array_equal(again, v)
    # off by at most half a step: half the group's scale per unit at the top, i.e. the scale itself, and never more than top / 3.5
    top = np.abs(x.reshape(64, 4, 32)).max(-1)
    inside = (scales > R.E_RANGE[dtype][0] + 127) & (scales < R.E_RANGE[dtype][1] + 127)
    off = np.abs(v - x).reshape(64, 4, 32).max(-1)
    assert (off <= top / 3.5)[inside].all()


def test_a_step_of_blocks_by_hand():
    b = R.Blocks(table_stride=4, block=4, n_blocks=10, first_token=100, seg_stride=4)
    # request 0 adds one token to 4 (a new block), 1 leaves with two blocks, 2 starts with 5 tokens
    table = np.array([[7, 0, 0, 0], [2, 3, 0, 0], [0, 0, 0, 0]])
    free = np.array([9, 8, 6, 0, 0, 0, 0, 0, 0, 0])
    s = b.step([4, 6, 0], [1, -1, 5], table, free, 3, [10, 0, 0])
    assert s["table"][:, :2].tolist() == [[7, 3], [2, 3], [2, 6]] and s["next_n_free"] == 2 and s["free"][:3].tolist() == [9, 8, 6]
    assert s["slots"] == [112, 108, 109, 110, 111, 124] and s["q_off"] == [0, 1, 1, 6] and s["next_len"] == [5, 0, 5]
    assert s["segs"][0] == [(128, 4, 10, 10, 0, -1), (0, 1, 0, 14, 2, -1)] and s["segs"][2] == [(1, 5, 0, 0, 2, -1)]
    assert s["flags"] == 0
    # a pool that runs short: the third request is not served, one that needs nothing is
    s = b.step([4, 0, 0, 6], [1, 4, 1, 1], np.zeros((4, 4), dtype=int) + 1, free, 2, [0] * 4)
    assert s["next_len"] == [5, 4, 0, 7] and s["flags"] == cf.CF_FLAG_NO_BLOCKS and s["slots"][5] == -1 and s["next_n_free"] == 0


def test_block_cache_refuses_tables_that_the_attention_does_not_take():
    s = pl.Q4Store(4, 2, "bf16", 1.0e4, 4096, 8, device="cpu")
    with pytest.raises(ValueError, match="entries"):
        pl.BlockCache(s.desc, 2, 16, 8, max_len=16 * 256, max_new=4, device="cpu")
    assert pl.BlockCache(s.desc, 2, 16, 8, max_len=16 * 255, max_new=4, device="cpu").ws_bytes > 0


def test_sizes_past_the_launch_are_no_small_workspace():
    s = pl.Q4Store(64, 64, "bf16", 1.0e4, 4096, 8, device="cpu")
    small = cf.cf_prefill_workspace_bytes_q4(s.desc, 1, 1 << 20, 4, 4096)
    assert cf.cf_prefill_workspace_bytes_q4(s.desc, 1, (1 << 31) - 1, 4, 4096) > small
    assert cf.cf_prefill_workspace_bytes_q4(s.desc, 65535, (1 << 24), 4, 4096) > small
