"""Limits that the calls on a 4-bit cache store keep to, checked on the host: runs without a GPU."""

import numpy as np
import pytest
import torch

from paper_2502_11101_amd import binding as cf
from paper_2502_11101_amd import pipeline as pl
from tests.test_q4_host import INVALID, _tables


@pytest.mark.parametrize("limit", [-1, -(1 << 31)])
def test_rows_per_request_are_not_negative(limit):
    assert _tables(max_fresh=limit) == INVALID


@pytest.fixture
def written(monkeypatch):
    """The sizes that cf_quantize_cache is called with, which is not called."""
    calls = []

    def record(desc, k, v, n_tokens, slots, shift, store, dev_flag=None, stream=None, n_live=None):
        calls.append((n_tokens, k.shape[0], v.shape[0], slots.shape[0], None if shift is None else shift.shape[0]))
    monkeypatch.setattr(cf, "cf_quantize_cache", record)
    return calls


def _rows(n):
    return torch.zeros((n, 2, 128), dtype=torch.bfloat16)


@pytest.mark.parametrize("rows", [0, 1, 7, 8, 9, 1000])
def test_padding_behind_a_step_names_no_slots_that_are_not_there(written, rows):
    s = pl.Q4Store(4, 2, "bf16", 1.0e4, 4096, 64, device="cpu")
    cache = pl.BlockCache(s.desc, 2, 16, 4, max_len=64, max_new=4, device="cpu")
    cache.append(s, _rows(rows), _rows(rows))
    (n, n_k, n_v, n_slots, n_shift), = written
    assert n == min(rows, cache.max_rows) and min(n_k, n_v, n_slots, n_shift) >= n


def test_writes_with_fewer_slots_than_rows_are_refused(written):
    s = pl.Q4Store(4, 2, "bf16", 1.0e4, 4096, 64, device="cpu")
    slots, shift = torch.zeros(5, dtype=torch.int64), torch.zeros(5, dtype=torch.int32)
    for k, v, at, by in ((6, 6, slots, None), (6, 6, slots, shift), (4, 3, slots, shift), (5, 5, slots, shift[:4])):
        with pytest.raises(ValueError, match="fewer"):
            s.write(_rows(k), _rows(v), at, by)
    assert written == []
    s.write(_rows(4), _rows(5), slots, shift)            # more of them than rows: the rest is not used
    assert written == [(4, 4, 5, 5, 5)]


@pytest.fixture
def attended(monkeypatch):
    """The arguments that cf_prefill_attention_q4 is called with, which is not called."""
    calls = []
    monkeypatch.setattr(cf, "cf_prefill_attention_q4", lambda *a, **k: calls.append(a))
    return calls


def test_a_batch_has_workspace_for_every_layer_it_is_given(attended):
    layers = [pl.Q4Store(hq, hkv, "bf16", 1.0e4, 4096, 700, device="cpu") for hq, hkv in ((4, 4), (32, 32), (28, 4), (4, 4))]
    lens = np.full((2, 5), 100)
    pb = pl.PrefillBatch(layers[0].desc, np.arange(10).reshape(2, 5) * 100, lens, 48, 4, 4, 700, device="cpu")
    for s in layers:
        pb.attention_q4(None, None, None, s, None)
        desc, seg_stride, batch, tq, kv, nbytes = (attended[-1][i] for i in (0, 10, 11, 12, 13, -2))
        assert nbytes >= cf.cf_prefill_workspace_bytes_q4(desc, batch, tq, seg_stride, kv) > 0
        assert attended[-1][-3].numel() >= nbytes
