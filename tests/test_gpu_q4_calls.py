"""Calls on a 4-bit store that the documentation allows beside the ordinary ones: stores with room between their rows, queries that carry other
positions than local ones, several own blocks in a table."""

import numpy as np
import pytest
import torch

from oracle import cachefocus_oracle as orc
from paper_2502_11101_amd import binding as cf
from paper_2502_11101_amd import pipeline as pl
from paper_2502_11101_amd import workloads as wl
from tests import q4_bounds as Q
from tests import q4_reference as R
from tests.test_gpu_q4_attention import BASE, POSITIONS, i32
from tests.test_gpu_q4_precision import within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("token_stride,head_stride", [(3 * 384, 384), (128, 100 * 128), (640, 128 * 700), (5 * 128, 128)])
@pytest.mark.parametrize("tq", [1, 30])
def test_stores_with_room_between_their_rows(token_stride, head_stride, tq):
    """Written, attended and gathered with strides wider than the rows need; what lies between them stays as it was."""
    rng = np.random.default_rng(tq)
    heads, n = 3, 61
    desc = cf.make_desc(heads, heads, 128, "bf16", BASE, POSITIONS, store_token_stride=token_stride, store_head_stride=head_stride)
    size = (n - 1) * token_stride + (heads - 1) * head_stride + 128
    codes = [torch.full((size // 2,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((size // 32,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(2)]
    store = cf.make_q4_store(codes[0], scales[0], codes[1], scales[1], n)
    normal = lambda m: wl.round_to_dtype(rng.standard_normal((m, heads, 128), dtype=np.float32), "bf16")     # noqa: E731
    k, v, q, own = normal(n), normal(n), normal(tq), (normal(tq), normal(tq))
    flag = i32([0])
    cf.cf_quantize_cache(desc, pl.to_device(k, "bf16"), pl.to_device(v, "bf16"), n, torch.arange(n, device="cuda"), None, store, flag)
    torch.cuda.synchronize()
    at = (np.arange(n)[:, None] * token_stride + np.arange(heads) * head_stride)
    values = []
    for x, c, s in zip((k, v), codes, scales):
        c, s = c.cpu().numpy(), s.cpu().numpy()
        ci, si = at[..., None] // 2 + np.arange(64), at[..., None] // 32 + np.arange(4)
        want = R.encode(x, "bf16")
        assert np.array_equal(c[ci], want[0]) and np.array_equal(s[si], want[1])
        for a, i in ((c, ci), (s, si)):
            rest = np.ones(len(a), dtype=bool)
            rest[i] = False
            assert (a[rest] == 0x5A).all()
        values.append(R.decode(c[ci], s[si]))
    rows = [(2, 50, 0, 30, cf.CF_SEG_DOC, 0), (0, 61, 5, 90, cf.CF_SEG_DOC, 1), (0, tq, 0, 200, cf.CF_SEG_SELF, -1)]
    need = cf.cf_prefill_workspace_bytes_q4(desc, 1, tq, 3, 111 + tq)
    ws, out, mass = torch.zeros(need, dtype=torch.uint8, device="cuda"), torch.zeros((tq, heads, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 3), device="cuda")
    dev = [pl.to_device(x, "bf16") for x in (q, *own)]
    table = cf.segments_to_device(cf.segments_array(rows))
    cf.cf_prefill_attention_q4(desc, dev[0], i32([0, tq]), 0, i32([200]), store, dev[1], dev[2], table, i32([3]), 3, 1, tq, 111 + tq, out, mass, None, 1,
                               ws, need, flag)
    kf, vf = (torch.zeros((111 + tq, heads, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    length = i32([0])
    cf.cf_assemble_cache_q4(desc, store, dev[1], dev[2], i32([0, tq]), table, i32([3]), 3, 1, tq, 61, torch.zeros(1, dtype=torch.int64, device="cuda"),
                            111 + tq, heads * 128, 128, kf, vf, length, None, flag)
    torch.cuda.synchronize()
    assert int(flag.item()) == 0 and length.tolist() == [111 + tq]
    segs = [orc.Segment(*r) for r in rows]
    want, want_mass, off, mass_off = Q.attention(q, 200, *values, *own, segs, heads, BASE)
    assert within(out.double().cpu().numpy(), want, off, "bf16") <= 1
    assert (np.abs(mass[0].double().cpu().numpy() - want_mass) <= mass_off).all()
    assert np.array_equal(vf.double().cpu().numpy(), np.concatenate([values[1][2:52], values[1], own[1]]))


@pytest.mark.parametrize("tq", [1, 18, 70, 150])
@pytest.mark.parametrize("dtype,pairing", [("bf16", "half"), ("f16", "interleaved")])
@pytest.mark.parametrize("stored", [0, 300])
def test_several_own_blocks_and_queries_that_carry_positions(tq, dtype, pairing, stored):
    """Two own blocks among the documents (one of another query's rows), and rows whose RoPE starts at `stored`."""
    rng = np.random.default_rng(tq + stored)
    heads, group, n, batch = 2, 2, 90, 2
    host = R.random_store(rng, n, heads, dtype)
    kind = {"half": cf.CF_ROPE_HALF, "interleaved": cf.CF_ROPE_INTERLEAVED}[pairing]
    s = pl.Q4Store(heads * group, heads, dtype, BASE, POSITIONS, n, "token", kind)
    for name, t in (("k_codes", s.k_codes), ("k_scales", s.k_scales), ("v_codes", s.v_codes), ("v_scales", s.v_scales)):
        t.copy_(torch.from_numpy(host[name]))
    ks, vs = R.decode(host["k_codes"], host["k_scales"]), R.decode(host["v_codes"], host["v_scales"])
    normal = lambda m, h: wl.round_to_dtype(rng.standard_normal((m, h, 128), dtype=np.float32), dtype)     # noqa: E731
    q, own = normal(batch * tq, heads * group), (normal(batch * tq, heads), normal(batch * tq, heads))
    q_new = [700, 40]
    tables = [[(3, 40, 0, 30, 1, 0), (tq, tq, stored, 600, 2, 1), (50, 40, 2, 90, 1, 2), (0, tq, stored, 700, 2, -1)],
              [(tq, max(tq - 1, 0), stored, 40, 2, -1), (0, 90, 0, 800, 1, 0), (0, 33, 0, 33, 0, -1), (0, tq, 5, 9, 2, 1)]]
    flag, need = i32([0]), cf.cf_prefill_workspace_bytes_q4(s.desc, batch, tq, 4, 123 + 2 * tq)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    dev = [pl.to_device(x, dtype) for x in (q, *own)]
    out, mass = torch.zeros_like(dev[0]), torch.zeros((batch, 4), device="cuda")
    cf.cf_prefill_attention_q4(s.desc, dev[0], i32([0, tq, 2 * tq]), stored, i32(q_new), s.store, dev[1], dev[2],
                               cf.segments_to_device(cf.segments_array([e for t in tables for e in t])), i32([4, 4]), 4, batch, tq, 123 + 2 * tq, out,
                               mass, None, 1, ws, need, flag)
    torch.cuda.synchronize()
    assert int(flag.item()) == 0
    got, mass = out.double().cpu().numpy(), mass.double().cpu().numpy()
    for b in range(batch):
        part = slice(b * tq, (b + 1) * tq)
        want, want_mass, off, mass_off = Q.attention(q[part], q_new[b] - stored, ks, vs, *own, [orc.Segment(*e) for e in tables[b]], heads, BASE, pairing,
                                                     dtype=dtype)
        assert within(got[part], want, off, dtype) <= 1, b
        assert (np.abs(mass[b] - want_mass) <= mass_off).all(), b
