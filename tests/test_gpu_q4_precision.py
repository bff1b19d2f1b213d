"""Attention over a 4-bit store where its numbers lie far apart: outputs made of small probabilities beside a dominant one, values near the
largest of the type."""

import numpy as np
import pytest
import torch

from oracle import cachefocus_oracle as orc
from paper_2502_11101_amd import binding as cf
from paper_2502_11101_amd import pipeline as pl
from paper_2502_11101_amd import workloads as wl
from tests import q4_bounds as Q
from tests import q4_reference as R
from tests.test_gpu_q4_attention import BASE, i32, upload

pytestmark = pytest.mark.gpu


def call(s, dtype, q, q_pos, own, entries, hkv, max_kv=None):
    """One query's output and masses; entries: (offset, length, stored, new) of the store, ahead of the own block (k, v) if there is one."""
    rows = [(o, n, a, p, cf.CF_SEG_DOC, i) for i, (o, n, a, p) in enumerate(entries)]
    tq = q.shape[0]
    if own is not None:
        rows.append((0, tq, 0, q_pos, cf.CF_SEG_SELF, -1))
    kv = sum(r[1] for r in rows) if max_kv is None else max_kv
    dq = pl.to_device(q, dtype)
    dev = [None, None] if own is None else [pl.to_device(x, dtype) for x in own]
    need = cf.cf_prefill_workspace_bytes_q4(s.desc, 1, tq, len(rows), kv)
    ws, flag = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda"), i32([0])
    out, mass = torch.empty_like(dq), torch.zeros((1, len(rows)), device="cuda")
    cf.cf_prefill_attention_q4(s.desc, dq, i32([0, tq]), 0, i32([q_pos]), s.store, *dev, cf.segments_to_device(cf.segments_array(rows)),
                               i32([len(rows)]), len(rows), 1, tq, kv, out, mass, None, 1, ws, need, flag)
    torch.cuda.synchronize()
    assert int(flag.item()) == 0
    segs = [orc.Segment(*r) for r in rows]
    return out.double().cpu().numpy(), mass[0].double().cpu().numpy(), segs


def within(got, want, off, dtype):
    """|got - want| over what it may be: `off` and the output's own rounding."""
    tiny = 2.0 ** -25 if dtype == "f16" else 2.0 ** -134
    return (np.abs(got - want) / (R.HALF_STEP[dtype] * (np.abs(want) + off) + off + tiny)).max()


# one row; two to four row blocks; a workgroup of 128 rows; of 192 or 256 (more workgroups of 128 than CUs)
SHAPES = [(1, 2, 5000), (20, 2, 5000), (70, 2, 5000), (200, 130, 700)]


@pytest.mark.parametrize("tq,heads,n", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("gap", [8, 14, 16, 17.25, 21, 24])
def test_small_probabilities_beside_a_dominant_token(gap, dtype, tq, heads, n):
    """The first token scores `gap` above all others, which score the same, and has values of zero: the output is what the small ones add up to."""
    rng = np.random.default_rng(tq)
    q = wl.round_to_dtype(rng.standard_normal((1, heads, 128), dtype=np.float32), dtype)
    k, v = np.zeros((n, heads, 128)), 1.0 + rng.random((n, heads, 128))
    # a head's dominant key is its query's signs: their product is the sum of magnitudes, and the queries are scaled to agree in it
    k[0] = np.sign(q[0])
    v[0] = 0
    q = wl.round_to_dtype((q / np.abs(q).sum(-1, keepdims=True) * 128).astype(np.float32), dtype)
    host = {}
    host["k_codes"], host["k_scales"], _ = R.encode(k, dtype)
    host["v_codes"], host["v_scales"], _ = R.encode(v, dtype)
    host["k_scales"][1:] = host["k_scales"][0]           # zeros, with a scale as their neighbours have
    host["v_scales"][0] = 127
    scale = gap / 128.0
    s = upload(host, heads, dtype, "head", "half", scale)
    q = np.repeat(q, tq, axis=0)
    # (one split: the bound on the tokens only sizes the call)
    got, mass, segs = call(s, dtype, q, 0, None, [(0, n, 0, 0)], heads, max_kv=32)
    want, _, off, _ = Q.attention(q[:1], 0, R.decode(host["k_codes"], host["k_scales"]), R.decode(host["v_codes"], host["v_scales"]), None, None, segs,
                                  heads, BASE, scale=scale, dtype=dtype)
    assert within(got, np.repeat(want, tq, axis=0), np.repeat(off, tq, axis=0), dtype) <= 1
    assert mass[0] == pytest.approx(tq * heads, rel=1e-5)


@pytest.mark.parametrize("tq,heads,n", [(1, 2, 300), (20, 2, 300), (70, 2, 300), (200, 130, 40)])
def test_values_near_the_largest_of_the_type(tq, heads, n):
    """bf16 values of 2^125 and more, in the store and in the own block, among ordinary ones: finite outputs, as near as any."""
    rng = np.random.default_rng(tq)
    host = R.random_store(rng, n, heads, "bf16")
    host["v_scales"][n // 2:] = 127 + 122                # 6 * 2^122
    s = upload(host, heads, "bf16", "head", "half")
    ks, vs = R.decode(host["k_codes"], host["k_scales"]), R.decode(host["v_codes"], host["v_scales"])
    normal = lambda m: wl.round_to_dtype(rng.standard_normal((m, heads, 128), dtype=np.float32), "bf16")     # noqa: E731
    k_self, v_self = normal(tq), normal(tq)
    q = normal(tq)
    for own in (None, (k_self, v_self), (k_self, np.where(np.arange(tq)[:, None, None] % 3 == 0, v_self * np.float32(2.0 ** 124), v_self))):
        for entries in ([(0, n, 0, 0)], [(0, n // 3, 0, 0)]):
            got, mass, segs = call(s, "bf16", q, 400, own, entries, heads)
            want, _, off, _ = Q.attention(q, 400, ks, vs, *(own or (None, None)), segs, heads, BASE)
            assert np.isfinite(got).all() and within(got, want, off, "bf16") <= 1


@pytest.mark.parametrize("tq,heads", [(1, 2), (20, 2), (70, 2), (40, 130)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("scale", [1e-18, 1e-25, 1e-38])
def test_softmax_scales_next_to_nothing(scale, dtype, tq, heads):
    """Every token weighs the same, for rows of zeros and of tiny values as well, in tiles that are not full."""
    rng = np.random.default_rng(tq)
    n = 77
    host = R.random_store(rng, n, heads, dtype)
    s = upload(host, heads, dtype, "head", "half", scale)
    ks, vs = R.decode(host["k_codes"], host["k_scales"]), R.decode(host["v_codes"], host["v_scales"])
    normal = lambda m: wl.round_to_dtype(rng.standard_normal((m, heads, 128), dtype=np.float32), dtype)     # noqa: E731
    q, own = normal(tq), (normal(tq), normal(tq))
    q[0, 0] = 0
    q[tq // 2, 1] = wl.round_to_dtype(q[tq // 2, 1] * np.float32(2.0 ** (-90 if dtype == "bf16" else -20)), dtype)
    got, mass, segs = call(s, dtype, q, 400, own, [(0, n, 0, 0)], heads)
    want, want_mass, off, mass_off = Q.attention(q, 400, ks, vs, *own, segs, heads, BASE, scale=scale, dtype=dtype)
    assert within(got, want, off, dtype) <= 1
    assert (np.abs(mass - want_mass) <= mass_off).all()


@pytest.mark.parametrize("tq,heads,n", [(1, 2, 300), (20, 2, 300), (70, 2, 300), (200, 130, 40)])
def test_values_next_to_nothing(tq, heads, n):
    """bf16 values of 2^-112 and less, in the store and in the own block: as near as any, relative to themselves."""
    rng = np.random.default_rng(tq)
    host = R.random_store(rng, n, heads, "bf16")
    host["v_scales"][:] = 127 - 112
    s = upload(host, heads, "bf16", "head", "half")
    ks, vs = R.decode(host["k_codes"], host["k_scales"]), R.decode(host["v_codes"], host["v_scales"])
    normal = lambda m: wl.round_to_dtype(rng.standard_normal((m, heads, 128), dtype=np.float32), "bf16")     # noqa: E731
    k_self, v_self, q = normal(tq), normal(tq) * np.float32(2.0 ** -111), normal(tq)
    for own in (None, (k_self, v_self)):
        got, mass, segs = call(s, "bf16", q, 400, own, [(0, n, 0, 0)], heads)
        want, _, off, _ = Q.attention(q, 400, ks, vs, *(own or (None, None)), segs, heads, BASE)
        assert within(got, want, off, "bf16") <= 1
