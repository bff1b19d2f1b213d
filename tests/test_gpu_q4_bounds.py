"""Outputs and masses of attention over a 4-bit store within bounds that follow from the kernels' arithmetic, row by row and head by head
(q4_bounds), which fewer bits of the query would break."""

import numpy as np
import pytest

from paper_2502_11101_amd import workloads as wl
from tests import q4_bounds as Q
from tests import q4_reference as R
from tests.test_gpu_q4_attention import BASE, CASES, upload
from tests.test_gpu_q4_precision import call, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", list(CASES))
def test_every_case_within_its_bound(name):
    """The cases of the comparison with the oracle, query by query, against bounds of every row and head."""
    c = dict(CASES[name])
    dtype, pairing, layout = c.get("dtype", "bf16"), c.get("pairing", "half"), c.get("layout", "head")
    rng = np.random.default_rng(len(name))
    hq, hkv = c["hq"], c["hkv"]
    host = R.random_store(rng, c.get("n_store", 600), hkv, dtype)
    s = upload(host, hkv, dtype, layout, pairing, group=hq // hkv)
    ks, vs = R.decode(host["k_codes"], host["k_scales"]), R.decode(host["v_codes"], host["v_scales"])
    normal = lambda n, h: wl.round_to_dtype(rng.standard_normal((n, h, 128), dtype=np.float32), dtype)     # noqa: E731
    for b, (entries, tq) in enumerate(zip(c["tables"], c["lengths"])):
        own = None if b in c.get("no_own", ()) else (normal(max(tq, 1), hkv), normal(max(tq, 1), hkv))
        if tq == 0 or (own is None and not sum(e[1] for e in entries)):
            continue
        q = normal(tq, hq)
        pos = c.get("q_pos", [5000 + 7 * b] * (b + 1))[b]
        got, mass, segs = call(s, dtype, q, pos, own, entries, hkv)
        want, want_mass, off, mass_off = Q.attention(q, pos, ks, vs, *(own or (None, None)), segs, hkv, BASE, pairing, dtype=dtype)
        assert within(got, want, off, dtype) <= 1, b
        assert (np.abs(mass - want_mass) <= mass_off).all(), (b, (np.abs(mass - want_mass) / np.maximum(mass_off, 1e-300)).max())


@pytest.mark.parametrize("tq,heads", [(1, 8), (20, 4), (70, 2), (140, 2)])
@pytest.mark.parametrize("dtype,pairing", [("bf16", "half"), ("f16", "interleaved")])
def test_masses_of_single_tokens(tq, heads, dtype, pairing):
    """Entries of one token each and loud queries: a mass is as good as the score that it is made of, of store and own tokens."""
    rng = np.random.default_rng(tq + heads)
    n = 60
    host, q = Q.single_tokens(rng, heads, n, dtype, tq)
    q = wl.round_to_dtype(q.astype(np.float32), dtype)
    s = upload(host, heads, dtype, "head", pairing)
    ks, vs = R.decode(host["k_codes"], host["k_scales"]), R.decode(host["v_codes"], host["v_scales"])
    own = tuple(wl.round_to_dtype(rng.standard_normal((tq, heads, 128), dtype=np.float32), dtype) for _ in range(2))
    for moved in (False, True):
        entries = [(int(t), 1, 40, 40 + (7 * i if moved else 0)) for i, t in enumerate(rng.permutation(n))]
        pos = 900 if moved else 0
        got, mass, segs = call(s, dtype, q, pos, own, entries, heads)
        want, want_mass, off, mass_off = Q.attention(q, pos, ks, vs, *own, segs, heads, BASE, pairing, dtype=dtype)
        assert within(got, want, off, dtype) <= 1
        assert (np.abs(mass - want_mass) <= mass_off).all(), (np.abs(mass - want_mass) / mass_off).max()


@pytest.mark.parametrize("tq", [1, 20, 70, 140])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_masses_with_queries_of_one_channel(tq, dtype):
    """Nothing averages out of a score: two terms of eight bits in place of the documented ones would be twice the bound off."""
    rng = np.random.default_rng(1)
    n = 60
    host, q = Q.one_channel(rng, n, dtype, tq)
    s = upload(host, 1, dtype, "head", "half", 0.05)
    ks, vs = R.decode(host["k_codes"], host["k_scales"]), R.decode(host["v_codes"], host["v_scales"])
    got, mass, segs = call(s, dtype, q, 0, None, [(i, 1, 40, 40) for i in range(n)], 1)
    want, want_mass, off, mass_off = Q.attention(q, 0, ks, vs, None, None, segs, 1, BASE, scale=0.05, dtype=dtype)
    assert within(got, want, off, dtype) <= 1
    assert (np.abs(mass - want_mass) <= mass_off).all(), (np.abs(mass - want_mass) / mass_off).max()
