"""The bounds that attention over a 4-bit store is held to (q4_bounds): their values are the oracle's, and they tell the documented arithmetic from
one with fewer bits.  Runs without a GPU."""

import numpy as np
import pytest

from oracle import cachefocus_oracle as orc
from paper_2502_11101_amd import workloads as wl
from tests import q4_bounds as Q
from tests import q4_reference as R

BASE = 1.0e4


def _inputs(make, dtype, pairing, own_block, rows=1, heads=6, n=60):
    rng = np.random.default_rng(11)
    host, q = make(rng, heads, n, dtype, rows)
    q = wl.round_to_dtype(q.astype(np.float32), dtype)
    own = [wl.round_to_dtype(rng.standard_normal((rows, heads, 128), dtype=np.float32), dtype) for _ in range(2)]
    segs = [orc.Segment(i, 1, 40, 40 + 7 * i, orc.KIND_DOC, i) for i in range(n)]
    if own_block:
        segs.append(orc.Segment(0, rows, 0, 900, orc.KIND_SELF, -1))
    return q, 900, R.decode(host["k_codes"], host["k_scales"]), R.decode(host["v_codes"], host["v_scales"]), *own, segs, heads, BASE, pairing


@pytest.mark.parametrize("pairing", ["half", "interleaved"])
def test_values_are_the_oracles(pairing):
    a = _inputs(Q.single_tokens, "bf16", pairing, True, rows=5)
    out, mass, off, mass_off = Q.attention(*a)
    q, pos, *rest = a
    ref, ref_mass = orc.prefill_attention(q.astype(np.float64), 0, pos, *rest)
    assert np.abs(out - ref).max() < 1e-11 and np.abs(mass - np.asarray(ref_mass)).max() < 1e-11
    assert (off > 0).all() and (mass_off[mass > 0] > 0).all()


@pytest.mark.parametrize("pairing", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("terms,bits,own_block,passes", [
    (2, 11, False, True), (1, 11, False, False), (1, 8, False, False),                   # one term of either type: more than the bound
    # with own tokens among them, whose bound is wider where they are bf16
    (2, 11, True, True), (1, 11, True, False)])
def test_fewer_bits_are_told_apart(terms, bits, own_block, passes, dtype, pairing):
    a = _inputs(Q.single_tokens, dtype, pairing, own_block)
    out, mass, off, mass_off = Q.attention(*a, dtype=dtype)
    got, got_mass, _, _ = Q.attention(*a, dtype=dtype, query=Q.rounded_query(terms, bits))
    worst = (np.abs(got_mass - mass) / mass_off).max()
    assert worst <= 0.25 and (np.abs(got - out) / off).max() <= 0.25 if passes else worst > 2


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_fifteen_bits_are_told_from_twenty_two(dtype):
    rng = np.random.default_rng(1)
    host, q = Q.one_channel(rng, 60, dtype)
    segs = [orc.Segment(i, 1, 40, 40, orc.KIND_DOC, i) for i in range(60)]
    a = (q, 0, R.decode(host["k_codes"], host["k_scales"]), R.decode(host["v_codes"], host["v_scales"]), None, None, segs, 1, BASE, "half", 0.05)
    _, mass, _, mass_off = Q.attention(*a, dtype=dtype)
    worst = [(np.abs(Q.attention(*a, dtype=dtype, query=Q.rounded_query(t, b, Q.factor(0.05)))[1] - mass) / mass_off).max() for t, b in ((2, 11), (2, 8))]
    assert worst[0] < 0.25 and worst[1] > 2


def test_own_keys_of_bf16_calls_meet_16_bits():
    a = _inputs(Q.single_tokens, "bf16", "half", True, rows=3)
    segs = [orc.Segment(0, 3, 0, 890, orc.KIND_SELF, -1)]
    a = (*a[:6], segs, *a[7:])
    out, mass, off, _ = Q.attention(*a)
    for terms, passes in ((2, True), (1, False)):
        got = Q.attention(*a, query=Q.rounded_query(terms, 8))[0]
        assert ((np.abs(got - out) / off).max() <= 1) == passes
