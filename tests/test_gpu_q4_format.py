"""Scale bytes over the format's whole range in a 4-bit store that another program filled: gathered, and attended to."""

import numpy as np
import pytest
import torch

from paper_2502_11101_amd import binding as cf
from paper_2502_11101_amd import pipeline as pl
from paper_2502_11101_amd import workloads as wl
from tests import q4_bounds as Q
from tests import q4_reference as R
from tests.test_gpu_q4_attention import BASE, PAIRING, i32, upload
from tests.test_gpu_q4_precision import call, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("pairing", ["half", "interleaved"])
def test_gather_of_every_scale_and_code(dtype, pairing):
    """Every value that is a number of the 16-bit type is gathered as it is, keys and values, one past the type's largest as an infinity;
    scale 255 reads as NaN."""
    n = 256
    rng = np.random.default_rng(1)
    codes = rng.permuted(np.tile(np.arange(256, dtype=np.uint8), (n, 1, 1)), axis=-1)[..., :64]
    codes[:, 0, :8] = [0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE]                     # every code in the first group
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None, None], 4, axis=-1)
    host = dict(k_codes=codes, k_scales=scales, v_codes=codes[::-1].copy(), v_scales=scales[::-1].copy())
    s = upload(host, 1, dtype, "token", pairing)
    kf, vf = (torch.zeros((n, 1, 128), dtype=pl.TORCH_DTYPE[dtype], device="cuda") for _ in range(2))
    flag, length = i32([0]), i32([0])
    cf.cf_assemble_cache_q4(s.desc, s.store, None, None, i32([0, 0]), cf.segments_to_device(cf.segments_array([(0, n, 7, 7, cf.CF_SEG_DOC, 0)])),
                            i32([1]), 1, 1, 1, n, torch.zeros(1, dtype=torch.int64, device="cuda"), n, 128, 128, kf, vf, length, None, flag)
    torch.cuda.synchronize()
    assert int(flag.item()) == 0
    for got, c, x in ((kf, "k_codes", "k_scales"), (vf, "v_codes", "v_scales")):
        want = R.decode(host[c], host[x])
        with np.errstate(over="ignore"):
            of_type = torch.from_numpy(want).to(pl.TORCH_DTYPE[dtype]).double().numpy() == want
        got = got.double().cpu().numpy()
        bad = of_type & (got != want)
        assert not bad.any(), sorted({int(b) for b in np.broadcast_to(host[x].repeat(32, -1), want.shape)[bad]})
        assert np.isnan(got[np.isnan(want)]).all()
        past = np.abs(want) >= 2.0 ** (128 if dtype == "bf16" else 16)                   # (NaN: not so)
        assert past.any() and np.array_equal(got[past], np.sign(want[past]) * np.inf)


@pytest.mark.parametrize("tq", [1, 20, 70])
# (252 is the largest byte whose every code is a number of bf16: 6 * 2^125 = 1.5 * 2^127, while 4 * 2^126 = 2^128 is past its largest, 2^128 - 2^120)
@pytest.mark.parametrize("byte", [0, 1, 2, 3, 250, 252])
def test_keys_of_every_scale(byte, tq):
    """Keys at both ends of the scales' range, and queries that bring the scores back to ordinary sizes."""
    rng = np.random.default_rng(byte + tq)
    heads, n = 2, 70
    host = R.random_store(rng, n, heads, "bf16")
    shift = byte - 127
    host["k_scales"][:] = byte
    s = upload(host, heads, "bf16", "head", "half")
    ks, vs = R.decode(host["k_codes"], host["k_scales"]), R.decode(host["v_codes"], host["v_scales"])
    q = wl.round_to_dtype((rng.standard_normal((tq, heads, 128)) * 2.0 ** np.clip(-shift, -125, 124)).astype(np.float32), "bf16")
    got, mass, segs = call(s, "bf16", q, 0, None, [(0, n, 3, 3)], heads)
    want, want_mass, off, mass_off = Q.attention(q, 0, ks, vs, None, None, segs, heads, BASE)
    assert np.isfinite(got).all() and within(got, want, off, "bf16") <= 1
    assert (np.abs(mass - want_mass) <= mass_off).all()
