"""Token writes and reads at the edges: values that leave 32 bits on the way into 4-bit rows, values that are not finite, calls
without tokens."""
import numpy as np
import pytest

from attention_sim import to64
from paper_2608_13263_b200 import binding as vt
from test_gpu_tokens import GEOMETRIES, Writer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exponents", [(-30, -30), (-60, -45), (-28, 0)])
@pytest.mark.parametrize("geometry", [GEOMETRIES[3], GEOMETRIES[6]], ids=["128", "64"])
def test_4_bit_rows_saturate_beyond_32_bits(geometry, exponents):
    """Finite values whose multiple by 2^-exponent is not a 32-bit number are held as the largest, not as NaN."""
    w = Writer(np.random.default_rng(50), geometry, 40, exponents=exponents, scale=3e29, weights=False)
    w.write()
    w.check()
    w.close()


@pytest.mark.parametrize("rot,interleaved", [(0, False), (16, False), (16, True), (48, False), (48, True)])
@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[1], GEOMETRIES[2]], ids=["bf16", "fp16", "64"])
def test_values_that_are_not_finite_stay_where_they_are(geometry, rot, interleaved):
    """NaN, infinities and negative zeros outside the rotated dimensions touch no other value of the head."""
    import torch
    w = Writer(np.random.default_rng(51), geometry, 30, rot=rot, interleaved=interleaved, weights=False, packed=False)
    d = w.d
    for heads, x in ((w.hq, w.q), (w.hkv, w.k)):
        y = x.view(-1, heads, d)
        for i in range(30):
            y[i, i % heads, rot + i % (d - rot)] = (float("nan"), float("inf"), -float("inf"), -0.0)[i % 4]
    q, k = (x.clone().view(30, -1, d)[..., rot:].contiguous().view(torch.int16) for x in (w.q, w.k))
    w.q64, w.k64 = to64(w.q), to64(w.k)
    w.write()
    rows = w.pools[0][w.layer][torch.from_numpy(w.slots).to(w.dev).long()]
    got_q, got_k = (x.view(30, -1, d) for x in (w.q_out, rows))
    for got, ref in ((got_q, q), (got_k, k)):
        g = got[..., rot:].contiguous()
        nan = torch.isnan(ref.view(g.dtype))
        assert torch.equal(torch.isnan(g), nan)
        assert torch.equal(g.view(torch.int16)[~nan], ref[~nan])
    with np.errstate(all="ignore"):
        want_q, want_k, _ = w.expected()
    if rot:
        w.near(to64(got_q)[..., :rot], want_q[..., :rot])
        w.near(to64(got_k)[..., :rot], want_k[..., :rot])
    w.close()


@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[3]], ids=["16", "4"])
def test_normalised_rows_with_an_infinity(geometry):
    """The definition: a row with an infinity has an infinite mean square, so its finite values become zero and the infinity NaN;
    a rotation then takes the NaN to its partner alone."""
    w = Writer(np.random.default_rng(52), geometry, 12, rot=32)
    for i in range(12):
        w.q.view(12, -1)[i, 5 + 128 * (i % w.hq) + 8 * i] = float("inf")
    w.q64 = to64(w.q)
    w.write()
    with np.errstate(all="ignore"):
        want, _, _ = w.expected()
    got = to64(w.q_out).reshape(12, w.hq, w.d)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want).any()
    ok = np.isfinite(want)
    assert (np.abs(got - want)[ok] <= 2.0 ** -8 * np.abs(want)[ok] + 2.0 ** -15).all()
    w.close()


def test_calls_without_tokens_need_no_tensors():
    """A tensor without elements has no address."""
    import torch
    for g in (GEOMETRIES[0], GEOMETRIES[3]):
        w = Writer(np.random.default_rng(53), g, 4)
        empty = torch.empty(0, device=w.dev, dtype=w.q.dtype)
        none = torch.empty(0, device=w.dev, dtype=torch.int32)
        assert empty.data_ptr() == 0 and none.data_ptr() == 0
        w.write(max_tokens=0, q=empty, k=empty, v=empty, q_out=empty, slots=none, positions=none)
        vt.vtoken_read_tokens(w.ctx, heads=w.heads, layer=0, max_tokens=0, slots=none, out_k=empty, out_v=empty)
        assert w.flags() == 0
        with pytest.raises(vt.VtokenError):                   # what is not about the tokens is still checked
            w.write(max_tokens=0, layer=7)
        with pytest.raises(vt.VtokenError):
            w.write(max_tokens=0, rot_dim=8)
        w.close()
