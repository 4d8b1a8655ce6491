"""Attention behind shared prefixes to the bits that vtoken_attention gives the same rows: the weights enter the product over V as sums
of two 16-bit numbers (over 4-bit rows with bf16 queries: as one in half precision), for the prefix and for own tokens alike.  Requests
of many query rows are the prompt kernel's, in both calls.

The bound is one of sums: |out - exact| <= rounding of the output + (weights' own error) * sum of w |v|, so an output near zero shows
what larger ones hide.  Queries are small, which makes the error of the scores small next to that of a weight."""
import numpy as np
import pytest

from attention_sim import unit
from paper_2608_13263_b200 import binding as vt
from test_gpu_shared import Groups

pytestmark = pytest.mark.gpu

GEOMETRIES = [("bf16", "bf16", 8, 2, 128), ("fp16", "fp16", 7, 1, 128), ("bf16", "bf16", 4, 4, 64), ("fp16", "fp16", 16, 1, 64),
              ("fp16", "fp4", 14, 2, 64), ("fp16", "fp4", 3, 3, 128), ("bf16", "fp4", 8, 2, 128)]
IDS = ["-".join(map(str, g)) for g in GEOMETRIES]


def reference(st):
    """(out, bound), float64."""
    c = st.c
    q = st.q_all.double().cpu().numpy()[:st.n, :c.hq * c.d].reshape(st.n, c.hq, c.d)
    out, tol = (np.zeros((st.n, c.hq, c.d)) for _ in range(2))
    u = unit(c.act)
    # what is left of a weight that is held as two numbers of the type is half a step of the second: u^2 of it; in half precision as one 2^-11
    few = 2.0 ** -11 if c.kv == "fp4" and c.act == "bf16" else u * u
    # requests of more than 32 query rows are the prompt kernel's when the hint tells of such: one number of the product's type, half a step
    # of it at most, u (over 4-bit rows half precision's, 2^-11)
    group = c.hq // c.hkv
    many = 2.0 ** -11 if c.kv == "fp4" else u
    for r in range(len(st.ids)):
        held = many if st.max_query_len * group > 32 and len(st.positions[r]) * group > 32 else few
        for j, p in enumerate(st.positions[r]):
            row = int(st.q_off[r]) + j
            seen = [s for i, s in zip(st.ids[r], st.slots[r]) if i <= p and (not st.window or i > p - st.window or i < st.sinks)]
            if not seen:
                continue
            k, v = (np.repeat(np.stack([x[s] for s in seen]), c.hq // c.hkv, 1) for x in (c.k64, c.v64))
            s = np.einsum("hd,lhd->hl", q[row], k) * st.sm_scale
            w = np.exp(s - s.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            out[row] = np.einsum("hl,lhd->hd", w, v)
            # a score: D exact products summed in 32 bits by accumulators that cut, D 2^-23 of their absolute values; differences and
            # exponents 2^-21; both for the weight and for the sum under the quotient
            ds = (c.d * 2.0 ** -23 * np.einsum("hd,lhd->hl", np.abs(q[row]), np.abs(k)) * abs(st.sm_scale)).max(-1)
            ds = ds + 2.0 ** -21 * (1 + np.abs(s).max(-1))
            # the products over V: 16 tokens an addition, twice, 2^-23 of the sum each; and up to 32 joins of parts
            sums = (len(seen) / 8 + 32) * 2.0 ** -23
            tol[row] = 1.01 * u * np.abs(out[row]) + (held + 2 * ds[:, None] + sums) * np.einsum("hl,lhd->hd", w, np.abs(v)) + 2.0 ** -25
    return out, tol


def run_and_check(g):
    g.call()
    out, _ = g.st.outputs()
    ref, tol = reference(g.st)
    off = np.abs(out - ref)
    assert (off <= tol).all(), f"{(off > tol).mean()} of the values, {(off / tol).max()} of the bound"
    assert g.c.flags() == 0
    g.close()


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
@pytest.mark.parametrize("prefix", [40, 300])
def test_single_tokens(geometry, prefix):
    run_and_check(Groups(np.random.default_rng(prefix), geometry, [(prefix, [1, 2, 17, 3, 40])], q_scale=0.1))


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
def test_drafts_behind_windowed_prefixes(geometry):
    def queries(lens):
        return [list(range(n - min(m, n), n)) for n, m in zip(lens, [1, 4, 0, 3, 2, 1, 2])]
    run_and_check(Groups(np.random.default_rng(2), geometry, [(200, [5, 30, 9, 4]), (70, [9, 12, 3])], queries, keep=0.8, window=150, sinks=5,
                         q_scale=0.1))


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
def test_several_row_tiles_and_parts(geometry):
    act, kv, hq, hkv, d = geometry
    members = 300 // (hq // hkv) + 2
    run_and_check(Groups(np.random.default_rng(3), geometry, [(500, [1 + i % 5 for i in range(members)])], keep=0.9, q_scale=0.1))


@pytest.mark.parametrize("geometry", GEOMETRIES[:2], ids=IDS[:2])
@pytest.mark.parametrize("hint", [1, 1000])
def test_requests_of_many_rows_by_either_hint(geometry, hint):
    """With a hint of few query tokens requests of many rows are behind the prefix too, otherwise they are the prompt kernel's (whose
    weights are one number, as in vtoken_attention): what is checked here are the short ones among them."""
    rng = np.random.default_rng(4)
    g = Groups(rng, geometry, [(200, [11, 9, 60])], lambda lens: [[210], list(range(205, 209)), list(range(100, 260))], max_query_len=hint, q_scale=0.1)
    g.call()
    out, _ = g.st.outputs()
    ref, tol = reference(g.st)
    rows = slice(0, None if hint == 1 else int(g.st.q_off[2]))
    assert (np.abs(out - ref)[rows] <= tol[rows]).all()
    g.close()
