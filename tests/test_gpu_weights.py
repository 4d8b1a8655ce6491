"""Attention weights per cached token against the definition in 64 bits: geometries, lengths, windows, masks that leave rows
empty, poisoned keys, strides, decay, streams, graphs, refusals.  The bounds are derived in reference()."""
import numpy as np
import pytest

from attention_sim import Cache, Step, spread, to64
from paper_2608_13263_b200 import binding as vt

pytestmark = pytest.mark.gpu

GEOMETRIES = [("bf16", "bf16", 8, 2, 128), ("fp16", "fp16", 7, 1, 128), ("bf16", "bf16", 4, 4, 64), ("fp16", "fp16", 16, 1, 64),
              ("bf16", "fp4", 8, 2, 128), ("fp16", "fp4", 14, 2, 64), ("bf16", "fp4", 20, 1, 64), ("fp16", "fp4", 3, 3, 128),
              ("bf16", "bf16", 12, 12, 64), ("bf16", "bf16", 40, 8, 128)]
IDS = ["-".join(map(str, g)) for g in GEOMETRIES]


class Scored:
    """A Step whose queries score the cache: the logarithms of its sums as 32-bit inputs, previous scores, outputs."""

    def __init__(self, rng, step, decay=1.0, with_prev=True, in_place=False):
        import torch
        self.st, self.decay, self.in_place = step, decay, in_place
        c = step.c
        self.seen, lse = [], np.full((max(1, step.n), c.hq), -np.inf)
        q = to64(step.q_all)[:step.n, :c.hq * c.d].reshape(step.n, c.hq, c.d)
        self.scores = []                                     # per query row: entries seen, scaled scores [hq, seen], their error
        for r in range(len(step.ids)):
            live = [(e, i, s) for e, (i, s) in enumerate(zip(step.ids[r], step.slots[r])) if 0 <= s < c.slots]
            for j, p in enumerate(step.positions[r]):
                row = int(step.q_off[r]) + j
                seen = [(e, s) for e, i, s in live if i <= p and (not step.window or i > p - step.window or i < step.sinks)]
                if not seen:
                    self.scores.append((r, [], None, None))
                    continue
                k = np.repeat(np.stack([c.k64[s] for _, s in seen]), c.hq // c.hkv, 1)
                with np.errstate(all="ignore"):
                    x = np.einsum("hd,lhd->hl", q[row], k) * step.sm_scale
                    # see Step.reference: a 32-bit sum of D exact products, in any order, cutting accumulators
                    ds = c.d * 2.0 ** -23 * np.einsum("hd,lhd->hl", np.abs(q[row]), np.abs(k)) * abs(step.sm_scale)
                    top = x.max(-1)
                    lse[row] = np.where(np.isfinite(top), top + np.log(np.exp(x - np.where(np.isfinite(top), top, 0)[:, None]).sum(-1)), top)
                self.scores.append((r, [e for e, _ in seen], x, ds))
        self.lse64 = lse.astype(np.float32).astype(np.float64)
        self.lse = torch.from_numpy(lse.astype(np.float32)).to(c.dev)
        self.prev64 = rng.random(c.max_tokens).astype(np.float32).astype(np.float64) if with_prev else np.zeros(c.max_tokens)
        self.prev = torch.from_numpy(self.prev64.astype(np.float32)).to(c.dev) if with_prev else None
        self.out = self.prev if in_place else torch.full((c.max_tokens,), 77.0, device=c.dev)
        n = vt.vtoken_token_weights_workspace_bytes(c.ctx, c.heads, max(1, step.n))
        self.workspace, self.workspace_bytes = torch.zeros(max(16, n), dtype=torch.uint8, device=c.dev), n

    def call(self, stream=None, **changed):
        st, c = self.st, self.st.c
        args = dict(heads=c.heads, layer=c.layer, num_requests=st.num_requests, q_offsets=st.q_offsets, positions=st.pos,
                    q=st.q_all, max_query_tokens=st.n, max_query_len=st.max_query_len, tt_offsets=st.tt_offsets,
                    cache_slots=st.cache_slots, cache_ids=st.cache_ids, cache_len=st.cache_len, lse=self.lse,
                    sm_scale=st.sm_scale, window=st.window, sinks=st.sinks, decay=self.decay, prev=self.prev, scores=self.out,
                    q_stride=st.stride, workspace=self.workspace, workspace_bytes=self.workspace_bytes, stream=stream)
        vt.vtoken_token_weights(c.ctx, **{**args, **changed})
        return self

    def reference(self):
        """(score per table entry, bound of its error), float64; 77 (or the score before, in place) where nothing is written."""
        st, c = self.st, self.st.c
        ref = self.prev64.copy() if self.in_place else np.full(c.max_tokens, 77.0)
        tol = np.zeros(c.max_tokens)
        weight = [np.zeros(len(i)) for i in st.ids]
        err = [np.zeros(len(i)) for i in st.ids]
        terms = [np.zeros(len(i)) for i in st.ids]
        for row, (r, entries, x, ds) in enumerate(self.scores):
            if not entries:
                continue
            lse = self.lse64[row][:, None]
            with np.errstate(all="ignore"):
                w = np.where(np.isneginf(lse), 0.0, np.exp(x - lse))
                # relative: the score's own error; factor and logarithm rounded to 32 bits and one rounding of their difference; exp2 to
                # 2^-22.  The scores are far from the logarithms at times: all of these grow with both
                e = w * (ds + 2.0 ** -22 * (np.abs(x) + np.abs(np.where(np.isneginf(lse), 0, lse)) + 1) * 1.5)
                e = np.where(w == 0, 0.0, e)                 # (a score of minus infinity: its bound is no number)
            weight[r][entries] += w.sum(0)
            err[r][entries] += e.sum(0)
            terms[r][entries] += c.hq
        for r in range(len(st.ids)):
            if not len(st.positions[r]):
                continue
            at = int(st.offsets[r]) + np.asarray(st.ids[r], int)
            ok = np.asarray(st.ids[r]) < st.offsets[r + 1] - st.offsets[r]
            old = self.decay * self.prev64[at[ok]] if self.prev is not None and self.decay else 0.0
            ref[at[ok]] = old + weight[r][ok]
            # 2^-24 of the sum for each term (they have one sign), two more for the score before
            tol[at[ok]] = err[r][ok] + (terms[r][ok] + 2) * 2.0 ** -24 * (weight[r][ok] + np.abs(old)) + 1e-38
        return ref, tol

    def check(self):
        ref, tol = self.reference()
        out = to64(self.out)
        fine = np.isfinite(ref)
        assert np.array_equal(np.isfinite(out), fine)
        off = np.abs(out - ref)[fine]
        assert (off <= tol[fine]).all(), f"off by {off.max()} ({np.max(off / np.maximum(tol[fine], 1e-300))} of the bound)"
        return out


def problem(rng, geometry, lens, positions=None, keep=1.0, window=0, sinks=0, cache_options=None, decay=1.0, with_prev=True,
            in_place=False, **step_options):
    act, kv, hq, hkv, d = geometry
    ids, slots, total = spread(rng, lens, keep)
    used = np.concatenate([np.asarray(s) for s in slots] + [np.zeros(0, int)]).astype(int)
    # scores lie at tt_offsets + id: the table has room for every logical token
    c = Cache(rng, kv, act, hq, hkv, d, total, used, max_requests=max(8, len(lens)), max_tokens=max(64, sum(lens) + 64 + 8 * len(lens)),
              **(cache_options or {}))
    if positions is None:
        positions = [[n - 1] if n else [0] for n in lens]
    st = RoomyStep(rng, c, ids, slots, positions, window, sinks, lens=lens, **step_options)
    return Scored(rng, st, decay, with_prev, in_place)


class RoomyStep(Step):
    """A Step whose tables have an entry for every logical token, evicted or not."""

    def __init__(self, rng, cache, ids, slots, positions, window=0, sinks=0, lens=None, gap=0, **options):
        import torch
        super().__init__(rng, cache, ids, slots, positions, window, sinks, **options)
        R = len(ids)
        self.offsets = np.concatenate([[0], np.cumsum([n + gap for n in lens])]).astype(np.int32)
        s, i = np.full(cache.max_tokens, 1 << 30, np.int32), np.full(cache.max_tokens, 7, np.int32)
        for r in range(R):
            o = self.offsets[r]
            s[o:o + len(ids[r])], i[o:o + len(ids[r])] = slots[r], ids[r]
        self.tt_offsets[:R + 1] = torch.from_numpy(self.offsets).to(cache.dev)
        self.cache_slots = torch.from_numpy(s).to(cache.dev)
        if self.cache_ids is not None:
            self.cache_ids = torch.from_numpy(i).to(cache.dev)


def run_and_check(sc):
    out = sc.call().check()
    assert sc.st.c.flags() == 0
    sc.st.c.close()
    return out


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
def test_single_tokens_of_every_length(geometry):
    rng = np.random.default_rng(1)
    run_and_check(problem(rng, geometry, [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 300, 0, 1000], identity=True))


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 4), (129, 17), (5000, 4)])
def test_window_and_sinks_over_an_evicted_cache(geometry, window, sinks):
    rng = np.random.default_rng(2)
    run_and_check(problem(rng, geometry, [1, 5, 40, 200, 777, 1300], keep=0.4, window=window, sinks=sinks, gap=3, q_pad=8, decay=0.9))


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3)])
def test_several_query_tokens(geometry, window, sinks):
    """1 to 9 query tokens, at the end, in the middle and out of order; a request without any, whose scores stay."""
    rng = np.random.default_rng(3)
    positions = [[39], [195, 196, 197, 198, 199], [3, 100, 50], [], list(range(81, 90))]
    run_and_check(problem(rng, geometry, [40, 200, 333, 70, 90], positions, keep=0.6, window=window, sinks=sinks, in_place=True, decay=0.5))


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
@pytest.mark.parametrize("window,sinks,keep", [(0, 0, 1.0), (0, 0, 0.5), (70, 4, 0.7), (1, 0, 1.0)])
def test_prompts(geometry, window, sinks, keep):
    """Whole prompts and chunks behind a cache, of odd lengths around the tiles; short requests among them."""
    rng = np.random.default_rng(4)
    positions = [[0], list(range(130)), list(range(257)), list(range(171, 300)), list(range(64)), list(range(100, 101))]
    run_and_check(problem(rng, geometry, [1, 130, 257, 300, 64, 200], positions, keep=keep, window=window, sinks=sinks, q_pad=16, gap=1))


@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[5]], ids=["bf16", "fp4"])
@pytest.mark.parametrize("decay,with_prev", [(0.0, True), (0.0, False), (1.0, False), (-0.5, True), (1e-3, True)])
def test_decay(geometry, decay, with_prev):
    """Decay 0 reads no earlier score, not even a NaN; without earlier scores the weights stand alone."""
    rng = np.random.default_rng(5)
    sc = problem(rng, geometry, [40, 200], [[39], list(range(150, 200))], keep=0.7, decay=decay, with_prev=with_prev)
    if decay == 0.0 and with_prev:
        sc.prev.fill_(float("nan"))
    run_and_check(sc)


@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[1], GEOMETRIES[4]], ids=["bf16", "fp16", "fp4"])
@pytest.mark.parametrize("many", [1, 40])
def test_rows_that_see_nothing_and_masked_nan(geometry, many):
    """Positions before every id and outside the window: minus infinity as their logarithm, and nothing added, although keys that
    such a row must not see hold NaN; the pool is poisoned elsewhere."""
    rng = np.random.default_rng(6)
    act, kv, hq, hkv, d = geometry
    lens = [60, 100]
    ids = [np.arange(10, 60), np.array([3, 4, 5, 90])]
    slots = [np.arange(50), np.array([70, 71, 72, 73])]
    c = Cache(rng, kv, act, hq, hkv, d, 96, np.concatenate(slots), max_tokens=512)
    positions = [([9, 30, -1, 20, 8] * many)[:many], ([80, 2, 4, 95] * many)[:max(1, many - 1)]]
    import torch
    bad = int(slots[0][25])                                   # id 35: beyond every position of the first request
    if kv == "fp4":
        c.k_pool[c.layer, bad, hkv * d // 2:hkv * d // 2 + hkv * d // 16] = 0x7f
    else:
        c.k_pool[c.layer, bad] = float("nan")
    torch.cuda.synchronize()
    run_and_check(Scored(rng, RoomyStep(rng, c, ids, slots, positions, 6, 0, lens=lens)))


@pytest.mark.parametrize("many", [1, 3, 60])
@pytest.mark.parametrize("group", [1, 3])
def test_infinite_keys_follow_the_definition(many, group):
    """A key channel at infinity that the queries are positive in: minus infinity with a negative factor, and weight 0 -- also
    next to rows of the tile that are not there."""
    import torch
    rng = np.random.default_rng(7)
    sc = problem(rng, ("bf16", "bf16", group, 1, 64), [200], [list(range(200 - many, 200))])
    c, st = sc.st.c, sc.st
    st.q_all[:, 3::64] = 1.0
    s = int(st.slots[0][20])
    c.k_pool[c.layer, s, 3] = float("-inf")
    c.k64[s] = c.k64[s].copy()
    c.k64[s][0, 3] = -np.inf
    torch.cuda.synchronize()
    sc = Scored(rng, st)
    out = sc.call().check()
    assert out[20] == sc.prev64[20]
    c.close()


def test_slots_and_ids_outside_are_flagged():
    import torch
    rng = np.random.default_rng(8)
    for many in (1, 50):
        sc = problem(rng, GEOMETRIES[0], [60, 80], [[59] * many, [79] * many])
        st, c = sc.st, sc.st.c
        o = int(st.offsets[1])
        st.cache_slots[o + 7] = c.slots + 5
        st.slots[1] = st.slots[1].copy()
        st.slots[1][7] = c.slots + 5
        torch.cuda.synchronize()
        sc = Scored(rng, st)
        sc.call().check()
        assert c.flags() == vt.FLAG_BAD_SLOT
        st.cache_ids[o + 79] = 80                            # one behind the table: not written, though it is a token of the cache
        st.ids[1] = st.ids[1].copy()
        st.ids[1][79] = 80
        st.slots[1][7] = -1
        st.cache_slots[o + 7] = -1
        sc = Scored(rng, st)
        sc.call().check()
        assert c.flags() == vt.FLAG_BAD_VICTIM
        c.close()


def test_large_scores_and_scales():
    for scale, q_scale in ((1.0, 30.0), (-0.3, 1.0), (0.0, 1.0), (1e-20, 1.0)):
        rng = np.random.default_rng(9)
        sc = problem(rng, GEOMETRIES[0], [300, 90], [[299], list(range(30, 90))], q_scale=q_scale)
        sc.st.sm_scale = scale
        sc = Scored(rng, sc.st)
        run_and_check(sc)


def test_exponents_of_the_4bit_keys():
    for e in (-37, 25):
        rng = np.random.default_rng(10)
        sc = problem(rng, GEOMETRIES[4], [100, 200], [[99], list(range(140, 200))], cache_options=dict(k_exponent=e))
        sc.st.sm_scale = 2.0 ** -e * 0.1
        run_and_check(Scored(rng, sc.st))


@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[4]], ids=["bf16", "fp4"])
def test_weights_of_attention_sum_to_the_rows(geometry):
    """With the logarithms that attention leaves, the scores of a request sum to its rows times heads."""
    rng = np.random.default_rng(11)
    sc = problem(rng, geometry, [500, 300, 64], [[499], list(range(200, 300)), [60, 61]], keep=0.8, with_prev=False, decay=0.0)
    st = sc.st
    st.run()
    sc.lse = st.lse
    sc.call()
    out = to64(sc.out)
    for r in range(3):
        rows = len(st.positions[r]) * st.c.hq
        total = out[st.offsets[r] + np.asarray(st.ids[r])].sum()
        assert abs(total - rows) <= rows * 2.0 ** -15        # (lse and the scores on either side: 2^-20 (1 + |lse|) and ds, |lse| < 16)
    st.c.close()


def test_streams_graphs_and_calls_that_overlap():
    """A call captured and replayed after its inputs changed, next to one on another stream with a workspace of its own."""
    import torch
    rng = np.random.default_rng(12)
    one = problem(rng, GEOMETRIES[0], [200, 900], [[199], list(range(700, 900))], keep=0.5)
    two = problem(rng, GEOMETRIES[1], [600, 64], [list(range(500, 600)), [63]])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        one.call(stream=torch.cuda.current_stream())
    for seed in (1, 2):
        one.st.q_all.copy_(torch.from_numpy(np.random.default_rng(seed).standard_normal(tuple(one.st.q_all.shape))).to(one.st.q_all))
        fresh = Scored(rng, one.st)
        one.lse.copy_(fresh.lse)
        fresh.out, fresh.prev64 = one.out, one.prev64
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        two.call(stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        fresh.check()
        two.check()
    one.st.c.close()
    two.st.c.close()


@pytest.mark.parametrize("hint", [1, 1000])
def test_any_hint_is_right(hint):
    rng = np.random.default_rng(13)
    positions = [[199], list(range(180, 189)), list(range(100, 300))]
    for geometry in (GEOMETRIES[0], GEOMETRIES[4], GEOMETRIES[3]):
        run_and_check(problem(rng, geometry, [200, 190, 300], positions, keep=0.9, max_query_len=hint))


def test_the_same_call_twice_is_the_same_to_the_bit():
    import torch
    rng = np.random.default_rng(14)
    sc = problem(rng, GEOMETRIES[0], [2000, 700, 300], [[1999], list(range(300, 700)), list(range(200, 300))], keep=0.9)
    sc.call()
    first = sc.out.clone()
    for _ in range(3):
        sc.call()
        torch.cuda.synchronize()
        assert torch.equal(first, sc.out)
    sc.st.c.close()


def test_offsets_beyond_the_capacities_are_clipped():
    import torch
    rng = np.random.default_rng(15)
    sc = problem(rng, GEOMETRIES[0], [40, 50], [[39], [49]])
    st, c = sc.st, sc.st.c
    st.q_offsets[2] = 1 << 20
    st.cache_len[1] = 1 << 20
    st.tt_offsets[2] = 1 << 30
    sc.call()
    torch.cuda.synchronize()
    assert c.flags() & vt.FLAG_CAPACITY
    c.close()


def test_refusals():
    rng = np.random.default_rng(16)
    sc = problem(rng, GEOMETRIES[0], [40, 50])
    c = sc.st.c
    refused = [dict(scores=None), dict(num_requests=None), dict(lse=None), dict(q=None), dict(positions=None), dict(workspace=None),
               dict(tt_offsets=None), dict(cache_slots=None), dict(cache_len=None), dict(q_offsets=None), dict(layer=2), dict(layer=-1),
               dict(decay=float("nan")), dict(decay=float("inf")), dict(sm_scale=float("nan")), dict(sm_scale=1e31), dict(window=-1),
               dict(sinks=-1), dict(max_query_tokens=-1), dict(max_query_len=0), dict(q_stride=c.hq * c.d - 8),
               dict(q_stride=c.hq * c.d + 4), dict(q=sc.st.q_all.data_ptr() + 2), dict(scores=sc.out.data_ptr() + 2),
               dict(lse=sc.lse.data_ptr() + 2), dict(prev=sc.prev.data_ptr() + 1), dict(workspace=sc.workspace.data_ptr() + 4),
               dict(heads=vt.Heads(8, 3, 128, vt.KV_BF16, vt.KV_BF16, 0, 0)), dict(heads=vt.Heads(8, 2, 96, vt.KV_BF16, vt.KV_BF16, 0, 0))]
    before = sc.out.clone()
    for change in refused:
        with pytest.raises(vt.VtokenError) as e:
            sc.call(**change)
        assert e.value.code == vt.EINVAL, change
    with pytest.raises(vt.VtokenError) as e:
        sc.call(workspace_bytes=sc.workspace_bytes - 1)
    assert e.value.code == vt.ECAPACITY
    sc.call(max_query_tokens=0, q=None, positions=None, lse=None)    # a call without rows
    import torch
    torch.cuda.synchronize()
    assert torch.equal(before, sc.out)
    with pytest.raises(vt.VtokenError):
        vt.vtoken_token_weights_workspace_bytes(c.ctx, vt.Heads(8, 3, 128, 0, 0, 0, 0), 4)
    with pytest.raises(vt.VtokenError):
        vt.vtoken_token_weights_workspace_bytes(c.ctx, c.heads, -1)
    c.close()


@pytest.mark.parametrize("group", [65, 128, 130])
def test_many_query_heads_on_a_key_head(group):
    """Row tiles of one query token, and more heads than a tile has rows."""
    rng = np.random.default_rng(17)
    positions = [list(range(290, 300)), [63], list(range(130))]
    run_and_check(problem(rng, ("bf16", "bf16", group, 1, 64), [300, 64, 130], positions, keep=0.8))


def test_more_key_heads_than_warps_and_longer_caches():
    rng = np.random.default_rng(18)
    run_and_check(problem(rng, ("fp16", "fp16", 33, 11, 64), [3000, 17, 900], [[2999], [15, 16], list(range(800, 900))], keep=0.9))


def test_a_projection_of_queries_as_the_input():
    """Queries inside wider rows, and scores of layers added up call by call."""
    rng = np.random.default_rng(19)
    sc = problem(rng, ("bf16", "bf16", 8, 2, 128), [200, 500], [[199], list(range(440, 500))], q_pad=512, in_place=True)
    first = sc.reference()[0]
    sc.call().check()
    sc.prev64 = to64(sc.out).copy()
    sc.call().check()
    assert (sc.reference()[0] >= first - 1e-6).all()
    sc.st.c.close()
