"""Attention over the slot cache against the definition in 64 bits: geometries, lengths, windows, masks that leave rows
empty, poisoned pools, strides, streams, graphs, refusals.  Bounds are derived in attention_sim.Step.reference."""
import numpy as np
import pytest

from attention_sim import Cache, Step, spread, to64
from paper_2608_13263_b200 import binding as vt

pytestmark = pytest.mark.gpu

GEOMETRIES = [("bf16", "bf16", 8, 2, 128), ("fp16", "fp16", 7, 1, 128), ("bf16", "bf16", 4, 4, 64), ("fp16", "fp16", 16, 1, 64),
              ("bf16", "fp4", 8, 2, 128), ("fp16", "fp4", 14, 2, 64), ("bf16", "fp4", 20, 1, 64), ("fp16", "fp4", 3, 3, 128),
              ("bf16", "bf16", 20, 1, 128)]
IDS = ["-".join(map(str, g)) for g in GEOMETRIES]


def problem(rng, geometry, lens, positions=None, keep=1.0, window=0, sinks=0, cache_options=None, **step_options):
    act, kv, hq, hkv, d = geometry
    ids, slots, total = spread(rng, lens, keep)
    used = np.concatenate([np.asarray(s) for s in slots] + [np.zeros(0, int)]).astype(int)
    c = Cache(rng, kv, act, hq, hkv, d, total, used, max_requests=max(8, len(lens)), max_tokens=max(64, sum(lens) + 64 + 8 * len(lens)),
              **(cache_options or {}))
    if positions is None:
        positions = [[n - 1] if n else [0] for n in lens]
    return Step(rng, c, ids, slots, positions, window, sinks, **step_options)


def run_and_check(step):
    step.run()
    out = step.check()
    assert step.c.flags() == 0
    step.c.close()
    return out


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
def test_single_tokens_of_every_length(geometry):
    rng = np.random.default_rng(1)
    lens = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 300, 0, 1000]
    run_and_check(problem(rng, geometry, lens))


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 4), (100, 0), (129, 17), (5000, 4)])
def test_window_and_sinks_over_an_evicted_cache(geometry, window, sinks):
    rng = np.random.default_rng(2)
    lens = [1, 5, 40, 200, 777, 1300]
    run_and_check(problem(rng, geometry, lens, keep=0.4, window=window, sinks=sinks, gap=3, q_pad=8))


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3)])
def test_several_query_tokens(geometry, window, sinks):
    """1 to 9 query tokens, at the end, in the middle and out of order; a request without any."""
    rng = np.random.default_rng(3)
    lens = [40, 200, 333, 70, 90]
    positions = [[39], [195, 196, 197, 198, 199], [3, 100, 50], [], list(range(81, 90))]
    run_and_check(problem(rng, geometry, lens, positions, keep=0.6, window=window, sinks=sinks))


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
@pytest.mark.parametrize("window,sinks,keep", [(0, 0, 1.0), (0, 0, 0.5), (70, 4, 0.7), (1, 0, 1.0)])
def test_prompts(geometry, window, sinks, keep):
    """Whole prompts and chunks behind a cache, of odd lengths around the tiles."""
    rng = np.random.default_rng(4)
    lens = [1, 130, 257, 300, 64, 200]
    positions = [[0], list(range(130)), list(range(257)), list(range(171, 300)), list(range(64)), list(range(100, 101))]
    run_and_check(problem(rng, geometry, lens, positions, keep=keep, window=window, sinks=sinks, q_pad=16, gap=1))


@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[1], GEOMETRIES[4], GEOMETRIES[5]], ids=["bf16", "fp16", "fp4", "fp4-fp16"])
def test_rows_that_see_nothing(geometry):
    """Every token evicted from the window, positions before every id, negative positions: zeros and minus infinity."""
    rng = np.random.default_rng(5)
    act, kv, hq, hkv, d = geometry
    ids = [np.array([10, 11, 50]), np.array([5]), np.array([0, 1]), np.array([3, 4, 5, 90])]
    slots = [np.array([0, 17, 33]), np.array([40]), np.array([60, 61]), np.array([70, 71, 72, 73])]
    for positions in ([[9], [4], [-1], [80]], [[9, 200, 12], [4, 5], [-1, 0, 1], [80, 6, 3, 95] * 10]):
        c = Cache(rng, kv, act, hq, hkv, d, 96, np.concatenate(slots))
        out, lse = run_and_check(Step(rng, c, ids, slots, positions, window=6, sinks=0))
        assert np.isneginf(lse).any() and np.isneginf(lse[0]).all()


@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[1], GEOMETRIES[4]], ids=["bf16", "fp16", "fp4"])
@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("many", [2, 40])
def test_a_later_tokens_nan_does_not_reach_earlier_rows(geometry, value, many):
    """The pool is poisoned wherever no request has a token; here one visible token holds NaN or infinity as well: rows
    that see it are not finite, the others are as if it were not there."""
    import torch
    rng = np.random.default_rng(6)
    lens = [60, 200]
    positions = [list(range(60 - many, 60)) if many < 60 else list(range(60)), list(range(200 - many, 200))]
    st = problem(rng, geometry, lens, positions)
    c = st.c
    for r, tok in ((0, 60 - many // 2), (1, 199)):
        s = int(st.slots[r][tok])
        if c.kv == "fp4":
            c.v_pool[c.layer, s, c.hkv * c.d // 2] = 0x7f
            c.v64[s] = c.v64[s].copy()
            c.v64[s][0, :16] = np.nan
        else:
            c.v_pool[c.layer, s, 3] = value
            c.v64[s] = c.v64[s].copy()
            c.v64[s][0, 3] = value
    torch.cuda.synchronize()
    st.run()
    out, _ = st.outputs()
    ref, _, tol, _ = st.reference()
    fine = np.isfinite(ref)
    assert fine.any() and not fine.all()
    assert np.array_equal(np.isfinite(out), fine)
    assert (np.abs(out - ref)[fine] <= tol[fine]).all()
    c.close()


def test_infinite_scores_follow_the_definition():
    rng = np.random.default_rng(7)
    st = problem(rng, GEOMETRIES[0], [50, 70])
    s = int(st.slots[0][20])
    st.c.k_pool[st.c.layer, s] = float("inf")           # q . k is NaN or an infinity: NaN by the definition, or zero weight
    st.c.k64[s] = np.full_like(st.c.k64[s], np.inf)
    st.run()
    out, _ = st.outputs()
    assert np.isnan(out[0]).any() and np.isfinite(out[1]).all()
    st.c.close()


@pytest.mark.parametrize("scale", [1e-3, 30.0])
@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[1], GEOMETRIES[4], GEOMETRIES[5]], ids=["bf16", "fp16", "fp4", "fp4-fp16"])
def test_flat_and_peaked_softmax(geometry, scale):
    rng = np.random.default_rng(8)
    run_and_check(problem(rng, geometry, [400, 33, 90], positions=[[399], [32], list(range(50, 90))], q_scale=scale))


@pytest.mark.parametrize("exponents", [(0, 0), (-9, 11), (20, -20)])
def test_exponents_of_4_bit_pools(exponents):
    rng = np.random.default_rng(9)
    st = problem(rng, ("bf16", "fp4", 8, 2, 128), [100, 260], positions=[[99], list(range(200, 260))],
                 cache_options=dict(k_exponent=exponents[0], v_exponent=exponents[1]), q_scale=2.0 ** -exponents[0])
    run_and_check(st)


def test_no_ids_means_nothing_was_evicted():
    rng = np.random.default_rng(10)
    for window, sinks in ((0, 0), (30, 2)):
        run_and_check(problem(rng, GEOMETRIES[0], [100, 64, 1], positions=[[99], [10, 63], [0]], window=window, sinks=sinks, identity=True))
        run_and_check(problem(rng, GEOMETRIES[1], [300], positions=[list(range(30, 300))], window=window, sinks=sinks, identity=True))


def test_long_split_rows_are_the_same_twice_and_leave_the_workspace_ready():
    """One long request is cut over many CTAs; the joined rows are right, identical from call to call on one workspace,
    and other problems can use the workspace afterwards."""
    import torch
    rng = np.random.default_rng(11)
    for geometry in (GEOMETRIES[0], GEOMETRIES[4]):
        st = problem(rng, geometry, [9000, 3, 5000], positions=[[8999], [2], [4000, 4999]])
        st.run()
        first = st.check()
        for _ in range(3):
            st.out_all.fill_(9.0)
            st.call()
            again = st.outputs()
            assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])
        torch.cuda.synchronize()
        counters = st.workspace[:4096].cpu().numpy()
        assert not counters.any()
        small = Step(rng, st.c, [st.ids[1]], [st.slots[1]], [[2]])
        small.run(workspace=st.workspace)
        small.check()
        st.c.close()


def test_many_requests():
    """More requests than threads of a CTA, most of them short, some without queries."""
    rng = np.random.default_rng(12)
    lens = [int(n) for n in rng.integers(0, 60, 700)]
    positions = [[n - 1] if n and i % 5 else [] for i, n in enumerate(lens)]
    run_and_check(problem(rng, ("bf16", "bf16", 4, 2, 64), lens, positions))
    positions = [[0, max(0, n - 1), 3] if n and i % 7 else [] for i, n in enumerate(lens)]
    run_and_check(problem(rng, ("fp16", "fp4", 14, 2, 64), lens, positions))


def test_no_requests_and_no_queries():
    rng = np.random.default_rng(13)
    st = problem(rng, GEOMETRIES[0], [50, 60], positions=[[49], [59]])
    st.num_requests.fill_(0)
    st.run()
    assert (to64(st.out_all) == 77.0).all() and st.c.flags() == 0
    st.c.close()
    st = problem(rng, GEOMETRIES[0], [50, 60], positions=[[], []])
    st.run()
    assert st.c.flags() == 0
    st.c.close()


def test_table_faults_are_flagged_and_clipped():
    rng = np.random.default_rng(14)
    # a slot outside the pool: the token is invisible
    for positions in ([[49], [59]], [[49], list(range(60))]):
        st = problem(rng, GEOMETRIES[0], [50, 60], positions=positions)
        st.slots[0] = st.slots[0].copy()
        for i, s in ((7, st.c.slots), (9, -1), (11, 1 << 30)):
            st.slots[0][i] = s
            st.cache_slots[i] = s
        st.run()
        st.check()
        assert st.c.flags() == vt.FLAG_BAD_SLOT
        st.c.close()
    # more query rows than the buffer has, a cache longer than its range, more requests than the capacity
    st = problem(rng, GEOMETRIES[0], [50, 60], positions=[[49], [59]])
    st.q_offsets[2] = 9
    st.cache_len[0] = 5000
    st.run()
    assert st.c.flags() & vt.FLAG_CAPACITY
    assert (to64(st.out_all)[1] != 77.0).all()
    st.num_requests.fill_(1000)
    st.call()
    assert st.c.flags() & vt.FLAG_CAPACITY
    st.c.close()


@pytest.mark.parametrize("kv", ["bf16", "fp4"])
def test_slots_beyond_32_bit_byte_offsets(kv):
    """Rows whose byte offset in the layer passes 2^32."""
    import torch
    rng = np.random.default_rng(15)
    hkv, d, block = 8, 128, 32
    rb = 2048 if kv == "bf16" else 576
    slots = ((1 << 32) // rb // block + 40) * block
    used = np.array([0, 5, slots - 1, slots - 33, slots // 2, slots - 700])
    dtype = torch.bfloat16 if kv == "bf16" else torch.uint8
    pools = [torch.zeros((1, slots, hkv * d if kv == "bf16" else rb), dtype=dtype, device="cuda:0") for _ in range(2)]
    small = Cache(rng, kv, "bf16", 16, hkv, d, 64, np.arange(6), layers=1, poison=False)
    at = torch.from_numpy(used).to("cuda:0")
    for big, little in zip(pools, (small.k_pool, small.v_pool)):
        big[0, at] = little[0, :6]
    geo = (1, rb, 1) if kv == "fp4" else (hkv, d, 2)
    vt.vtoken_destroy(small.ctx)
    small.ctx = vt.vtoken_create(1, slots // block, block, geo[0], geo[1], pools[0], pools[1], 8, 4096, 4096, 4, elem_bytes=geo[2])
    small.slots = slots
    small.k64 = {int(s): small.k64[i] for i, s in enumerate(used)}
    small.v64 = {int(s): small.v64[i] for i, s in enumerate(used)}
    for positions in ([[5]], [list(range(6)) * 7]):
        Step(rng, small, [np.arange(6)], [used], positions).run().check()
    assert small.flags() == 0
    small.close()


def test_other_stream_and_graph_replay():
    import torch
    rng = np.random.default_rng(16)
    for positions in ([[299], [63]], [list(range(40, 300)), list(range(64))]):
        st = problem(rng, GEOMETRIES[0], [300, 64], positions=positions)
        st.run()
        first = st.check()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        st.out_all.fill_(5.0)
        side.wait_stream(torch.cuda.current_stream())
        st.call(stream=side)
        side.synchronize()
        assert np.array_equal(st.outputs()[0], first[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            st.call(stream=torch.cuda.current_stream())
        q = torch.randn_like(st.q_all.float()).to(st.q_all.dtype)
        st.q_all.copy_(q)
        graph.replay()
        torch.cuda.synchronize()
        st.check()
        st.c.close()


@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[3], GEOMETRIES[4], GEOMETRIES[7]], ids=["bf16", "fp16", "fp4", "fp4-fp16"])
def test_every_index_stays_in_its_array(geometry):
    """The checked build: the same results, no index outside its array."""
    prev = vt.use_library("checked")
    try:
        rng = np.random.default_rng(17)
        run_and_check(problem(rng, geometry, [1, 0, 40, 500, 1200], keep=0.5))
        run_and_check(problem(rng, geometry, [1, 130, 300], positions=[[0], list(range(130)), list(range(250, 300))], window=40, sinks=2))
    finally:
        vt.use_library(prev)


def test_refusals():
    rng = np.random.default_rng(18)
    st = problem(rng, GEOMETRIES[0], [50, 60])
    st.run()
    c = st.c
    good = dict(heads=c.heads, layer=c.layer, num_requests=st.num_requests, q_offsets=st.q_offsets, positions=st.pos, q=st.q_all,
                max_query_tokens=st.n, max_query_len=1, tt_offsets=st.tt_offsets, cache_slots=st.cache_slots, cache_ids=st.cache_ids,
                cache_len=st.cache_len, out=st.out_all, lse=st.lse, sm_scale=0.1, workspace=st.workspace,
                workspace_bytes=st.workspace_bytes)

    def refused(code=vt.EINVAL, **change):
        with pytest.raises(vt.VtokenError) as e:
            vt.vtoken_attention(c.ctx, **{**good, **change})
        assert e.value.code == code
    for name in ("num_requests", "q_offsets", "positions", "q", "tt_offsets", "cache_slots", "cache_len", "out", "workspace"):
        refused(**{name: None})
    for change in (dict(layer=-1), dict(layer=2), dict(max_query_tokens=-1), dict(max_query_len=0), dict(window=-1), dict(sinks=-1),
                   dict(sm_scale=float("nan")), dict(sm_scale=float("inf")), dict(q=st.q_all.data_ptr() + 2), dict(out=st.out_all.data_ptr() + 8),
                   dict(q_stride=c.hq * c.d + 4), dict(out_stride=c.hq * c.d - 8), dict(q_stride=-8)):
        refused(**change)
    refused(vt.ECAPACITY, workspace_bytes=st.workspace_bytes - 1)
    H = vt.Heads
    for heads in (H(8, 3, 128, 0, 0, 0, 0), H(8, 2, 96, 0, 0, 0, 0), H(8, 2, 128, 0, 1, 0, 0), H(8, 2, 128, 1, 0, 0, 0), H(8, 2, 128, 3, 0, 0, 0),
                  H(0, 2, 128, 0, 0, 0, 0), H(8, 0, 128, 0, 0, 0, 0), H(8, 4, 128, 0, 0, 0, 0), H(8, 2, 128, 2, 0, 0, 0), H(8, 2, 128, 0, 0, 1, 0)):
        refused(heads=heads)
    assert c.flags() == 0
    c.close()
