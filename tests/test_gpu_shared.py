"""Attention behind shared prefixes against the definition in 64 bits: every request by itself (attention_sim.Step.reference, whose
bounds hold: parts of a row are joined in 32 bits), whatever the groups."""
import numpy as np
import pytest

from attention_sim import Cache, Step, to64
from paper_2608_13263_b200 import binding as vt

pytestmark = pytest.mark.gpu

GEOMETRIES = [("bf16", "bf16", 8, 2, 128), ("fp16", "fp16", 7, 1, 128), ("bf16", "bf16", 4, 4, 64), ("fp16", "fp16", 16, 1, 64),
              ("bf16", "fp4", 8, 2, 128), ("fp16", "fp4", 14, 2, 64), ("bf16", "fp4", 20, 1, 64), ("fp16", "fp4", 3, 3, 128)]
IDS = ["-".join(map(str, g)) for g in GEOMETRIES]


class Groups:
    """groups: list of (prefix tokens, [own tokens of each member]); keep: share of the tokens that an eviction left."""

    def __init__(self, rng, geometry, groups, queries=None, keep=1.0, window=0, sinks=0, shared=None, outside=0, cache_options=None,
                 identity=False, **step_options):
        act, kv, hq, hkv, d = geometry
        block, at = 16, 0
        ids, slots, self.shared, edges, lens = [], [], [], [outside], []
        total = sum(-(-p // block) + sum(-(-n // block) for n in own) for p, own in groups) * block + 64
        order = rng.permutation(total // block)

        def take(n):
            nonlocal at
            b = -(-n // block)
            mine = order[at:at + b]
            at += b
            i = np.arange(n)
            return mine[i // block] * block + i % block if n else np.zeros(0, int)
        for r, (p, own) in enumerate(groups):
            alive = np.nonzero(rng.random(p) < keep)[0] if keep < 1 else np.arange(p)
            prefix = take(p)[alive]
            for n in own:
                mine = np.nonzero((rng.random(n) < keep) | (np.arange(n) == n - 1))[0] if keep < 1 else np.arange(n)
                ids.append(np.concatenate([alive, p + mine]).astype(int))
                slots.append(np.concatenate([prefix, take(n)[mine]]).astype(int))
                self.shared.append(len(alive))
                lens.append(p + n)
            edges.append(len(ids))
        # requests in front of the first group share nothing, whatever their shared_len says
        edges = [max(outside, e) for e in edges]
        R = len(ids)
        used = np.unique(np.concatenate(slots + [np.zeros(0, int)]).astype(int))
        self.c = Cache(rng, kv, act, hq, hkv, d, total, used, max_requests=max(8, R + 2), max_tokens=max(64, sum(len(i) for i in ids) + 64 + 8 * R),
                       **(cache_options or {}))
        positions = queries(lens) if queries else [[n - 1] if n else [0] for n in lens]
        self.st = Step(rng, self.c, ids, slots, positions, window, sinks, identity=identity, **step_options)
        self.shared = self.shared if shared is None else shared(self.shared)
        dev = lambda x: __import__("torch").tensor(x, dtype=__import__("torch").int32, device="cuda:0")        # noqa: E731
        pad = self.c.max_requests
        self.num_groups = dev([len(edges) - 1])
        self.group_offsets = dev(edges + [R] * (pad + 1 - len(edges)))
        self.shared_len = dev(self.shared + [0] * (pad - R))
        import torch
        n = vt.vtoken_attention_shared_workspace_bytes(self.c.ctx, self.c.heads, max(1, self.st.n))
        self.workspace, self.workspace_bytes = torch.zeros(n, dtype=torch.uint8, device="cuda:0"), n

    def call(self, stream=None, **changed):
        st, c = self.st, self.c
        args = dict(heads=c.heads, layer=c.layer, num_requests=st.num_requests, q_offsets=st.q_offsets, positions=st.pos, q=st.q_all,
                    max_query_tokens=st.n, max_query_len=st.max_query_len, tt_offsets=st.tt_offsets, cache_slots=st.cache_slots,
                    cache_ids=st.cache_ids, cache_len=st.cache_len, out=st.out_all, lse=st.lse, sm_scale=st.sm_scale, window=st.window,
                    sinks=st.sinks, q_stride=st.stride, out_stride=st.stride, workspace=self.workspace, workspace_bytes=self.workspace_bytes,
                    num_groups=self.num_groups, group_offsets=self.group_offsets, shared_len=self.shared_len, stream=stream)
        vt.vtoken_attention_shared(c.ctx, **{**args, **changed})
        return self

    def check(self, flags=0):
        out = self.st.check()
        assert self.c.flags() == flags
        return out

    def close(self):
        self.c.close()


def run_and_check(g):
    out = g.call().check()
    g.close()
    return out


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
@pytest.mark.parametrize("prefix", [1, 127, 128, 129, 300, 1000])
def test_one_group_of_single_tokens(geometry, prefix):
    rng = np.random.default_rng(prefix)
    run_and_check(Groups(rng, geometry, [(prefix, [1, 2, 40, 15, 0, 129, 16, 17, 3])], identity=prefix == 300))


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
@pytest.mark.parametrize("window,sinks,keep", [(0, 0, 0.5), (50, 3, 0.7), (400, 17, 1.0), (1, 0, 1.0)])
def test_groups_windows_and_evictions(geometry, window, sinks, keep):
    """Several groups of several query tokens, a group of one, prefixes of no token, requests without queries."""
    rng = np.random.default_rng(2)
    groups = [(200, [5, 30, 400]), (70, [9]), (0, [40, 50]), (333, [1, 1, 1, 60, 2]), (16, [7, 8])]

    def queries(lens):
        many = [1, 4, 0, 3, 2, 1, 1, 1, 0, 4, 2, 3, 1]
        return [list(range(n - min(m, n), n)) for n, m in zip(lens, many)]
    run_and_check(Groups(rng, geometry, groups, queries, keep=keep, window=window, sinks=sinks, q_pad=8, gap=3))


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
def test_a_group_over_several_row_tiles_and_parts(geometry):
    """More than 256 query rows a key head, a prefix of several parts."""
    rng = np.random.default_rng(3)
    act, kv, hq, hkv, d = geometry
    members = 300 // (hq // hkv) + 2
    run_and_check(Groups(rng, geometry, [(900, [1 + i % 9 for i in range(members)]), (600, [3, 4])], keep=0.9))


@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[1], GEOMETRIES[4]], ids=["bf16", "fp16", "fp4"])
def test_prompts_in_a_group(geometry):
    """Requests of many query rows next to such of few: they read the prefix for themselves, in front, between and behind."""
    rng = np.random.default_rng(4)
    groups = [(200, [150, 3, 300, 5, 6, 2]), (90, [100, 120])]

    def queries(lens):
        many = [150, 1, 290, 2, 1, 90, 100, 1]
        return [list(range(n - min(m, n), n)) for n, m in zip(lens, many)]
    run_and_check(Groups(rng, geometry, groups, queries, keep=0.8))


def test_positions_inside_and_before_the_prefix():
    """Queries that see a part of the prefix only, or nothing at all, in any order."""
    for geometry in (GEOMETRIES[0], GEOMETRIES[4], GEOMETRIES[3]):
        rng = np.random.default_rng(5)
        positions = [[299, 5, 140], [-1, 130], [0], [250, 302]]
        g = Groups(rng, geometry, [(290, [10, 5, 3, 20])], lambda lens: positions)
        out, lse = run_and_check(g)
        assert np.isneginf(lse[3]).all() and (out[3] == 0).all()


def test_rows_that_see_nothing_of_the_prefix():
    rng = np.random.default_rng(6)
    run_and_check(Groups(rng, GEOMETRIES[0], [(500, [300, 200, 100])], window=90))


@pytest.mark.parametrize("shared", [lambda s: [n - i for i, n in enumerate(s)], lambda s: [1 << 20, -4] + s[2:], lambda s: [0] * len(s),
                                    lambda s: [n if i else 1 << 30 for i, n in enumerate(s)]])
def test_shared_lengths_that_differ(shared):
    """The smallest of a group counts, clipped to what its caches hold."""
    rng = np.random.default_rng(7)
    run_and_check(Groups(rng, GEOMETRIES[0], [(300, [20, 5, 0, 7])], shared=shared))


def test_requests_outside_every_group():
    rng = np.random.default_rng(8)
    groups = [(100, [5, 6]), (120, [7, 8, 9]), (64, [3, 3])]
    for outside in (1, 2, 3):
        run_and_check(Groups(rng, GEOMETRIES[0], groups, outside=outside))
    g = Groups(rng, GEOMETRIES[0], groups)
    g.num_groups.fill_(0)
    run_and_check(g)
    g = Groups(rng, GEOMETRIES[0], groups)
    g.num_groups.fill_(1)
    run_and_check(g)


@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[1], GEOMETRIES[4]], ids=["bf16", "fp16", "fp4"])
@pytest.mark.parametrize("value", [np.nan, np.inf])
def test_a_masked_nan_of_the_prefix_stays_there(geometry, value):
    """A token of the prefix that some rows see and others must not holds NaN or infinity."""
    import torch
    rng = np.random.default_rng(9)
    positions = [[199, 100], [203], [140, 150, 160], [204], [90, 149]]
    g = Groups(rng, geometry, [(200, [1, 4, 2, 5, 2])], lambda lens: positions)
    c = g.c
    s = int(g.st.slots[0][150])
    if c.kv == "fp4":
        c.v_pool[c.layer, s, c.hkv * c.d // 2] = 0x7f
        c.v64[s] = c.v64[s].copy()
        c.v64[s][0, :16] = np.nan
    else:
        c.v_pool[c.layer, s, 3] = value
        c.v64[s] = c.v64[s].copy()
        c.v64[s][0, 3] = value
    torch.cuda.synchronize()
    g.call()
    out, _ = g.st.outputs()
    ref, _, tol, _ = g.st.reference()
    fine = np.isfinite(ref)
    assert fine.any() and not fine.all()
    assert np.array_equal(np.isfinite(out), fine)
    assert (np.abs(out - ref)[fine] <= tol[fine]).all()
    g.close()


def test_slots_outside_the_pool_are_invisible():
    import torch
    rng = np.random.default_rng(10)
    g = Groups(rng, GEOMETRIES[0], [(200, [5, 6, 7])])
    for r in range(3):
        o = int(g.st.offsets[r])
        g.st.cache_slots[o + 77] = g.c.slots + 3
        g.st.slots[r] = g.st.slots[r].copy()
        g.st.slots[r][77] = g.c.slots + 3
    torch.cuda.synchronize()
    g.call().check(flags=vt.FLAG_BAD_SLOT)
    g.close()


def test_exponents_and_factors():
    for scale, ke, ve in ((1.0, 5, -7), (-0.4, -20, 30), (0.0, 0, 0)):
        rng = np.random.default_rng(11)
        g = Groups(rng, GEOMETRIES[4], [(300, [20, 5, 7])], cache_options=dict(k_exponent=ke, v_exponent=ve))
        g.st.sm_scale = scale * 2.0 ** -ke * 0.1
        g.call()
        out, lse = g.st.outputs()
        ref, ref_lse, tol, lse_tol = g.st.reference()
        # (the absolute floor of the bound is for values around 1)
        assert (np.abs(out - ref) <= tol + 2.0 ** -8 * np.abs(ref).max(-1, keepdims=True)).all()
        assert (np.abs(lse - ref_lse) <= lse_tol).all()
        g.close()


@pytest.mark.parametrize("hint", [1, 1000])
def test_any_hint_is_right(hint):
    for geometry in (GEOMETRIES[0], GEOMETRIES[4]):
        rng = np.random.default_rng(12)
        positions = [[210], list(range(200, 209)), list(range(100, 260))]
        run_and_check(Groups(rng, geometry, [(200, [11, 9, 60])], lambda lens: positions, max_query_len=hint))


def test_equal_to_attention_without_sharing():
    """The same rows as vtoken_attention to the last bits, give or take the order of sums."""
    import torch
    rng = np.random.default_rng(13)
    g = Groups(rng, GEOMETRIES[0], [(700, [40, 5, 60, 7, 300])])
    g.st.run()
    plain = g.st.out_all.clone()
    g.st.out_all.fill_(5.0)
    g.call().check()
    assert (plain.float() - g.st.out_all.float()).abs().max() < 2.0 ** -5
    first = g.st.out_all.clone()
    for _ in range(3):                                       # and the same bits from call to call
        g.st.out_all.fill_(5.0)
        g.call()
        torch.cuda.synchronize()
        assert torch.equal(first, g.st.out_all)
    g.close()


def test_streams_and_graphs():
    import torch
    rng = np.random.default_rng(14)
    one = Groups(rng, GEOMETRIES[0], [(500, [40, 5, 60, 7]), (80, [3, 4])])
    two = Groups(rng, GEOMETRIES[4], [(300, [9, 8, 7])])
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        one.call(stream=torch.cuda.current_stream())
    for seed in (1, 2):
        q = np.random.default_rng(seed).standard_normal(tuple(one.st.q_all.shape))
        one.st.q_all.copy_(torch.from_numpy(q).to(one.st.q_all))
        one.st.out_all.fill_(7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        two.call(stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        one.check()
        two.check()
    one.close()
    two.close()


def test_tables_beyond_the_capacities_are_clipped():
    import torch
    rng = np.random.default_rng(15)
    for field, at, value in (("group_offsets", 1, 1 << 20), ("group_offsets", 0, -3), ("num_groups", 0, 1 << 20), ("group_offsets", 1, -5)):
        g = Groups(rng, GEOMETRIES[0], [(100, [5, 6]), (120, [7, 8, 9])])
        getattr(g, field)[at] = value
        g.call()
        torch.cuda.synchronize()
        assert g.c.flags() & vt.FLAG_CAPACITY
        g.close()


def test_refusals():
    import torch
    rng = np.random.default_rng(16)
    g = Groups(rng, GEOMETRIES[0], [(100, [5, 6])])
    before = g.st.out_all.clone()
    for change in (dict(num_groups=None), dict(group_offsets=None), dict(shared_len=None), dict(q=None), dict(out=None), dict(layer=7),
                   dict(workspace=None), dict(window=-1), dict(max_query_tokens=-1), dict(max_query_len=0), dict(sm_scale=float("nan")),
                   dict(workspace=g.workspace.data_ptr() + 8), dict(cache_len=None), dict(q_stride=12)):
        with pytest.raises(vt.VtokenError) as e:
            g.call(**change)
        assert e.value.code == vt.EINVAL, change
    for n in (0, g.workspace_bytes - 1):
        with pytest.raises(vt.VtokenError) as e:
            g.call(workspace_bytes=n)
        assert e.value.code == vt.ECAPACITY
    g.call(max_query_tokens=0, q=None, out=None, positions=None)
    torch.cuda.synchronize()
    assert torch.equal(before, g.st.out_all)
    with pytest.raises(vt.VtokenError):
        vt.vtoken_attention_shared_workspace_bytes(g.c.ctx, g.c.heads, -1)
    g.close()


@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[4]], ids=["bf16", "fp4"])
def test_a_masked_nan_next_to_single_tokens(geometry):
    """Requests of one query token, whose own tokens are never masked: what they must not see is in the prefix alone."""
    import torch
    rng = np.random.default_rng(17)
    g = Groups(rng, geometry, [(200, [1, 4, 2, 5, 2, 1])], lambda lens: [[199], [120], [149], [204], [3], [150]])
    c, s = g.c, int(g.st.slots[0][150])
    if c.kv == "fp4":
        c.v_pool[c.layer, s, c.hkv * c.d // 2] = 0x7f
        c.v64[s] = c.v64[s].copy()
        c.v64[s][0, :16] = np.nan
    else:
        c.v_pool[c.layer, s, 3] = float("nan")
        c.v64[s] = c.v64[s].copy()
        c.v64[s][0, 3] = np.nan
    torch.cuda.synchronize()
    g.call()
    out, _ = g.st.outputs()
    ref, _, tol, _ = g.st.reference()
    fine = np.isfinite(ref)
    assert fine[[1, 2, 4]].all() and not fine[[0, 3, 5]].all((1, 2)).any()
    assert np.array_equal(np.isfinite(out), fine)
    assert (np.abs(out - ref)[fine] <= tol[fine]).all()
    g.close()


def test_many_short_requests_behind_windowed_prefixes():
    """More segments than shares of tiles, most of the prefix out of sight."""
    rng = np.random.default_rng(18)
    run_and_check(Groups(rng, ("fp16", "fp16", 7, 1, 128), [(400, [28] * 14), (300, [5] * 20), (64, [33] * 30)], window=45))
