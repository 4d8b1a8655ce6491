"""Attention over the slot cache at the edges of what the header promises: hints that are wrong, positions and scales at the ends of
their types, softmax weights far below one, values that a row may not see, calls without tokens.  References in 64 bits."""
import numpy as np
import pytest

from attention_sim import Cache, Step, quantise_rows, dequantise_rows, spread, to64, torch_dtype, unit
from paper_2608_13263_b200 import binding as vt
from test_gpu_attention import GEOMETRIES, IDS, problem, run_and_check

pytestmark = pytest.mark.gpu


# ---- hints ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("geometry", [("bf16", "bf16", 8, 2, 128), ("fp16", "fp4", 14, 2, 64)], ids=["16", "4"])
@pytest.mark.parametrize("hint", [1, 7, 100000])
def test_the_longest_query_is_a_hint(geometry, hint):
    rng = np.random.default_rng(30)
    lens = [300, 1, 77, 130]
    positions = [list(range(120, 300)), [0], [76], list(range(130))]
    for window, sinks in ((0, 0), (40, 3)):
        run_and_check(problem(rng, geometry, lens, positions, keep=0.7, window=window, sinks=sinks, max_query_len=hint))
        run_and_check(problem(rng, geometry, lens, window=window, sinks=sinks, max_query_len=hint))


def test_more_tiles_than_32_bits_count():
    """One request of 140 000 tokens over 264 000 entries with 8 heads a key head and a hint of one: 2.3e9 tiles.  The first query
    sees everything, the others the first token alone."""
    import torch
    dev, n, m, d, hq = "cuda:0", 264000, 140000, 64, 8
    gen = torch.Generator(device=dev).manual_seed(31)
    draw = lambda *shape: torch.randn(*shape, generator=gen, device=dev).to(torch.bfloat16)    # noqa: E731
    i32 = dict(dtype=torch.int32, device=dev)
    k, v, q = draw(1, n, d), draw(1, n, d), draw(m, hq, d)
    slots = torch.randperm(n, generator=gen, device=dev).int()
    ctx = vt.vtoken_create(1, n // 16, 16, 1, d, k, v, 1, n, n, 1, elem_bytes=2)
    heads = vt.Heads(hq, 1, d, vt.KV_BF16, vt.KV_BF16, 0, 0)
    size = vt.vtoken_attention_workspace_bytes(ctx, heads, m)
    positions = torch.zeros(m, **i32)
    positions[0] = n - 1
    out, lse = torch.full_like(q, 9.0), torch.full((m, hq), 9.0, device=dev)
    vt.vtoken_attention(ctx, heads=heads, layer=0, num_requests=torch.ones(1, **i32), q_offsets=torch.tensor([0, m], **i32),
                        positions=positions, q=q, max_query_tokens=m, max_query_len=1, tt_offsets=torch.tensor([0, n], **i32),
                        cache_slots=slots, cache_len=torch.tensor([n], **i32), out=out, lse=lse, sm_scale=0.125,
                        workspace=torch.zeros(size, dtype=torch.uint8, device=dev), workspace_bytes=size)
    assert vt.vtoken_read_counts(ctx)["error_flags"] == 0
    first = int(slots[0])
    assert (out[1:] == v[0, first]).all()                    # one weight, exactly one
    one = (q[1:].double() @ k[0, first].double()) * 0.125
    assert ((lse[1:].double() - one).abs() < 1e-4).all()     # a sum of 64 products of values up to 5
    s = q[0].double() @ k[0, slots.long()].double().T * 0.125
    w = torch.softmax(s, -1)
    ref = w @ v[0, slots.long()].double()
    # scores off by 64 * 2^-23 * 0.125 * sum |q k| < 1e-4; sums of 264 000 weights; the output's rounding
    assert ((out[0].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (2e-4 + 2.0 ** -16) * v.double().abs().max()).all()
    assert ((lse[0].double() - torch.logsumexp(s, -1)).abs() < 2e-4).all()
    vt.vtoken_destroy(ctx)


# ---- what is read ---------------------------------------------------------------------------------
@pytest.mark.parametrize("kv", ["bf16", "fp4"])
@pytest.mark.parametrize("group,queries", [(1, 9), (1, 32), (2, 16), (3, 10), (4, 40)])
@pytest.mark.parametrize("hint", [None, 1])
def test_tokens_that_no_query_sees_are_not_read(kv, group, queries, hint):
    """Behind the window and after the last position every row of the request is NaN or has a slot that is not in the pool: no flag,
    finite outputs.  With 9 and more query tokens, over both kernels and with a hint that is too small."""
    rng = np.random.default_rng(32)
    first, last, window, sinks = 2000, 2000 + queries, 50, 3
    for keep in (1.0, 0.4):
        ids, slots, total = spread(rng, [3000, 40], keep)
        seen = (ids[0] < sinks) | ((ids[0] > first - window) & (ids[0] < last))
        c = Cache(rng, kv, "bf16", 2 * group, 2, 128, total, np.concatenate([slots[0][seen], slots[1]]), max_tokens=3200)
        given = slots[0].copy()
        given[~seen & (ids[0] % 3 == 0)] = c.slots + 5
        for s in given[~seen]:
            c.k64[int(s)] = c.v64[int(s)] = np.full((2, 128), np.nan)
        st = Step(rng, c, ids, [given, slots[1]], [list(range(first, last)), [39]], window, sinks, max_query_len=hint)
        st.run()
        st.check()
        assert c.flags() == 0
        c.close()


# ---- weights far below one ------------------------------------------------------------------------
def fill(c, slots, k, v):
    """Keys and values [n, heads, d] into the rows of the slots."""
    import torch
    at = torch.from_numpy(slots).to(c.dev)
    for pool, x, name in ((c.k_pool, k, "k64"), (c.v_pool, v, "v64")):
        if c.kv == "fp4":
            rows = quantise_rows(x)
            pool[c.layer, at] = torch.from_numpy(rows).to(c.dev)
            x = dequantise_rows(rows, c.hkv, c.d)
        else:
            rows = torch.from_numpy(x.reshape(len(slots), -1)).to(c.dev).to(torch_dtype(c.act))
            pool[c.layer, at] = rows
            x = to64(rows).reshape(x.shape)
        setattr(c, name, dict(zip(slots.tolist(), x)))


def one_strong_token(geometry, n, gap, strong, rest, queries, hint=None):
    """A cache of n tokens whose first scores `gap` (in natural units, about) above all others, which score zero."""
    act, kv, hq, hkv, d = geometry
    rng = np.random.default_rng(33)
    ids, slots, total = spread(rng, [n])
    c = Cache(rng, kv, act, hq, hkv, d, total, slots[0], max_tokens=n + 64)
    k, v = np.zeros((n, hkv, d)), np.full((n, hkv, d), float(rest))
    k[0], v[0] = gap / d ** 0.5, strong
    fill(c, slots[0], k, v)
    st = Step(rng, c, ids, slots, [list(range(n - queries, n))], max_query_len=hint)
    st.q_all.fill_(1.0)
    return st, k, v


STRONG = [("fp16", "fp16", 4, 1, 64), ("bf16", "fp4", 4, 1, 64), ("fp16", "fp4", 4, 1, 128), ("bf16", "bf16", 4, 1, 128)]


@pytest.mark.parametrize("geometry", STRONG, ids=["fp16", "bf16-fp4", "fp16-fp4", "bf16"])
@pytest.mark.parametrize("queries,hint", [(1, None), (3, None), (12, None), (12, 1)])
def test_a_long_flat_tail_behind_one_strong_token(geometry, queries, hint):
    """Weights of about 2^-26 by the ten thousands: together 2^-11, each below half of the smallest 16-bit value of half precision."""
    n = 33000
    st, _, _ = one_strong_token(geometry, n, 18.0, 0.0, 6.0, queries, hint)
    st.run()
    out, lse = st.outputs()
    ref, ref_lse, _, lse_tol = st.reference()
    assert (ref > 0.001).all()
    # the output's rounding; scores as in attention_sim, here exact products of equal values (2^-20 of 18 on the weights); weights held
    # once in half precision at 2^7 times their size are off by 2^-25 - 7 each at most, or by one rounding
    tol = 1.01 * unit(geometry[0]) * ref + ref * (2.0 ** -20 * 20 + 2.0 ** -10) + 6 * n * 2.0 ** -32 + 2.0 ** -24
    assert (np.abs(out - ref) <= tol).all(), (np.abs(out - ref) / tol).max()
    assert (np.abs(lse - ref_lse) <= lse_tol).all()
    st.c.close()


@pytest.mark.parametrize("geometry", [("fp16", "fp16", 16, 8, 64), ("bf16", "fp4", 16, 8, 64), ("fp16", "fp4", 16, 8, 64)],
                         ids=["fp16", "bf16-fp4", "fp16-fp4"])
def test_many_requests_with_one_long_flat_tail(geometry):
    """The same cache for 128 requests: each warp meets the strong token and ten thousand others."""
    act, kv, hq, hkv, d = geometry
    n, R = 33000, 128
    st, k, v = one_strong_token(geometry, n, 18.0, 0.0, 6.0, 1)
    c, ids, slots = st.c, st.ids[0], st.slots[0]
    c.max_requests, c.max_tokens = R, R * n
    rb = c.k_pool.shape[-1]
    geo = (1, rb, 1) if kv == "fp4" else (hkv, d, 2)
    vt.vtoken_destroy(c.ctx)
    c.ctx = vt.vtoken_create(c.layers, c.slots // c.block, c.block, geo[0], geo[1], c.k_pool, c.v_pool, R, R * n, R * n, 4, elem_bytes=geo[2])
    st = Step(np.random.default_rng(42), c, [ids] * R, [slots] * R, [[n - 1]] * R)
    st.q_all.fill_(1.0)
    st.run()
    out, lse = st.outputs()
    k0, tail = float(c.k64[int(slots[0])][0, 0]), float(c.v64[int(slots[1])][0, 0])
    z = 1 + (n - 1) * np.exp(-k0 * d ** 0.5)
    ref = tail * (z - 1) / z
    # as above
    tol = 1.01 * unit(act) * ref + ref * (2.0 ** -20 * 20 + 2.0 ** -10) + 6 * n * 2.0 ** -32 + 2.0 ** -24
    assert (np.abs(out - ref) <= tol).all(), np.abs(out - ref).max() / tol
    # scores as above; a 32-bit sum that starts at one takes n / 8 additions of 2^-26 each with an error of 2^-24 at most
    assert (np.abs(lse - (k0 * d ** 0.5 + np.log(z))) <= 2.0 ** -20 * 20 + (n / 8 + 64) * 2.0 ** -24).all()
    c.close()


@pytest.mark.parametrize("geometry", STRONG, ids=["fp16", "bf16-fp4", "fp16-fp4", "bf16"])
@pytest.mark.parametrize("queries", [1, 2, 5, 40])
@pytest.mark.parametrize("gap", [0.55, 0.7, 0.86])
def test_weights_that_cancel(geometry, queries, gap):
    """Every other token scores `gap` more than the rest and has values of opposite sign: the output is small, so neither its own
    rounding nor a bound by max |v| hides the rounding of the weights.  Few rows over 16-bit rows have it twice as fine."""
    act, kv, hq, hkv, d = geometry
    n = 1002 + queries
    st, k, v = one_strong_token(geometry, n, 0.0, 1.5, 1.5, queries)
    k[1::2], v[1::2] = gap / d ** 0.5, -1.5 * np.exp(-gap)
    fill(st.c, st.slots[0], k, v)
    st.run()
    out, _ = st.outputs()
    ref, _, _, _ = st.reference()
    # one rounding of the weights to 16 bits, relative 2^-9 or 2^-12; as the sum of two, 2^-17 or less
    split = kv != "fp4" and queries * hq // hkv <= 32
    held = 2.0 ** -17 if split else (2.0 ** -9 if act == "bf16" and kv != "fp4" else 2.0 ** -12)
    # scores: exact products, 32-bit scale and exponential (2^-20 of the largest score); the sums, n / 8 32-bit additions each
    soft = 2.0 ** -20 * (1 + gap) + (n / 8 + 64) * 2.0 ** -23
    tol = 1.01 * unit(act) * np.abs(ref) + 1.5 * (held + 2 * soft) + 2.0 ** -24
    assert (np.abs(out - ref) <= tol).all(), (np.abs(out - ref) / tol).max()
    st.c.close()


# ---- ends of the types ----------------------------------------------------------------------------
@pytest.mark.parametrize("kv", ["bf16", "fp4"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 0), (100, 5)])
def test_the_largest_position(kv, window, sinks):
    """2^31 - 1 sees every token without a window, the first ones with one; nothing that is not there."""
    rng = np.random.default_rng(34)
    top = 2 ** 31 - 1
    for positions in ([[top], [top], [10]], [[top, 5], [top - 1, top], [top]], [[top] * 40, [20] * 20 + [top] * 30, [top]]):
        run_and_check(problem(rng, ("bf16", kv, 8, 2, 128), [37, 300, 16], positions, window=window, sinks=sinks))


@pytest.mark.parametrize("queries", [1, 40])
def test_queries_at_the_upper_end_of_bf16_over_4_bits(queries):
    rng = np.random.default_rng(35)
    st = problem(rng, ("bf16", "fp4", 8, 2, 128), [200], positions=[list(range(200 - queries, 200))],
                 cache_options=dict(k_exponent=-60), q_scale=2.0 ** 115)
    st.sm_scale = 2.0 ** -55 * 128 ** -0.5
    run_and_check(st)


def test_scales_that_leave_32_bits_are_refused():
    rng = np.random.default_rng(36)
    st = problem(rng, ("bf16", "fp4", 8, 2, 128), [50], cache_options=dict(k_exponent=60))
    st.sm_scale = 1e25
    with pytest.raises(vt.VtokenError) as e:
        st.run()
    assert e.value.code == vt.EINVAL
    st.sm_scale = 1e-25
    st.run()
    st.c.close()


def test_an_lse_between_its_words_is_refused():
    import torch
    rng = np.random.default_rng(37)
    st = problem(rng, ("bf16", "bf16", 8, 2, 128), [50])
    lse = st.lse
    st.lse = lse.data_ptr() + 2
    with pytest.raises(vt.VtokenError) as e:
        st.run()
    assert e.value.code == vt.EINVAL
    torch.cuda.synchronize()
    st.c.close()


def test_a_call_without_query_tokens_needs_no_tensors():
    """A tensor without elements has no address."""
    import torch
    rng = np.random.default_rng(38)
    st = problem(rng, ("bf16", "bf16", 8, 2, 128), [50], positions=[[]])
    empty = torch.empty(0, device=st.c.dev, dtype=torch.bfloat16)
    assert empty.data_ptr() == 0
    st.q_all = st.out_all = empty
    st.pos, st.lse = empty.int(), empty.float()
    st.run()
    assert st.c.flags() == 0
    st.c.close()


# ---- values that a row may not see ----------------------------------------------------------------
def poisoned(geometry, lens, positions, where, window=0, sinks=0, value=np.nan, **options):
    """where: (request, id, 'k' or 'v') of rows whose value 3 of head 0 (its first group over 4 bits) is not finite."""
    st = problem(np.random.default_rng(39), geometry, lens, positions, window=window, sinks=sinks, **options)
    c = st.c
    for r, tok, which in where:
        s = int(st.slots[r][list(st.ids[r]).index(tok)])
        pool, host = (c.k_pool, c.k64) if which == "k" else (c.v_pool, c.v64)
        host[s] = host[s].copy()
        if c.kv == "fp4":
            pool[c.layer, s, c.hkv * c.d // 2] = 0x7f
            host[s][0, :16] = np.nan
        else:
            pool[c.layer, s, 3] = value
            host[s][0, 3] = value
    return st


def check_poisoned(st):
    st.run()
    out, _ = st.outputs()
    ref, _, tol, _ = st.reference()
    fine = np.isfinite(ref)
    assert fine.any() and not fine.all()
    assert np.array_equal(np.isfinite(out), fine)
    assert (np.abs(out - ref)[fine] <= tol[fine]).all()
    assert st.c.flags() == 0
    st.c.close()


@pytest.mark.parametrize("geometry", [("bf16", "bf16", 8, 2, 128), ("fp16", "fp16", 7, 1, 128), ("bf16", "fp4", 8, 2, 128), ("fp16", "fp4", 14, 2, 64)],
                         ids=["bf16", "fp16", "fp4", "fp4-fp16"])
@pytest.mark.parametrize("hint", [None, 1])
@pytest.mark.parametrize("queries", [4, 300])
def test_values_that_are_not_finite_reach_the_rows_that_see_them_alone(geometry, hint, queries):
    """Keys and values, in rows that some queries see and others do not (yet, or any more), next to rows that all of them see."""
    n = 600
    positions = [list(range(n - queries, n)), [40, 80, 20]]
    for where in ([(0, n - queries // 2, "v")], [(0, n - queries // 2, "k"), (1, 50, "k")], [(0, 5, "v"), (0, n - 2, "v")],
                  [(0, n - 1, "v"), (1, 30, "v"), (1, 60, "k")], [(0, 0, "v"), (0, n - 3, "k")]):
        check_poisoned(poisoned(geometry, [n, 90], positions, where, max_query_len=hint))
    for where in ([(0, n - queries - 20, "v")], [(0, n - queries - 20, "k"), (1, 30, "v")], [(0, 2, "v"), (0, n - queries // 2, "v")],
                  [(0, n - queries, "v"), (0, n - queries - 10, "v"), (1, 1, "v")]):
        check_poisoned(poisoned(geometry, [n, 90], positions, where, window=30, sinks=4, max_query_len=hint))


@pytest.mark.parametrize("kv", ["bf16", "fp4"])
@pytest.mark.parametrize("queries,n", [(4096, 4096), (4, 60000)])
def test_one_value_that_is_not_finite_does_not_slow_the_call_down(kv, queries, n):
    """The first token is seen by every row: no row can be any better, and none is worked on again."""
    import torch
    times = []
    for where in ([], [(0, 0, "v"), (0, 1, "k")]):
        st = poisoned(("bf16", kv, 8, 2, 128), [n], [list(range(n - queries, n))], where, cache_options=dict(poison=False))
        st.run()
        best = 1e9
        for _ in range(5):
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
            st.call()
            e1.record()
            torch.cuda.synchronize()
            best = min(best, e0.elapsed_time(e1))
        times.append(best)
        out, _ = st.outputs()
        assert np.isfinite(out[:, 4:]).all()
        assert np.isfinite(out[:, :4]).all() == (not where)
        st.c.close()
    assert times[1] < 4 * times[0] + 0.05, times


# ---- many heads side by side, several streams -----------------------------------------------------
@pytest.mark.parametrize("act,hq,hkv,d", [("bf16", 16, 8, 128), ("fp16", 3, 3, 128), ("bf16", 20, 5, 64), ("fp16", 24, 12, 64), ("bf16", 12, 12, 128)])
@pytest.mark.parametrize("many", [False, True])
def test_many_requests_over_4_bits_and_many_heads(act, hq, hkv, d, many):
    """So many requests that the heads of a row are read side by side by a team of warps, with key heads that do not fill it."""
    rng = np.random.default_rng(40)
    lens = [int(n) for n in rng.integers(1, 120, 300)]
    positions = [[n - 1, max(0, n - 2), n // 2][:3 if many else 1] for n in lens]
    run_and_check(problem(rng, (act, "fp4", hq, hkv, d), lens, positions, keep=0.8, window=60, sinks=2))


def test_calls_that_overlap_on_two_streams():
    """A workspace for each stream; one call of few rows and one of prompts at the same time, again and again."""
    import torch
    rng = np.random.default_rng(41)
    few = problem(rng, ("bf16", "bf16", 8, 2, 128), [9000, 3000, 70], positions=[[8999], [2999], [69]])
    many = problem(rng, ("fp16", "fp16", 7, 1, 128), [900, 300], positions=[list(range(300, 900)), list(range(300))])
    few.run()
    many.run()
    want = [st.check() for st in (few, many)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        few.out_all.fill_(9.0)
        many.out_all.fill_(9.0)
        torch.cuda.synchronize()
        for _ in range(3):
            for st, s in zip((few, many), streams):
                st.call(stream=s)
        torch.cuda.synchronize()
        for st, w in zip((few, many), want):
            got = st.outputs()
            assert np.array_equal(got[0], w[0]) and np.array_equal(got[1], w[1])
    for st in (few, many):
        assert st.c.flags() == 0
        st.c.close()


# ---- shapes and factors ---------------------------------------------------------------------------
@pytest.mark.parametrize("geometry", [("bf16", "bf16", 64, 1, 128), ("fp16", "fp4", 96, 1, 64), ("bf16", "fp4", 99, 3, 128), ("fp16", "fp16", 300, 1, 64)],
                         ids=["64", "96-4", "33-4", "300"])
def test_many_query_heads_on_a_key_head(geometry):
    """More than 32 rows from one query token, 128 and 256 rows from a few, tiles that end inside a token's heads."""
    rng = np.random.default_rng(43)
    run_and_check(problem(rng, geometry, [300, 1, 40, 7], positions=[[299], [0], [37, 38, 39], [6]]))
    run_and_check(problem(rng, geometry, [300, 90], positions=[[200, 250, 280, 299], [80]], keep=0.5, window=33, sinks=2))


@pytest.mark.parametrize("kv", ["bf16", "fp4"])
def test_more_prompts_than_threads(kv):
    """600 requests of 40 query rows each, some without queries, some without entries."""
    rng = np.random.default_rng(44)
    lens = [int(n) for n in rng.integers(0, 50, 600)]
    positions = [list(range(max(0, n - 5), max(5, n))) if i % 9 else [] for i, n in enumerate(lens)]
    run_and_check(problem(rng, ("bf16", kv, 8, 1, 64), lens, positions))


@pytest.mark.parametrize("geometry", [("bf16", "bf16", 8, 2, 128), ("fp16", "fp16", 7, 1, 128), ("bf16", "fp4", 8, 2, 128), ("fp16", "fp4", 14, 2, 64)],
                         ids=["bf16", "fp16", "fp4", "fp4-fp16"])
@pytest.mark.parametrize("scale", [-0.1, 0.0, 1e-20, -3.0])
def test_any_factor_of_the_scores(geometry, scale):
    rng = np.random.default_rng(45)
    for window in (0, 40):
        st = problem(rng, geometry, [300, 33, 90], positions=[[299], [32], list(range(20, 90))], window=window)
        st.sm_scale = scale
        run_and_check(st)


# ---- every value counts ---------------------------------------------------------------------------
def held_to(st, row_tokens):
    """Relative rounding of the weights on their way into the product with V: as the sum of two numbers (few rows over 16-bit rows), once
    to the queries' type (prompts over 16-bit rows), once to half precision (over 4-bit rows)."""
    c = st.c
    few = st.max_query_len * c.hq // c.hkv <= 32 or row_tokens * c.hq // c.hkv <= 32
    if c.kv == "fp4":
        return 2.0 ** -12
    return 2.0 ** -17 if few else (2.0 ** -9 if c.act == "bf16" else 2.0 ** -12)


def check_sharply(st):
    """Outputs within their own rounding and errors that are relative to the sum of w |v|, not to the largest |v|: one value that is
    wrong among hundreds shows."""
    st.run()
    c = st.c
    out, _ = st.outputs()
    q = to64(st.q_all)[:st.n, :c.hq * c.d].reshape(st.n, c.hq, c.d)
    for r in range(len(st.ids)):
        for j, p in enumerate(st.positions[r]):
            row = int(st.q_off[r]) + j
            seen = [int(s) for i, s in zip(st.ids[r], st.slots[r]) if i <= p and (not st.window or i > p - st.window or i < st.sinks)]
            if not seen:
                assert (out[row] == 0).all()
                continue
            k, v = (np.repeat(np.stack([x[s] for s in seen]), c.hq // c.hkv, 1) for x in (c.k64, c.v64))
            s = np.einsum("hd,lhd->hl", q[row], k) * st.sm_scale
            w = np.exp(s - s.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            ref, mass = np.einsum("hl,lhd->hd", w, v), np.einsum("hl,lhd->hd", w, np.abs(v))
            # scores as in attention_sim: D * 2^-23 of the sum of |q k|, on both sides of the quotient; sums of n / 8 additions each
            ds = (c.d * 2.0 ** -23 * np.einsum("hd,lhd->hl", np.abs(q[row]), np.abs(k)) * abs(st.sm_scale)).max(-1) + 2.0 ** -20 * (1 + np.abs(s).max(-1))
            soft = held_to(st, len(st.positions[r])) + 2 * ds[:, None] + (len(seen) / 8 + 64) * 2.0 ** -23
            tol = 1.01 * unit(c.act) * np.abs(ref) + soft * mass + 2.0 ** -24
            assert (np.abs(out[row] - ref) <= tol).all(), (r, j, (np.abs(out[row] - ref) / tol).max())
    assert c.flags() == 0
    c.close()


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
def test_outputs_to_their_own_rounding(geometry):
    rng = np.random.default_rng(46)
    check_sharply(problem(rng, geometry, [1, 17, 64, 300, 1000, 3000]))
    check_sharply(problem(rng, geometry, [400, 1500, 33], positions=[[399, 398], [1400, 1499], [30, 31, 32]], keep=0.6, window=200, sinks=4))
    check_sharply(problem(rng, geometry, [300, 700, 20], positions=[list(range(250, 300)), list(range(640, 700)), list(range(20))], keep=0.8))
