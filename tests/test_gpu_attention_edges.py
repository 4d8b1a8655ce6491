"""Attention over the slot cache at the edges of what the header promises: hints that are wrong, positions and scales at the ends of
their types, softmax weights far below one, values that a row may not see, calls without tokens.  References in 64 bits."""
import numpy as np
import pytest

from attention_sim import Cache, Step, quantise_rows, dequantise_rows, spread, to64, torch_dtype, unit
from paper_2608_13263_b200 import binding as vt
from test_gpu_attention import problem, run_and_check

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
