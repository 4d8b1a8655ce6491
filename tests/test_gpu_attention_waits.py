"""The waits inside the prompt kernel of vtoken_attention: roles that run late, and waits that run out.  The hooks that make a
role late exist only in the checked build (vtoken_config.debug_stall_item); nothing faults."""
import numpy as np
import pytest

from attention_sim import Cache, Step, spread
from paper_2608_13263_b200 import binding as vt

pytestmark = pytest.mark.gpu

LATE = 1 << 32                   # debug_stall_item: from here on, nanoseconds that the lookup of slots is late at each tile


@pytest.fixture
def checked():
    prev = vt.use_library("checked")
    yield
    vt.use_library(prev)


def prompts(rng, kv, act="bf16", hq=8, hkv=2, d=128, lens=(900, 700), queries=(300, 200)):
    ids, slots, total = spread(rng, lens)
    c = Cache(rng, kv, act, hq, hkv, d, total, np.concatenate(slots), max_tokens=sum(lens) + 64)
    return Step(rng, c, ids, slots, [list(range(n - m, n)) for n, m in zip(lens, queries)])


def context(step, **options):
    """The cache's context again, with options."""
    c = step.c
    rb = c.k_pool.shape[-1]
    geo = (1, rb, 1) if c.kv == "fp4" else (c.hkv, c.d, 2)
    new = vt.vtoken_create(c.layers, c.slots // c.block, c.block, geo[0], geo[1], c.k_pool, c.v_pool, c.max_requests, c.max_tokens,
                           c.max_tokens, 4, elem_bytes=geo[2], **options)
    vt.vtoken_destroy(c.ctx)
    c.ctx = new


@pytest.mark.parametrize("kv,d,queries", [("bf16", 128, (300, 200)), ("bf16", 64, (40, 33)), ("fp4", 128, (300, 20)), ("fp4", 64, (70, 200))])
def test_slots_that_are_looked_up_late(checked, kv, d, queries):
    """20 us at each tile, ten times what a tile takes: the copies and products are always done with what they have before the next
    slots come."""
    st = prompts(np.random.default_rng(20), kv, d=d, queries=queries)
    context(st, debug_stall_item=LATE + 20000)
    st.run().check()
    assert st.c.flags() == 0
    st.c.close()


def test_the_hook_is_checked(checked):
    st = prompts(np.random.default_rng(21), "bf16", lens=(50,), queries=(40,))
    with pytest.raises(vt.VtokenError) as e:
        context(st, debug_stall_item=LATE + 1000001)
    assert e.value.code == vt.EINVAL
    st.c.close()


@pytest.mark.parametrize("kv", ["bf16", "fp4"])
def test_a_wait_that_runs_out(checked, kv):
    """The queries of one work item never come: its CTA gives up after the limit, the call ends with VTOKEN_FLAG_TIMEOUT, every other
    item is right, the workspace is ready for the next call, and that one is right throughout."""
    import torch
    for item in (0, 3):
        st = prompts(np.random.default_rng(22), kv)
        context(st, wait_limit_ms=5, debug_stall_item=item + 1)
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        st.run()
        e1.record()
        torch.cuda.synchronize()
        assert 4.0 < e0.elapsed_time(e1) < 2000.0
        assert st.c.flags() == vt.FLAG_TIMEOUT
        assert not st.workspace[:4096].cpu().numpy().any()
        out, _ = st.outputs()
        ref, _, tol, _ = st.reference()
        # items: pairs of row tiles from a request's last to its first, all key heads of a pair in turn; here of the first request,
        # 1200 rows of 4 heads and 300 tokens: 176 rows, then 256 at a time
        lost = np.zeros(out.shape[:2], bool)
        pair, kv_head = 4 - item // 2, item % 2
        lost[pair * 64:min(300, pair * 64 + 64), 4 * kv_head:4 * kv_head + 4] = True
        assert (out[lost] == 77.0).all()
        assert (np.abs(out - ref)[~lost] <= tol[~lost]).all()
        context(st)
        st.call()
        st.check()
        assert st.c.flags() == 0
        st.c.close()


def test_many_items_when_one_cta_gives_up(checked):
    """More items than SMs: what the CTA that gave up had already taken is lost, the others do the rest."""
    import torch
    st = prompts(np.random.default_rng(23), "bf16", hq=64, hkv=64, d=64, lens=(130, 150, 130), queries=(130, 129, 130))
    context(st, wait_limit_ms=5, debug_stall_item=4)
    st.run()
    torch.cuda.synchronize()
    assert st.c.flags() == vt.FLAG_TIMEOUT
    assert not st.workspace[:4096].cpu().numpy().any()
    out, _ = st.outputs()
    gone = (out == 77.0).all(-1)
    assert 129 <= gone.sum() <= 2 * 130
    context(st)
    st.call()
    st.check()
    assert st.c.flags() == 0
    st.c.close()
