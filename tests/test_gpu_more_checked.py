"""The calls that decide what leaves the cache, and attention behind shared prefixes, on the checked build (every index into a table
or scratch range-checked; none may be out of range), and their bounded waits running out there.  Nothing faults."""
import numpy as np
import pytest

import test_gpu_shared as shared
import test_gpu_victims as victims
import test_gpu_weights as weights
from paper_2608_13263_b200 import binding as vt

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def checked():
    prev = vt.use_library("checked")
    yield
    vt.use_library(prev)


@pytest.mark.parametrize("geometry", weights.GEOMETRIES, ids=weights.IDS)
def test_weights(geometry):
    weights.test_window_and_sinks_over_an_evicted_cache(geometry, 129, 17)
    weights.test_several_query_tokens(geometry, 50, 3)
    weights.test_prompts(geometry, 70, 4, 0.7)


@pytest.mark.parametrize("geometry", shared.GEOMETRIES, ids=shared.IDS)
def test_shared(geometry):
    shared.test_groups_windows_and_evictions(geometry, 50, 3, 0.7)
    shared.test_a_group_over_several_row_tiles_and_parts(geometry)


def test_victims():
    victims.test_lengths_and_budgets(False)
    victims.test_what_stays(4, 100)
    victims.test_long_requests_over_several_sms(40000)
    victims.test_many_requests()
    victims.test_vocabularies_and_types("bf16", 4097, True)
    victims.test_numbers_of_drafts([9, 0, 17] * 40, False)


def again(cache, **options):
    """The cache's context again, with options."""
    rb = cache.k_pool.shape[-1]
    geo = (1, rb, 1) if cache.kv == "fp4" else (cache.hkv, cache.d, 2)
    new = vt.vtoken_create(cache.layers, cache.slots // cache.block, cache.block, geo[0], geo[1], cache.k_pool, cache.v_pool,
                           cache.max_requests, cache.max_tokens, cache.max_tokens, 4, elem_bytes=geo[2], **options)
    vt.vtoken_destroy(cache.ctx)
    cache.ctx = new


@pytest.mark.parametrize("geometry", [weights.GEOMETRIES[0], weights.GEOMETRIES[4], weights.GEOMETRIES[5]], ids=["bf16", "fp4", "fp4-fp16"])
def test_a_wait_of_the_scores_that_runs_out(geometry):
    """The first queries of one item never come: its CTA gives up after the limit with VTOKEN_FLAG_TIMEOUT, tokens of other items are
    right, the workspace is ready for the next call, and that one is right throughout."""
    import torch
    sc = weights.problem(np.random.default_rng(30), geometry, [900, 700], [list(range(600, 900)), list(range(500, 700))])
    st, c = sc.st, sc.st.c
    again(c, wait_limit_ms=5, debug_stall_item=1)
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    sc.call()
    e1.record()
    torch.cuda.synchronize()
    assert 4.0 < e0.elapsed_time(e1) < 2000.0
    assert c.flags() == vt.FLAG_TIMEOUT
    assert not sc.workspace[:16].cpu().numpy().any()
    ref, tol = sc.reference()
    off = np.abs(weights.to64(sc.out) - ref) > tol
    # the item is of the first 256 tokens of the first request; the CTA may have drawn another one
    where = {(r, (e - int(st.offsets[r])) // 256) for e in np.nonzero(off)[0] for r in [int(e >= st.offsets[1])]}
    assert (0, 0) in where and len(where) <= 2
    again(c)
    sc.call().check()
    assert c.flags() == 0
    c.close()


def test_a_wait_of_a_prefix_that_runs_out():
    import torch
    g = shared.Groups(np.random.default_rng(31), shared.GEOMETRIES[0], [(700, [40, 5, 60, 7]), (300, [3, 4])])
    again(g.c, wait_limit_ms=5, debug_stall_item=2)
    g.call()
    torch.cuda.synchronize()
    assert g.c.flags() == vt.FLAG_TIMEOUT
    assert not g.workspace[:16].cpu().numpy().any()
    again(g.c)
    g.call().check()
    g.close()
