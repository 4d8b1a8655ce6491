"""Calls for a batch that has no requests at the moment, or none with queries, drafts or tokens: nothing is read or written but the
number of victims, and a batch behind it is right."""
import numpy as np
import pytest

import test_gpu_shared as shared
import test_gpu_weights as weights
from attention_sim import to64
from paper_2608_13263_b200 import binding as vt

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, params=["checked", "production"])
def library(request):
    prev = vt.use_library(request.param)
    yield
    vt.use_library(prev)


@pytest.mark.parametrize("geometry", [weights.GEOMETRIES[0], weights.GEOMETRIES[4]], ids=["bf16", "fp4"])
def test_scores(geometry):
    import torch
    sc = weights.problem(np.random.default_rng(1), geometry, [300, 90], [list(range(200, 300)), [89]])
    for field, value in (("num_requests", 0), ("q_offsets", 0)):
        kept = getattr(sc.st, field).clone()
        getattr(sc.st, field).fill_(value)
        sc.call()
        torch.cuda.synchronize()
        assert (to64(sc.out) == 77).all()
        getattr(sc.st, field).copy_(kept)
    weights.run_and_check(sc)


@pytest.mark.parametrize("geometry", [shared.GEOMETRIES[0], shared.GEOMETRIES[4]], ids=["bf16", "fp4"])
@pytest.mark.parametrize("hint", [1, 100])
def test_shared_prefixes(geometry, hint):
    import torch
    g = shared.Groups(np.random.default_rng(2), geometry, [(200, [3, 40, 9]), (64, [5, 6])], max_query_len=hint)
    for field, value in (("num_requests", 0), ("q_offsets", 0)):
        kept = getattr(g.st, field).clone()
        getattr(g.st, field).fill_(value)
        g.call()
        torch.cuda.synchronize()
        assert (to64(g.st.out_all) == 77).all() and (to64(g.st.lse) == 77).all()
        getattr(g.st, field).copy_(kept)
    g.c.flags()                                              # (groups of requests that are not there are clipped, with a flag)
    shared.run_and_check(g)


def test_victims_and_drafts():
    import torch
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.zeros(64, dtype=torch.uint8, device="cuda")
    ctx = vt.vtoken_create(1, 1, 1, 1, 16, pool, pool, 8, 64, 1, 1, elem_bytes=1)
    none, offsets, lens = torch.zeros(1, **i32), torch.zeros(9, **i32), torch.zeros(8, **i32)
    listed, count = torch.full((2, 16), -5, **i32), torch.full((1,), 9, **i32)
    scores = torch.zeros(64, device="cuda")
    for requests in (0, 8):                                  # no requests; requests without tokens
        none.fill_(requests)
        for hint in (1, 100000):
            count.fill_(9)
            vt.vtoken_select_victims(ctx, num_requests=none, tt_offsets=offsets, cache_len=lens, scores=scores, budget=lens, victim_req=listed[0],
                                     victim_tok=listed[1], max_victims=16, num_victims=count, max_cache_len=hint)
            torch.cuda.synchronize()
            assert int(count) == 0 and (listed == -5).all()
    none.fill_(0)
    count.fill_(9)
    accepted, tokens = torch.full((8,), -5, **i32), torch.full((8,), -5, **i32)
    probs = torch.full((16, 100), 0.01, device="cuda")
    vt.vtoken_verify_drafts(ctx, num_requests=none, draft_offsets=offsets, max_drafts=8, draft_tokens=torch.zeros(8, **i32), prob_type=vt.PROB_F32,
                            vocab=100, target_probs=probs, draft_probs=probs, accept_random=scores[:8], sample_random=scores[:8], first_id=lens,
                            accepted=accepted, next_tokens=tokens, victim_req=listed[0], victim_tok=listed[1], max_victims=16, num_victims=count)
    torch.cuda.synchronize()
    assert int(count) == 0 and (listed == -5).all() and (accepted == -5).all() and (tokens == -5).all()
    assert vt.vtoken_read_counts(ctx)["error_flags"] == 0
    vt.vtoken_destroy(ctx)
