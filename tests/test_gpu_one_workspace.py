"""One workspace for every call of a serving loop: scores of prompts and chunks, attention, attention behind shared prefixes by
turns, each against its 64-bit reference.  A workspace is zeroed once, and each call leaves it ready for the next, whichever that is."""
import numpy as np
import pytest

import test_gpu_shared as shared
import test_gpu_weights as weights
from attention_sim import Cache, spread
from paper_2608_13263_b200 import binding as vt
from test_gpu_evict_step import load_example

pytestmark = pytest.mark.gpu

GEOMETRIES = [weights.GEOMETRIES[0], weights.GEOMETRIES[1], weights.GEOMETRIES[2], weights.GEOMETRIES[4], weights.GEOMETRIES[5]]
IDS = ["-".join(map(str, g)) for g in GEOMETRIES]


def room(c, rows):
    """A workspace of zeros that is large enough for every call, and its bytes."""
    import torch
    n = max(f(c.ctx, c.heads, rows) for f in (vt.vtoken_attention_workspace_bytes, vt.vtoken_token_weights_workspace_bytes,
                                              vt.vtoken_attention_shared_workspace_bytes))
    return torch.zeros(n, dtype=torch.uint8, device=c.dev), n


def attend(st, workspace, n):
    st.workspace, st.workspace_bytes = workspace, n
    st.out_all.fill_(77.0)
    st.lse.fill_(77.0)
    st.call()
    st.check()


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
def test_scores_of_a_prompt_between_decode_steps(geometry):
    """Few requests with long caches, whose rows are split over many CTAs: what their parts count must still be zero when scores of many
    query rows have been there."""
    rng = np.random.default_rng(1)
    act, kv, hq, hkv, d = geometry
    lens = [3000, 40, 2500]
    ids, slots, total = spread(rng, lens)
    c = Cache(rng, kv, act, hq, hkv, d, total, np.concatenate(slots), max_tokens=sum(lens) + 64)
    prompt = weights.RoomyStep(rng, c, ids, slots, [list(range(2900, 3000)), list(range(40)), []], lens=lens)
    decode = weights.RoomyStep(rng, c, ids, slots, [[2999], [39], [2498, 2499]], lens=lens)
    scored = weights.Scored(rng, prompt)
    workspace, n = room(c, prompt.n)
    for _ in range(2):
        attend(decode, workspace, n)
        scored.call(workspace=workspace, workspace_bytes=n).check()
        attend(decode, workspace, n)
        attend(prompt, workspace, n)
    assert c.flags() == 0
    c.close()


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
def test_scores_of_a_prompt_between_steps_behind_a_prefix(geometry):
    rng = np.random.default_rng(2)
    g = shared.Groups(rng, geometry, [(300, [2500, 40, 1900])])
    c = g.c
    lens = [len(i) for i in g.st.ids]
    prompt = weights.RoomyStep(rng, c, g.st.ids, g.st.slots, [list(range(2700, 2800)), [], list(range(2150, 2200))], lens=lens)
    alone = weights.RoomyStep(rng, c, g.st.ids, g.st.slots, [[n - 1] for n in lens], lens=lens)
    scored = weights.Scored(rng, prompt)
    workspace, n = room(c, prompt.n)
    for _ in range(2):
        g.st.out_all.fill_(77.0)
        g.call(workspace=workspace, workspace_bytes=n).check()
        scored.call(workspace=workspace, workspace_bytes=n).check()
        attend(alone, workspace, n)
        g.st.out_all.fill_(77.0)
        g.call(workspace=workspace, workspace_bytes=n).check()
    g.close()


@pytest.mark.parametrize("kv", ["bf16", "fp16", "fp4"])
def test_the_serving_loop_with_steps_of_many_rows(kv):
    """examples/evict_step.py with chunks of twelve tokens (48 query rows of a key head) between its steps: the same bits as from a loop
    whose workspace is zeroed in front of every step."""
    import torch
    kept, fresh = (load_example().Server(kv, groups=2, members=2, prompt=48, capacity=1024) for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(4)
    width = (kept.hq + 2 * kept.hkv) * kept.d
    qkv = torch.randn(2 * 48, width, generator=gen, device="cuda").to(kept.act)
    for s in (kept, fresh):
        s.prompts(qkv)
    for step in range(50):
        n = 40 if step < 20 else [1, 12, 1, 3][step % 4]
        qkv = torch.randn(kept.R * n, width, generator=gen, device="cuda").to(kept.act)
        fresh.workspace.zero_()
        got, want = kept.step(qkv, n), fresh.step(qkv, n)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), step
        assert torch.equal(kept.scores, fresh.scores), step
        for s in (kept, fresh):
            s.place += n
    for s in (kept, fresh):
        assert vt.vtoken_read_counts(s.ctx)["error_flags"] == 0
        s.close()
