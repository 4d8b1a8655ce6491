"""Tables with more requests and groups than a kernel has threads for, and prompts whose work is cut coarser because there is no room
for more sums: scores and attention behind shared prefixes, on the checked build (every index into a table or scratch
range-checked; none may be out of range) and on the production one."""
import numpy as np
import pytest

import test_gpu_shared as shared
import test_gpu_weights as weights
from attention_sim import Cache, spread, to64
from paper_2608_13263_b200 import binding as vt

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, params=["checked", "production"])
def library(request):
    prev = vt.use_library(request.param)
    yield
    vt.use_library(prev)


NARROW = [("bf16", "bf16", 4, 2, 64), ("bf16", "fp4", 4, 2, 64)]


@pytest.mark.parametrize("geometry", NARROW, ids=["bf16", "fp4"])
@pytest.mark.parametrize("requests", [256, 257, 1000])
def test_scores_of_many_single_tokens(geometry, requests):
    rng = np.random.default_rng(requests)
    lens = rng.integers(0, 30, requests).tolist()
    lens[3], lens[requests - 1] = 400, 70
    weights.run_and_check(weights.problem(rng, geometry, lens, keep=0.7))


@pytest.mark.parametrize("geometry", [("fp16", "fp16", 16, 1, 64), ("bf16", "fp4", 16, 1, 64)], ids=["fp16", "fp4"])
@pytest.mark.parametrize("requests", [300, 769, 1600])
def test_scores_of_many_short_prompts(geometry, requests):
    """Two tokens are 32 rows and belong to the kernel for few, three are 48 and belong to the other one."""
    rng = np.random.default_rng(requests)
    lens = rng.integers(0, 24, requests).tolist()
    lens[5], lens[requests - 2] = 300, 515
    many = rng.integers(0, 4, requests).tolist()
    positions = [list(range(max(0, n - m), n)) for n, m in zip(lens, many)]
    weights.run_and_check(weights.problem(rng, geometry, lens, positions, keep=0.8))


def row_tiles_of_an_item(sms, requests, max_tokens, cache, queries, hq, hkv):
    """How the scores of one prompt are cut: about eight items a CTA, of 4 to 32 row tiles of whole query tokens, twice as many for as
    long as there is no room for the items' sums."""
    tokens = 128 // (hq // hkv)
    pairs, tiles = -(-cache // 256), -(-queries // tokens)
    room = (-(-max_tokens // 256) + requests) * hkv * -(-(queries // tokens + 1) // 1024) + 16 * sms
    c = min(32, max(4, pairs * tiles * hkv // (sms * 8)))
    while pairs * -(-tiles // c) * hkv > room and c < 1024:
        c *= 2
    return c


class OnDevice(weights.Scored):
    """A Scored of one request whose 64-bit reference is taken on the device, in steps of query tokens."""

    def __init__(self, rng, step):
        import torch
        c = step.c
        self.st, self.decay, self.in_place = step, 1.0, False
        f64 = dict(dtype=torch.float64, device=c.dev)
        ids = torch.from_numpy(np.asarray(step.ids[0])).to(c.dev)
        k = torch.from_numpy(np.stack([c.k64[int(s)] for s in step.slots[0]])).to(c.dev)            # [n, hkv, d]
        q = step.q_all[:step.n, :c.hq * c.d].double().view(step.n, c.hkv, c.hq // c.hkv, c.d)
        pos = step.pos[:step.n].long()
        lse = torch.full((step.n, c.hq), -float("inf"), **f64)
        weight, err, terms = (torch.zeros(len(ids), **f64) for _ in range(3))
        for t0 in range(0, step.n, 64):
            p = pos[t0:t0 + 64, None]
            seen = ids[None] <= p
            if step.window:
                seen &= (ids[None] > p - step.window) | (ids[None] < step.sinks)
            seen = seen[:, None]                                                                    # [t, 1, n]
            for h in range(c.hkv):
                part = q[t0:t0 + 64, h]
                x = torch.einsum("tgd,nd->tgn", part, k[:, h]) * step.sm_scale
                ds = c.d * 2.0 ** -23 * torch.einsum("tgd,nd->tgn", part.abs(), k[:, h].abs()) * abs(step.sm_scale)
                y = torch.logsumexp(x.masked_fill(~seen, -float("inf")), -1).float().double()       # [t, g], as the call gets it
                lse[t0:t0 + 64, h * (c.hq // c.hkv):(h + 1) * (c.hq // c.hkv)] = y
                w = torch.exp(x - y[..., None]).masked_fill(~seen | torch.isinf(y)[..., None], 0)
                # the bounds of Scored.reference
                e = w * (ds + 2.0 ** -22 * (x.abs() + torch.where(torch.isinf(y), 0, y).abs()[..., None] + 1) * 1.5)
                weight += w.sum((0, 1))
                err += e.sum((0, 1))
                terms += seen.sum((0, 1)) * (c.hq // c.hkv)
        self.lse = lse.float().contiguous()
        self.prev64 = rng.random(c.max_tokens).astype(np.float32).astype(np.float64)
        self.prev = torch.from_numpy(self.prev64.astype(np.float32)).to(c.dev)
        self.out = torch.full((c.max_tokens,), 77.0, device=c.dev)
        n = vt.vtoken_token_weights_workspace_bytes(c.ctx, c.heads, step.n)
        self.workspace, self.workspace_bytes = torch.zeros(n, dtype=torch.uint8, device=c.dev), n
        self.found = [to64(a) for a in (weight, err, terms)]

    def reference(self):
        st, c = self.st, self.st.c
        weight, err, terms = self.found
        ref, tol = np.full(c.max_tokens, 77.0), np.zeros(c.max_tokens)
        at = np.asarray(st.ids[0], int)
        ref[at] = self.prev64[at] + weight
        tol[at] = err + (terms + 2) * 2.0 ** -24 * ref[at] + 1e-38
        return ref, tol


@pytest.mark.parametrize("geometry", [("bf16", "bf16", 16, 1, 64), ("bf16", "fp4", 16, 1, 64), ("fp16", "fp16", 14, 2, 128)], ids=["bf16", "fp4", "fp16"])
@pytest.mark.parametrize("window", [0, 5000])
def test_items_of_more_than_32_row_tiles(geometry, window):
    import torch
    rng = np.random.default_rng(3)
    act, kv, hq, hkv, d = geometry
    cache, queries = (65536, 2900) if hkv == 1 else (60000, 4600)
    ids, slots, total = spread(rng, [cache], 0.95)
    c = Cache(rng, kv, act, hq, hkv, d, total, slots[0], max_requests=1, max_tokens=cache, layers=1)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert row_tiles_of_an_item(sms, 1, cache, len(ids[0]), queries, hq, hkv) > 32
    st = weights.RoomyStep(rng, c, ids, slots, [list(range(cache - queries, cache))], window, 4 if window else 0, lens=[cache])
    weights.run_and_check(OnDevice(rng, st))


@pytest.mark.parametrize("geometry", NARROW, ids=["bf16", "fp4"])
@pytest.mark.parametrize("groups", [64, 65, 600, 1024, 1025, 1100])
def test_many_groups_of_two(geometry, groups):
    """Lengths and readers of groups in shared memory and, of more than 1024, in global memory; more requests than threads."""
    rng = np.random.default_rng(groups)
    cut = [(int(p), [int(n) for n in rng.integers(0, 5, 2)]) for p in rng.integers(0, 20, groups)]
    cut[1], cut[groups - 1] = (300, [3, 40]), (140, [1, 2])
    shared.run_and_check(shared.Groups(rng, geometry, cut, keep=0.9, outside=2))


def test_a_group_of_more_requests_than_threads():
    rng = np.random.default_rng(5)
    shared.run_and_check(shared.Groups(rng, NARROW[0], [(20, [4, 5]), (530, rng.integers(0, 6, 1500).tolist()), (40, [1, 1, 2])]))
