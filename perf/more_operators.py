"""Cases, plain forms and work counts of the operators that decide what leaves a token-evicted paged KV cache, and
of attention over caches that begin with the same tokens.

  weights    the attention weight that every cached token received from the step's queries, summed over queries and
             heads and added to a running (decayed) score per token -- one query token to whole prompts, rows held in
             16 and in 4 bits
  select     the tokens that leave each request's cache when it is cut back to a budget: the lowest scores, except
             the first tokens, the shared ones and the newest
  shared     attention of requests whose caches begin with the same entries: a prefix is read once for its group
  verify     drafted tokens against the target's probabilities with given random numbers: accepted, drawn anew, and
             the rejected ones as a list of tokens to evict

A case is one pass through one of them (at one layer).  ``run`` computes the plain form with elementary torch
operations (``own`` false) or calls the library (``own`` true).
"""
import math

import torch

own = False

ACT = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}
# magnitudes of the 4-bit codes 0 .. 7 (bit 3 is the sign): 1 mantissa bit, 2 exponent bits
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
GROUP = 16                                    # values that share a scale (8 bits: 4 exponent, 3 mantissa)


# ---- cases ---------------------------------------------------------------------------------------
def _cache(name, op, act, kv, hq, hkv, d, requests, lo, hi, keep, q_lo=1, q_hi=1, window=0, sinks=0, block=16, members=1,
           prefix_lo=0, prefix_hi=0, decay=1.0):
    """requests of lo .. hi logical tokens behind a prefix of prefix_lo .. prefix_hi that `members` consecutive requests
    share; the share `keep` of the tokens before the step's own is still active."""
    return dict(name=name, op=op, act=act, kv=kv, hq=hq, hkv=hkv, d=d, requests=requests, lo=lo, hi=hi, keep=keep, q_lo=q_lo,
                q_hi=q_hi, window=window, sinks=sinks, block=block, members=members, prefix_lo=prefix_lo, prefix_hi=prefix_hi,
                decay=decay)


def _select(name, requests, lo, hi, keep, budget, sinks, recent, shared=0):
    """Active tokens: the share `keep` of lo .. hi; they are cut back to the share `budget` of them."""
    return dict(name=name, op="select", requests=requests, lo=lo, hi=hi, keep=keep, budget=budget, sinks=sinks, recent=recent,
                shared=shared)


def _verify(name, probs, requests, drafts_lo, drafts_hi, vocab, with_draft_probs):
    return dict(name=name, op="verify", probs=probs, requests=requests, drafts_lo=drafts_lo, drafts_hi=drafts_hi, vocab=vocab,
                with_draft_probs=with_draft_probs)


def listed():
    return [
        # one new token of one short request of the small geometry: pure latency
        _cache("weights_one", "weights", "bf16", "bf16", 4, 2, 64, 1, 300, 300, 0.5),
        # every request of a full batch scores its cache after a decode step
        _cache("weights_steady", "weights", "bf16", "bf16", 32, 8, 128, 512, 256, 8192, 0.35, decay=0.98),
        # the same over rows held in 4 bits, up to four query tokens (a drafted step)
        _cache("weights_4bit", "weights", "bf16", "fp4", 32, 8, 128, 256, 512, 8192, 0.5, q_lo=1, q_hi=4),
        # the queries of a whole prompt score its tokens: what a first eviction goes by
        _cache("weights_prompt", "weights", "bf16", "bf16", 32, 8, 128, 1, 8192, 8192, 1.0, q_lo=8192, q_hi=8192, decay=0.0),
        # the last queries of ragged chunks of 16 prompts, behind an evicted cache and through a window
        _cache("weights_chunks", "weights", "fp16", "fp16", 28, 4, 128, 16, 1500, 4100, 0.7, q_lo=33, q_hi=130, window=1000, sinks=4),
        # a full batch cut back to half: first and newest tokens stay
        _select("select_steady", 512, 256, 8192, 0.7, 0.5, 4, 64),
        # few very long contexts cut back to a fifth, a shared beginning stays
        _select("select_long", 6, 50000, 131072, 1.0, 0.2, 4, 256, shared=777),
        # 64 requests behind one system prompt
        _cache("shared_step", "shared", "bf16", "bf16", 32, 8, 128, 64, 200, 1000, 1.0, members=64, prefix_lo=8192, prefix_hi=8192),
        # 32 prompts, each continued by up to eight requests with drafted tokens, after an eviction and through a window
        _cache("shared_groups", "shared", "fp16", "fp16", 28, 4, 128, 250, 30, 700, 0.6, q_lo=1, q_hi=3, window=3000, sinks=4,
               block=32, members=8, prefix_lo=500, prefix_hi=4096),
        # four prefixes, rows held in 4 bits
        _cache("shared_4bit", "shared", "bf16", "fp4", 32, 8, 128, 128, 100, 2000, 0.8, members=32, prefix_lo=2000, prefix_hi=6000),
        # one request's four drafts, a small vocabulary: latency
        _verify("verify_one", "f32", 1, 4, 4, 32000, True),
        # a batch with none to eight drafts each over a large vocabulary
        _verify("verify_batch", "f32", 200, 0, 8, 128256, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("weights", "weights_rows", "shared", "shared", "select", "verify"))
    act = rng.choice(("bf16", "fp16"))
    kv = rng.choice((act, act, "fp4"))
    hkv = rng.choice((1, 2, 4, 8))
    hq = hkv * rng.choice((1, 2, 4, 5, 7, 8))
    d = rng.choice((64, 128, 128))
    block = rng.choice((16, 32))
    keep = rng.choice((1.0, rng.uniform(0.1, 0.9)))
    window, sinks = rng.choice(((0, 0), (0, 0), (_log(rng, 32, 4096), rng.choice((0, 4, 17)))))
    if kind == "weights":
        requests = _log(rng, 1, 512)
        hi = _log(rng, 40, max(80, min(32768, 1500000 // requests)))
        case = _cache("", "weights", act, kv, hq, hkv, d, requests, max(1, hi // rng.choice((1, 3, 8))), hi, keep, 1,
                      rng.choice((1, 1, 1, 3)), window, sinks, block, decay=rng.choice((0.0, 0.9, 1.0)))
    elif kind == "weights_rows":
        q_hi = _log(rng, 20, 4096)
        hi = q_hi + rng.choice((0, _log(rng, 1, 4096)))
        requests = _log(rng, 1, max(2, min(32, (1 << 30) // (hq * q_hi * hi))))
        case = _cache("", "weights", act, kv, hq, hkv, d, requests, max(q_hi, hi // 2), hi, keep, max(1, q_hi // rng.choice((1, 2, 9))),
                      q_hi, window, sinks, block, decay=rng.choice((0.0, 0.9, 1.0)))
    elif kind == "shared":
        members = _log(rng, 2, 64)
        requests = members * _log(rng, 1, max(1, 256 // members)) - rng.choice((0, 0, 1))
        prefix = _log(rng, 64, 8192)
        hi = _log(rng, 16, max(32, min(4096, 250000 // requests)))
        case = _cache("", "shared", act, kv, hq, hkv, d, requests, max(1, hi // rng.choice((1, 4))), hi, keep, 1, rng.choice((1, 1, 2, 4)),
                      window, sinks, block, members, max(1, prefix // rng.choice((1, 4))), prefix)
    elif kind == "select":
        requests = _log(rng, 1, 512)
        hi = _log(rng, 40, max(80, min(131072, 2000000 // requests)))
        case = _select("", requests, max(1, hi // rng.choice((1, 3, 8))), hi, keep, rng.choice((0.05, 0.2, 0.5, 0.9)),
                       rng.choice((0, 4)), rng.choice((0, 16, 256)), rng.choice((0, 0, 100)))
    else:
        drafts = rng.choice((0, 1, 3, 5, 8))
        requests, vocab = _log(rng, 1, 200), _log(rng, 1000, 128256)
        case = _verify("", rng.choice(("f32", "f32", "bf16", "fp16")), requests, rng.choice((0, drafts)), drafts, vocab, rng.random() < 0.7)
    del case["name"]
    return case


def _spread(lo, hi, count, shift=0):
    """``count`` lengths over lo .. hi in a fixed scrambled order: the same for every seed, so that the work of
    a case is its own."""
    return [lo + int((hi - lo) * ((0.6180339887498949 * (i + 1 + shift)) % 1.0) + 0.5) if count > 1 else hi for i in range(count)]


def _lengths(case):
    """Per request: group, prefix tokens, active ones of them, own tokens, active ones of them, query tokens (the
    newest of the own tokens, always active)."""
    R = case["requests"]
    n = _spread(case["lo"], case["hi"], R)
    m = [min(a, b) for a, b in zip(_spread(case["q_lo"], case["q_hi"], R), n)]
    live = [q + max(0, math.ceil(case["keep"] * (a - q))) for a, q in zip(n, m)]
    group = [r // case["members"] for r in range(R)]
    prefix = _spread(case["prefix_lo"], case["prefix_hi"], group[-1] + 1, 3)
    return [(g, prefix[g], math.ceil(case["keep"] * prefix[g]), a, b, q) for g, a, b, q in zip(group, n, live, m)]


# ---- work ----------------------------------------------------------------------------------------
def _row_bytes(case):
    if case["kv"] == "fp4":
        return case["hkv"] * (case["d"] // 2 + case["d"] // GROUP)
    return case["hkv"] * case["d"] * 2


def work(case):
    if case["op"] == "select":
        live = sum(max(1, math.ceil(case["keep"] * n)) for n in _spread(case["lo"], case["hi"], case["requests"]))
        return {"bytes": live * 8 + int((1 - case["budget"]) * live) * 8, "flops": live}
    if case["op"] == "verify":                                 # the row that is drawn from, and the drafts' beside it
        size = 4 if case["probs"] == "f32" else 2
        rows = case["requests"] * (2 if case["with_draft_probs"] and case["drafts_hi"] else 1)
        return {"bytes": rows * case["vocab"] * size, "flops": rows * case["vocab"]}
    hq, d, w, s = case["hq"], case["d"], case["window"], case["sinks"]
    pairs = rows = tokens = 0
    widest = {}                                                # per group: active prefix tokens that some member sees
    for g, prefix, prefix_live, n, live, m in _lengths(case):
        old = n - m                                            # own tokens older than the step, density f
        f = (live - m) / old if old else 0.0
        fp = prefix_live / prefix if prefix else 0.0
        own_below = lambda x: f * min(max(x, 0), old) + max(0, x - old)          # noqa: E731
        pre_below = lambda x: fp * min(max(x, 0), prefix)                        # noqa: E731

        def seen(p, below):                                    # active tokens that position p sees
            first = max(0, p + 1 - w) if w else 0
            return below(p + 1) - below(first) + below(min(s, first))
        everything = lambda x: pre_below(x) + own_below(x - prefix)              # noqa: E731
        some = min(m, 64)                                      # the step's positions, sampled
        at = [prefix + old + (2 * i + 1) * m // (2 * some) for i in range(some)]
        pairs += sum(seen(p, everything) for p in at) * m / some
        first = max(0, prefix + old + 1 - w) if w else 0
        here = lambda below: below(prefix + n) - below(first) + below(min(s, first))                     # noqa: E731
        rows += here(lambda x: own_below(x - prefix))
        widest[g] = max(widest.get(g, 0), here(pre_below))
        tokens += m
    rows += sum(widest.values())
    if case["op"] == "weights":
        return {"bytes": int(rows * (_row_bytes(case) + 16)) + tokens * (hq * (2 * d + 4) + 4), "flops": int(2 * pairs * hq * d)}
    return {"bytes": int(rows * (2 * _row_bytes(case) + 8)) + tokens * hq * (2 * d * 2 + 4) + tokens * 4,
            "flops": int(4 * pairs * hq * d)}


# ---- the 4-bit rows ------------------------------------------------------------------------------
def _codes(x):
    """Codes of values that are divided by their scale already: nearest, ties to the even code."""
    a = x.abs()
    c = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    return c | ((x < 0).to(torch.uint8) << 3)


def _quantise(x):
    """[.., heads, d] 32-bit values -> rows of bytes: per head d/2 bytes of codes (even element in the low half),
    then per head d/16 bytes of scales, padded to a multiple of 16 bytes."""
    n, h, d = x.shape
    g = x.view(n, h, d // GROUP, GROUP)
    scale = (g.abs().amax(-1) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    s = scale.float().unsqueeze(-1)
    c = _codes(torch.where(s > 0, g / s, torch.zeros_like(g))).view(n, h, d)
    codes = (c[..., 0::2] | (c[..., 1::2] << 4)).view(n, h * d // 2)
    row = torch.cat([codes, scale.view(torch.uint8).view(n, h * d // GROUP)], 1)
    return torch.nn.functional.pad(row, (0, -row.shape[1] % 16))


def _dequantise(row, h, d):
    """Rows of bytes -> [n, h, d] 32-bit values."""
    n = row.shape[0]
    codes, scale = row[:, :h * d // 2].view(n, h, d // 2), row[:, h * d // 2:h * d // 2 + h * d // GROUP]
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=row.device)
    c = torch.stack([codes & 15, codes >> 4], -1).view(n, h, d // GROUP, GROUP)
    s = scale.contiguous().view(torch.float8_e4m3fn).float().view(n, h, d // GROUP, 1)
    return (grid[c.int()] * s).view(n, h, d)


# ---- inputs --------------------------------------------------------------------------------------
class _Context:
    """The library's handle on the pools with the workspaces that a serving program keeps."""

    def __init__(self, s, case):
        from paper_2608_13263_b200 import binding as vt
        self.vt = vt
        requests = case["requests"]
        if case["op"] in ("select", "verify"):                 # neither looks at the pools
            self.pool = torch.zeros(64, dtype=torch.uint8, device="cuda")
            tokens = s.get("tokens", 1)
            self.ctx = vt.vtoken_create(1, 1, 1, 1, 16, self.pool, self.pool, requests, tokens, 1, 1, elem_bytes=1)
            return
        kinds = {"bf16": vt.KV_BF16, "fp16": vt.KV_FP16, "fp4": vt.KV_FP4}
        self.heads = vt.Heads(case["hq"], case["hkv"], case["d"], kinds[case["kv"]], kinds[case["act"]], 0, 0)
        geometry = (1, s["k_pool"].shape[-1], 1) if case["kv"] == "fp4" else (case["hkv"], case["d"], 2)
        tokens = s["tokens"]
        self.ctx = vt.vtoken_create(1, s["k_pool"].shape[0] // case["block"], case["block"], geometry[0], geometry[1],
                                    s["k_pool"], s["v_pool"], requests, tokens, tokens, 1, elem_bytes=geometry[2])
        size = vt.vtoken_token_weights_workspace_bytes if case["op"] == "weights" else vt.vtoken_attention_shared_workspace_bytes
        self.workspace_bytes = size(self.ctx, self.heads, s["q"].shape[0])
        self.workspace = torch.zeros(max(16, self.workspace_bytes), dtype=torch.uint8, device="cuda")

    def __del__(self):
        if getattr(self, "ctx", None) is not None:
            self.vt.vtoken_destroy(self.ctx)


def _values(gen, n, h, d, dtype, like="v"):
    """Projection outputs: keys and queries with a few strong channels, values without."""
    x = torch.randn(n, h, d, generator=gen, device="cuda", dtype=torch.float32)
    if like != "v":
        gain = 1.0 + 2.0 * (torch.rand(1, h, d, generator=gen, device="cuda") < 0.04).float()
        x = x * gain
    return x.to(dtype)


def _pool_rows(gen, case, n, like):
    """[n, row] pool rows, made in pieces: 16-bit values, or bytes."""
    dtype = ACT[case["act"]]
    if case["kv"] != "fp4":
        out = torch.empty(n, case["hkv"], case["d"], dtype=dtype, device="cuda")
    else:
        out = torch.empty(n, -(-_row_bytes(case) // 16) * 16, dtype=torch.uint8, device="cuda")
    for a in range(0, n, 1 << 17):
        x = _values(gen, min(n - a, 1 << 17), case["hkv"], case["d"], dtype, like)
        out[a:a + len(x)] = x if case["kv"] != "fp4" else _quantise(x.float())
    return out.view(n, -1)


def _kept(gen, n, a):
    """Which a of n tokens an eviction has left: the first four and the newest, the others by chance."""
    if a == n:
        return torch.arange(n, device="cuda")
    score = torch.rand(n, generator=gen, device="cuda")
    score[:4] += 2.0
    score[max(0, n - 64):] += 1.0
    return score.topk(a).indices.sort().values


def _prepare_cache(case, gen):
    S, dtype, each = case["block"], ACT[case["act"]], _lengths(case)
    R, groups = len(each), each[-1][0] + 1
    pre = {g: (p, a) for g, p, a, _, _, _ in each}
    need = [-(-pre[g][1] // S) for g in range(groups)] + [-(-a // S) for _, _, _, _, a, _ in each]
    blocks = sum(need) + 3
    order = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32)
    first = [0]
    for b in need:
        first.append(first[-1] + b)

    def rows(i, a):                                            # the slots of the a tokens of piece i, packed
        at = torch.arange(a, device="cuda")
        return order[first[i] + at // S] * S + (at % S).to(torch.int32)
    prefix = [(rows(g, pre[g][1]), _kept(gen, *pre[g]).to(torch.int32)) for g in range(groups)]
    off, live, q_off = [0], [], [0]
    for g, p, pa, n, a, m in each:
        off.append(off[-1] + p + n)
        live.append(pa + a)
        q_off.append(q_off[-1] + m)
    slots = torch.full((off[-1],), -1, dtype=torch.int32, device="cuda")
    ids = torch.full((off[-1],), -1, dtype=torch.int32, device="cuda")
    for r, (g, p, pa, n, a, m) in enumerate(each):
        o = off[r]
        slots[o:o + pa], ids[o:o + pa] = prefix[g]
        mine = torch.cat([_kept(gen, n - m, a - m), torch.arange(n - m, n, device="cuda")])
        slots[o + pa:o + pa + a] = rows(groups + r, a)
        ids[o + pa:o + pa + a] = p + mine.to(torch.int32)
    dev = dict(dtype=torch.int32, device="cuda")
    total = q_off[-1]
    back = torch.tensor([p + n - b for (_, p, _, n, _, _), b in zip(each, q_off[1:])], **dev)
    pos = torch.arange(total, **dev) + torch.repeat_interleave(back, torch.tensor([e[5] for e in each], device="cuda"))
    edges = sorted({min(R, g * case["members"]) for g in range(groups + 1)})
    s = dict(case=case, q=_values(gen, total, case["hq"], case["d"], dtype, "q"), k_pool=_pool_rows(gen, case, blocks * S, "k"),
             v_pool=_pool_rows(gen, case, blocks * S, "v") if case["op"] == "shared" else None, tokens=off[-1],
             num_requests=torch.tensor([R], **dev), tt_offsets=torch.tensor(off, **dev), cache_slots=slots, cache_ids=ids,
             cache_len=torch.tensor(live, **dev), q_offsets=torch.tensor(q_off, **dev), positions=pos,
             max_query_len=max(e[5] for e in each), max_live=max(live), num_groups=torch.tensor([len(edges) - 1], **dev),
             group_offsets=torch.tensor(edges, **dev), shared_len=torch.tensor([e[2] for e in each], **dev),
             lse=torch.empty(total, case["hq"], dtype=torch.float32, device="cuda"))
    if s["v_pool"] is None:                                    # (a cache has values too; nothing here reads them)
        s["v_pool"] = s["k_pool"]
    if case["op"] == "weights":
        s["lse"] = _rows(s, _scores(s).logsumexp(-1))          # attention has left them
        s["before"] = torch.rand(off[-1], generator=gen, device="cuda")
        s["scores"] = torch.zeros(off[-1], device="cuda")
    else:
        s["out"] = torch.empty(total, case["hq"], case["d"], dtype=dtype, device="cuda")
    return s


def _prepare_select(case, gen):
    R = case["requests"]
    n = _spread(case["lo"], case["hi"], R)
    live = [max(1, math.ceil(case["keep"] * x)) for x in n]
    off = [0]
    for x in n:
        off.append(off[-1] + x)
    ids = torch.full((off[-1],), -1, dtype=torch.int32, device="cuda")
    for r in range(R):
        ids[off[r]:off[r] + live[r]] = _kept(gen, n[r], live[r]).to(torch.int32)
    # sums of softmax weights: over five decades, with tokens that nothing has looked at and equal values among them
    scores = torch.exp(2.5 * torch.randn(off[-1], generator=gen, device="cuda") - 4.0)
    scores = torch.where(torch.rand(off[-1], generator=gen, device="cuda") < 0.05, torch.zeros_like(scores), scores)
    coarse = (scores * 64).round() / 64
    scores = torch.where(torch.rand(off[-1], generator=gen, device="cuda") < 0.2, coarse, scores)
    dev = dict(dtype=torch.int32, device="cuda")
    most = sum(live)
    return dict(case=case, num_requests=torch.tensor([R], **dev), tt_offsets=torch.tensor(off, **dev), tokens=off[-1], cache_ids=ids,
                cache_len=torch.tensor(live, **dev), scores=scores, budget=torch.tensor([int(case["budget"] * x) for x in live], **dev),
                shared_len=torch.tensor([min(x, case["shared"]) for x in live], **dev), max_live=max(live),
                victim_req=torch.full((most,), -1, **dev), victim_tok=torch.full((most,), -1, **dev), num_victims=torch.zeros(1, **dev))


def _prepare_verify(case, gen):
    R, V, dtype = case["requests"], case["vocab"], ACT[case["probs"]]
    drafts = _spread(case["drafts_lo"], case["drafts_hi"], R, 5)
    off = [0]
    for k in drafts:
        off.append(off[-1] + k)
    D = off[-1]
    dev = dict(dtype=torch.int32, device="cuda")
    at = torch.repeat_interleave(torch.arange(R, device="cuda"), torch.tensor(drafts, device="cuda"), output_size=D)
    row = torch.arange(D, device="cuda") + at                  # a request has a row more than drafts
    target = torch.empty(D + R, V, dtype=dtype, device="cuda")
    draft = torch.empty(D, V, dtype=dtype, device="cuda")
    tokens = torch.empty(D, **dev)
    for a in range(0, D + R, 256):
        target[a:a + 256] = torch.softmax(3.0 * torch.randn(min(256, D + R - a), V, generator=gen, device="cuda"), -1).to(dtype)
    for a in range(0, D, 256):                                 # a smaller model's view of the same rows
        p = target[row[a:a + 256]].float()
        noise = torch.randn(p.shape, generator=gen, device="cuda")
        q = torch.softmax(torch.log(p.clamp(min=1e-30)) * 0.9 + 0.7 * noise, -1)
        draft[a:a + 256] = q.to(dtype)
        luck = torch.rand(p.shape, generator=gen, device="cuda").clamp(min=1e-30)
        tokens[a:a + 256] = (draft[a:a + 256].float() / -torch.log(luck)).argmax(-1).to(torch.int32)
    return dict(case=case, num_requests=torch.tensor([R], **dev), draft_offsets=torch.tensor(off, **dev), draft_tokens=tokens,
                target=target, draft=draft if case["with_draft_probs"] else None,
                accept=torch.rand(D, generator=gen, device="cuda"), sample=torch.rand(R, generator=gen, device="cuda"),
                first_id=torch.randint(0, 8192, (R,), generator=gen, device="cuda").to(torch.int32), drafts=D,
                accepted=torch.empty(R, **dev), next_tokens=torch.empty(R, **dev), out_tokens=torch.empty(D + R, **dev),
                victim_req=torch.full((max(1, D),), -1, **dev), victim_tok=torch.full((max(1, D),), -1, **dev),
                num_victims=torch.zeros(1, **dev))


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return {"select": _prepare_select, "verify": _prepare_verify}.get(case["op"], _prepare_cache)(case, gen)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:                                   # the handle and the workspace a serving program keeps
        s["lib"] = _Context(s, case)
    return s


# ---- one pass ------------------------------------------------------------------------------------
def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


def _own_weights(s):
    c, lib = s["case"], s["lib"]
    lib.vt.vtoken_token_weights(lib.ctx, heads=lib.heads, layer=0, num_requests=s["num_requests"], q_offsets=s["q_offsets"],
                                positions=s["positions"], q=s["q"], max_query_tokens=s["q"].shape[0],
                                max_query_len=s["max_query_len"], tt_offsets=s["tt_offsets"], cache_slots=s["cache_slots"],
                                cache_ids=s["cache_ids"], cache_len=s["cache_len"], lse=s["lse"], sm_scale=c["d"] ** -0.5,
                                window=c["window"], sinks=c["sinks"], decay=c["decay"], prev=s["before"], scores=s["scores"],
                                workspace=lib.workspace, workspace_bytes=lib.workspace_bytes)
    return s["scores"]


def _own_shared(s):
    c, lib = s["case"], s["lib"]
    lib.vt.vtoken_attention_shared(lib.ctx, heads=lib.heads, layer=0, num_requests=s["num_requests"], q_offsets=s["q_offsets"],
                                   positions=s["positions"], q=s["q"], max_query_tokens=s["q"].shape[0],
                                   max_query_len=s["max_query_len"], tt_offsets=s["tt_offsets"], cache_slots=s["cache_slots"],
                                   cache_ids=s["cache_ids"], cache_len=s["cache_len"], out=s["out"], lse=s["lse"],
                                   sm_scale=c["d"] ** -0.5, window=c["window"], sinks=c["sinks"], num_groups=s["num_groups"],
                                   group_offsets=s["group_offsets"], shared_len=s["shared_len"], workspace=lib.workspace,
                                   workspace_bytes=lib.workspace_bytes)
    return s["out"], s["lse"]


def _own_select(s):
    c, lib = s["case"], s["lib"]
    lib.vt.vtoken_select_victims(lib.ctx, num_requests=s["num_requests"], tt_offsets=s["tt_offsets"], cache_ids=s["cache_ids"],
                                 cache_len=s["cache_len"], scores=s["scores"], budget=s["budget"], shared_len=s["shared_len"],
                                 sinks=c["sinks"], recent=c["recent"], max_cache_len=s["max_live"],
                                 victim_req=s["victim_req"], victim_tok=s["victim_tok"], max_victims=s["victim_req"].shape[0], num_victims=s["num_victims"])
    return s["victim_req"], s["victim_tok"], s["num_victims"]


def _own_verify(s):
    c, lib = s["case"], s["lib"]
    kinds = {"bf16": lib.vt.PROB_BF16, "fp16": lib.vt.PROB_FP16, "f32": lib.vt.PROB_F32}
    lib.vt.vtoken_verify_drafts(lib.ctx, num_requests=s["num_requests"], draft_offsets=s["draft_offsets"], max_drafts=s["drafts"],
                                draft_tokens=s["draft_tokens"], prob_type=kinds[c["probs"]], vocab=c["vocab"],
                                target_probs=s["target"], draft_probs=s["draft"], accept_random=s["accept"],
                                sample_random=s["sample"], first_id=s["first_id"], accepted=s["accepted"],
                                next_tokens=s["next_tokens"], out_tokens=s["out_tokens"], victim_req=s["victim_req"],
                                victim_tok=s["victim_tok"], max_victims=s["victim_req"].shape[0], num_victims=s["num_victims"])
    return s["accepted"], s["next_tokens"], s["out_tokens"], s["victim_req"], s["victim_tok"], s["num_victims"]


# ---- plain forms ---------------------------------------------------------------------------------
def _rows_of(s, pool, slots):
    c = s["case"]
    rows = s[pool][slots]
    return _dequantise(rows, c["hkv"], c["d"]) if c["kv"] == "fp4" else rows.float().view(-1, c["hkv"], c["d"])


def _padded(s):
    """Cache entries of every request, padded to the longest: entry, whether it is there, id, slot [R, L]; rows of its
    queries, whether they are there, position [R, M]."""
    L, M = s["max_live"], s["max_query_len"]
    at = torch.arange(L, device="cuda")
    entry = (s["tt_offsets"][:-1].long().unsqueeze(1) + at).clamp(max=s["cache_ids"].shape[0] - 1)
    there = at < s["cache_len"].unsqueeze(1)
    ids = torch.where(there, s["cache_ids"][entry], torch.full_like(entry, 1 << 30, dtype=torch.int32))
    slots = torch.where(there, s["cache_slots"][entry], 0).long()
    row = torch.arange(M, device="cuda")
    have = row < (s["q_offsets"][1:] - s["q_offsets"][:-1]).unsqueeze(1)
    query = (s["q_offsets"][:-1].long().unsqueeze(1) + row).clamp(max=s["q"].shape[0] - 1)
    return there, ids, slots, query, have, s["positions"][query]


def _scores(s):
    """Scaled scores of every query over its request's cache, minus infinity where it does not look [R, hq, M, L]."""
    c = s["case"]
    R, L, M, hq, hkv, d = c["requests"], s["max_live"], s["max_query_len"], c["hq"], c["hkv"], c["d"]
    _, ids, slots, query, have, pos = _padded(s)
    k = _rows_of(s, "k_pool", slots.flatten()).view(R, L, hkv, d).transpose(1, 2)
    q = s["q"][query.flatten()].float().view(R, M, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(R, hkv, -1, d)
    score = (q @ k.transpose(-1, -2)).view(R, hq, M, L) * d ** -0.5
    sees = ids.unsqueeze(1) <= pos.unsqueeze(2)
    if c["window"]:
        sees &= (ids.unsqueeze(1) > pos.unsqueeze(2) - c["window"]) | (ids.unsqueeze(1) < c["sinks"])
    return score.masked_fill_(~(sees & have.unsqueeze(2)).unsqueeze(1), -math.inf)


def _rows(s, x):
    """[R, hq, M, ...] of padded requests -> [query rows, hq, ...]."""
    have = _padded(s)[4].flatten()
    return x.transpose(1, 2).flatten(0, 1)[have].contiguous()


def _plain_weights(s):
    c = s["case"]
    R, M, hq = c["requests"], s["max_query_len"], c["hq"]
    there, ids, _, query, have, _ = _padded(s)
    score = _scores(s)
    lse = s["lse"][query.flatten()].view(R, M, hq).permute(0, 2, 1).unsqueeze(-1)
    weight = torch.where(score == -math.inf, score, score.sub_(lse.clamp(min=-3.0e38))).exp_().sum((1, 2))        # [R, L]
    at = (s["tt_offsets"][:-1].unsqueeze(1) + ids)[there].long()
    s["scores"][at] = (c["decay"] * s["before"][at] if c["decay"] else 0.0) + weight[there]
    return s["scores"]


def _plain_shared(s):
    """Every request by itself: the sharing saves reading, it changes no value."""
    c = s["case"]
    R, L, M, hq, hkv, d = c["requests"], s["max_live"], s["max_query_len"], c["hq"], c["hkv"], c["d"]
    slots = _padded(s)[2]
    score = _scores(s)
    top = score.amax(-1, keepdim=True).clamp(min=-3.0e38)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = _rows_of(s, "v_pool", slots.flatten()).view(R, L, hkv, d).transpose(1, 2)
    out = (p.view(R, hkv, -1, L) @ v).view(R, hq, M, d) / total.clamp(min=1e-38)
    lse = (total.log() + top).squeeze(-1)
    return _rows(s, out).to(ACT[c["act"]]), _rows(s, lse)


def _victims(s, req, tok):
    for name, x in (("victim_req", req), ("victim_tok", tok)):
        s[name].fill_(-1)
        s[name][:x.shape[0]] = x.to(torch.int32)
    s["num_victims"][0] = req.shape[0]
    return s["victim_req"], s["victim_tok"], s["num_victims"]


def _plain_select(s):
    c = s["case"]
    at = torch.arange(s["max_live"], device="cuda")
    entry = (s["tt_offsets"][:-1].long().unsqueeze(1) + at).clamp(max=s["cache_ids"].shape[0] - 1)
    n = s["cache_len"].unsqueeze(1)
    ids = s["cache_ids"][entry]
    value = s["scores"][(s["tt_offsets"][:-1].unsqueeze(1) + ids.clamp(min=0)).long()]
    free = (at < n - c["recent"]) & (at >= s["shared_len"].unsqueeze(1)) & (ids >= c["sinks"]) & (at < n)
    value = torch.where(free, value, math.inf)
    # lowest first, of equal ones the last first
    order = value.flip(1).sort(dim=1, stable=True).indices
    rank = torch.empty_like(order).scatter_(1, order, at.expand_as(order).contiguous()).flip(1)
    out = free & (rank < n - s["budget"].unsqueeze(1))
    req, where = out.nonzero(as_tuple=True)
    return _victims(s, req, ids[req, where])


def _plain_verify(s):
    c = s["case"]
    R, V, D = c["requests"], c["vocab"], s["drafts"]
    off = s["draft_offsets"].long()
    drafts = off[1:] - off[:-1]
    of = torch.repeat_interleave(torch.arange(R, device="cuda"), drafts, output_size=D)
    which = torch.arange(D, device="cuda") - off[of]           # its place among the request's drafts
    x = s["draft_tokens"].long()
    p = s["target"][torch.arange(D, device="cuda") + of, x].double()
    q = s["draft"][torch.arange(D, device="cuda"), x].double() if s["draft"] is not None else torch.ones_like(p)
    refused = s["accept"].double() * q >= p
    accepted = drafts.clone().scatter_reduce_(0, of, torch.where(refused, which, drafts[of]), "amin")
    rest = s["target"][off[:-1] + torch.arange(R, device="cuda") + accepted].double()
    some = accepted < drafts                                   # a refused draft: what the target has more than the draft's source
    at = (off[:-1] + accepted).clamp(max=max(0, D - 1))
    if D:
        if s["draft"] is not None:
            less = (rest - s["draft"][at].double()).clamp(min=0.0)
        else:
            less = rest.scatter(1, x[at].unsqueeze(1), 0.0)
        less = torch.where(less.sum(1, keepdim=True) > 0, less, rest)
        rest = torch.where(some.unsqueeze(1), less, rest)
    upto = rest.cumsum(1)
    token = (upto > s["sample"].double().unsqueeze(1) * upto[:, -1:]).int().argmax(1)
    out = torch.full((D + R,), -1, dtype=torch.int32, device="cuda")
    fine = which < accepted[of]
    out[(torch.arange(D, device="cuda") + of)[fine]] = s["draft_tokens"][fine]
    out[off[:-1] + torch.arange(R, device="cuda") + accepted] = token.to(torch.int32)
    gone = ~fine
    return (accepted.to(torch.int32), token.to(torch.int32), out) + _victims(s, of[gone], s["first_id"][of[gone]] + which[gone])


_OWN = {"weights": _own_weights, "shared": _own_shared, "select": _own_select, "verify": _own_verify}
_PLAIN = {"weights": _plain_weights, "shared": _plain_shared, "select": _plain_select, "verify": _plain_verify}


# ---- the definitions in 64 bits ------------------------------------------------------------------
def _rows64(case, pool, slots):
    rows, h, d = pool[slots.long()], case["hkv"], case["d"]
    if case["kv"] != "fp4":
        return rows.double().view(-1, h, d)
    value = torch.tensor([(-1.0 if b & 8 else 1.0) * GRID[b & 7] for b in range(16)], dtype=torch.float64, device="cuda")
    byte = torch.arange(256, device="cuda")
    e, f = (byte >> 3) & 15, (byte & 7).double()
    scale = torch.where(e > 0, (1 + f / 8) * torch.exp2(e.double() - 7), f * 2.0 ** -9)
    b = rows[:, :h * d // 2].long().view(-1, h, d // 2)
    out = torch.empty(len(rows), h, d, dtype=torch.float64, device="cuda")
    out[..., 0::2], out[..., 1::2] = value[b % 16], value[b // 16]
    return out * scale[rows[:, h * d // 2:h * d // 2 + h * d // GROUP].long()].view(-1, h, d // GROUP).repeat_interleave(GROUP, -1)


def _each_block(case, s):
    """Per request, up to 1024 of its queries and key head: entries, query rows, heads, scores [m, g, l] in 64 bits with
    minus infinity where a query does not look."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    off, q_off, live = s["tt_offsets"].tolist(), s["q_offsets"].tolist(), s["cache_len"].tolist()
    for r in range(case["requests"]):
        here = slice(off[r], off[r] + live[r])
        k = _rows64(case, s["k_pool"], s["cache_slots"][here])
        ids = s["cache_ids"][here]
        for a in range(q_off[r], q_off[r + 1], 1024):
            b = min(a + 1024, q_off[r + 1])
            pos = s["positions"][a:b].unsqueeze(1)
            hidden = ids > pos
            if case["window"]:
                hidden |= (ids <= pos - case["window"]) & (ids >= case["sinks"])
            for h in range(hkv):
                g = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
                x = torch.einsum("mgd,ld->mgl", s["q"][a:b, g].double(), k[:, h]) / math.sqrt(d)
                yield r, here, slice(a, b), g, h, x.masked_fill_(hidden.unsqueeze(1), -math.inf)


def exact(case, seed):
    if case["op"] in ("select", "verify"):                     # whole numbers, by the rules of the plain form
        return None
    s = _inputs(case, seed)
    if case["op"] == "weights":
        total = torch.zeros(s["tokens"], dtype=torch.float64, device="cuda")
        for r, here, rows, g, _, x in _each_block(case, s):
            at = int(s["tt_offsets"][r]) + s["cache_ids"][here].long()
            total[at] += torch.exp(x - s["lse"][rows, g].double().unsqueeze(-1)).nan_to_num(0.0).sum((0, 1))
        for r in range(case["requests"]):
            o = int(s["tt_offsets"][r])
            at = o + s["cache_ids"][o:o + int(s["cache_len"][r])].long()
            total[at] += case["decay"] * s["before"][at].double()
        return total
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    for r, here, rows, g, h, x in _each_block(case, s):
        v = _rows64(case, s["v_pool"], s["cache_slots"][here])[:, h]
        z = torch.logsumexp(x, -1)
        out[rows, g] = torch.einsum("mgl,ld->mgd", torch.exp(x - z.unsqueeze(-1)).nan_to_num(0.0), v)
        lse[rows, g] = z
    return out, lse
