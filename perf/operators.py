"""Cases, plain forms and work counts of the attention operators next to the repack.

Three operators of a decode or prompt step over a token-evicted paged KV cache:

  write      queries and keys normalised per head and rotated by position, keys and values written to
             the slots of their tokens -- 16-bit rows, or 4-bit rows with one 8-bit scale per 16 values
  attention  queries against the active tokens of a slot cache (``cache_slots`` / ``cache_ids``), causal by
             logical id, optionally a sliding window with the first tokens kept visible; one to many
             query tokens per request, the cache held in 16 bits
  attention  the same over a cache held in 4 bits

A case is one pass through one of them at one layer.  ``run`` computes the plain form with elementary
torch operations in 32 bits (``own`` false) or calls the library (``own`` true).
"""
import math

import torch

own = False

ACT = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6
# magnitudes of the 4-bit codes 0 .. 7 (bit 3 is the sign): 1 mantissa bit, 2 exponent bits
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
GROUP = 16                                    # values that share a scale (8 bits: 4 exponent, 3 mantissa)


# ---- cases ---------------------------------------------------------------------------------------
def _write(name, act, kv, hq, hkv, d, tokens, packed, interleaved=False, rot=0):
    """rot: rotated dimensions of a head (0: all); packed: q, k and v are slices of one projection output."""
    return dict(name=name, op="write", act=act, kv=kv, hq=hq, hkv=hkv, d=d, tokens=tokens, packed=packed,
                interleaved=interleaved, rot=rot or d, block=16)


def _attn(name, act, kv, hq, hkv, d, requests, lo, hi, keep, q_lo=1, q_hi=1, window=0, sinks=0, block=16,
          packed_blocks=True):
    """requests of lo .. hi logical tokens of which the share ``keep`` is still active (the q_lo .. q_hi tokens
    of the step always are); packed_blocks: the table as a repack leaves it, else with the holes of the eviction."""
    return dict(name=name, op="attention", act=act, kv=kv, hq=hq, hkv=hkv, d=d, requests=requests, lo=lo, hi=hi,
                keep=keep, q_lo=q_lo, q_hi=q_hi, window=window, sinks=sinks, block=block, packed_blocks=packed_blocks)


def listed():
    return [
        # one new token of one request: pure latency
        _write("write_one", "bf16", "bf16", 32, 8, 128, 1, True),
        # the decode step of 512 requests, from the packed projection output
        _write("write_step", "bf16", "bf16", 32, 8, 128, 512, True),
        # a long prompt in half precision, 28 query heads over 4, half of each head rotated, pairs interleaved
        _write("write_prompt", "fp16", "fp16", 28, 4, 128, 16384, False, interleaved=True, rot=64),
        # a decode step that quantises on the way into the cache, and the rows read back
        _write("write_4bit", "bf16", "fp4", 32, 8, 128, 300, True),
        # a single short request of the small geometry: latency
        _attn("decode_one", "bf16", "bf16", 4, 2, 64, 1, 300, 300, 0.5),
        # 64 requests after a heavy-hitter eviction to a fifth, packed by a repack
        _attn("decode_evicted", "bf16", "bf16", 32, 8, 128, 64, 1024, 4096, 0.2),
        # long contexts read through a window with four first tokens kept
        _attn("decode_window", "fp16", "fp16", 28, 4, 128, 32, 16384, 32768, 1.0, window=4096, sinks=4, block=32),
        # the steady state: 512 requests whose tables still have the holes of the eviction
        _attn("decode_steady", "bf16", "bf16", 32, 8, 128, 512, 256, 8192, 0.35, packed_blocks=False),
        # one long prompt from its first token on
        _attn("prompt_long", "bf16", "bf16", 32, 8, 128, 1, 8192, 8192, 1.0, q_lo=8192, q_hi=8192),
        # chunks of prompts behind an evicted cache, windowed, odd lengths
        _attn("prompt_chunks", "fp16", "fp16", 28, 4, 128, 16, 1500, 4100, 0.7, q_lo=129, q_hi=515, window=1000, sinks=4),
        # the steady decode over the cache in 4 bits
        _attn("decode_4bit", "bf16", "fp4", 32, 8, 128, 256, 512, 8192, 0.5),
        # a chunk of each of four prompts over the cache in 4 bits
        _attn("prompt_4bit", "bf16", "fp4", 32, 8, 128, 4, 2048, 4096, 1.0, q_lo=1024, q_hi=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    act = rng.choice(("bf16", "fp16"))
    kv = rng.choice((act, act, "fp4"))
    hkv = rng.choice((1, 2, 4, 8))
    hq = hkv * rng.choice((1, 2, 4, 5, 7, 8))
    d = rng.choice((64, 128, 128))
    kind = rng.choice(("write", "decode", "decode", "prompt"))
    if kind == "write":
        tokens = _log(rng, 1, 16384) if kv != "fp4" else _log(rng, 1, 300)
        case = _write("", act, kv, hq, hkv, d, tokens, rng.random() < 0.5, rng.random() < 0.5, rng.choice((d, d, d // 2)))
    else:
        window, sinks = rng.choice(((0, 0), (0, 0), (_log(rng, 32, 4096), rng.choice((0, 4, 17)))))
        keep = rng.choice((1.0, rng.uniform(0.1, 0.9)))
        block = rng.choice((16, 32))
        if kind == "decode":
            requests = _log(rng, 1, 512)
            hi = _log(rng, 40, max(80, min(32768, 1500000 // requests)))
            case = _attn("", act, kv, hq, hkv, d, requests, max(1, hi // rng.choice((1, 3, 8))), hi, keep, 1,
                         rng.choice((1, 1, 1, 3)), window, sinks, block, rng.random() < 0.5)
        else:
            q_hi = _log(rng, 20, 4096)
            hi = q_hi + rng.choice((0, _log(rng, 1, 4096)))
            requests = _log(rng, 1, max(2, min(32, (1 << 30) // (hq * q_hi * hi))))
            q_lo = max(1, q_hi // rng.choice((1, 2, 9)))
            case = _attn("", act, kv, hq, hkv, d, requests, max(q_hi, hi // 2), hi, keep, q_lo, q_hi, window, sinks, block,
                         rng.random() < 0.5)
    del case["name"]
    return case


def _spread(lo, hi, count):
    """``count`` lengths over lo .. hi in a fixed scrambled order: the same for every seed, so that the work of
    a case is its own."""
    return [lo + int((hi - lo) * ((0.6180339887498949 * (i + 1)) % 1.0) + 0.5) if count > 1 else hi for i in range(count)]


def _lengths(case):
    """Per request: logical tokens, active tokens, query tokens."""
    n = _spread(case["lo"], case["hi"], case["requests"])
    m = [min(a, b) for a, b in zip(_spread(case["q_lo"], case["q_hi"], case["requests"]), n)]
    live = [q + max(0, math.ceil(case["keep"] * (a - q))) for a, q in zip(n, m)]
    return n, live, m


# ---- work ----------------------------------------------------------------------------------------
def _row_bytes(case):
    if case["kv"] == "fp4":
        return case["hkv"] * (case["d"] // 2 + case["d"] // GROUP)
    return case["hkv"] * case["d"] * 2


def work(case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "write":
        n = case["tokens"]
        moved = n * ((2 * hq + 2 * hkv) * d * 2 + 2 * _row_bytes(case) + case["rot"] * 4 + 8)
        if case["kv"] == "fp4":                               # the rows that are read back
            moved += n * (2 * _row_bytes(case) + 2 * hkv * d * 2)
        return {"bytes": moved, "flops": n * (hq + hkv) * d * 8}
    w, s = case["window"], case["sinks"]
    pairs = rows = tokens = 0
    for n, live, m in zip(*_lengths(case)):
        old = n - m                                            # tokens older than the step, density f
        f = (live - m) / old if old else 0.0
        below = lambda x: f * min(x, old) + max(0, x - old)    # active tokens with an id below x  # noqa: E731

        def seen(p):                                           # active tokens that position p sees
            first = max(0, p + 1 - w) if w else 0
            return below(p + 1) - below(first) + below(min(s, first))
        some = min(m, 64)                                      # the step's positions, sampled
        pairs += sum(seen(old + (2 * i + 1) * m // (2 * some)) for i in range(some)) * m / some
        first = max(0, old + 1 - w) if w else 0
        rows += below(n) - below(first) + below(min(s, first))
        tokens += m
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
    """The library's handle on the pools, as a serving program keeps it."""

    def __init__(self, s, case):
        from paper_2608_13263_b200 import binding as vt
        self.vt = vt
        kinds = {"bf16": vt.KV_BF16, "fp16": vt.KV_FP16, "fp4": vt.KV_FP4}
        self.heads = vt.Heads(case["hq"], case["hkv"], case["d"], kinds[case["kv"]], kinds[case["act"]], 0, 0)
        geometry = (1, s["k_pool"].shape[-1], 1) if case["kv"] == "fp4" else (case["hkv"], case["d"], 2)
        requests, tokens = case.get("requests", 1), s["tokens"]
        self.ctx = vt.vtoken_create(1, s["k_pool"].shape[0] // case["block"], case["block"], geometry[0], geometry[1],
                                    s["k_pool"], s["v_pool"], requests, tokens, tokens, 1, elem_bytes=geometry[2])
        if case["op"] == "attention":
            self.workspace_bytes = vt.vtoken_attention_workspace_bytes(self.ctx, self.heads, s["q"].shape[0])
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
    return out


def _prepare_write(case, gen):
    n, hq, hkv, d, dtype = case["tokens"], case["hq"], case["hkv"], case["d"], ACT[case["act"]]
    blocks = -(-n // case["block"]) + 3
    q, k, v = _values(gen, n, hq, d, dtype, "q"), _values(gen, n, hkv, d, dtype, "k"), _values(gen, n, hkv, d, dtype)
    if case["packed"]:
        all3 = torch.cat([q, k, v], 1)
        q, k, v = all3[:, :hq], all3[:, hq:hq + hkv], all3[:, hq + hkv:]
    top = max(n, 4096)
    half = case["rot"] // 2
    angle = torch.outer(torch.arange(top, device="cuda", dtype=torch.float64),
                        10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half))
    first = int(torch.randint(0, top - n + 1, (1,), generator=gen, device="cuda"))
    row = hkv * d if case["kv"] != "fp4" else -(-_row_bytes(case) // 16) * 16
    pools = [torch.zeros(blocks * case["block"], row, device="cuda", dtype=dtype if case["kv"] != "fp4" else torch.uint8)
             for _ in range(2)]
    order = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32)
    at = torch.arange(n, device="cuda", dtype=torch.int32)
    return dict(q=q, k=k, v=v, k_pool=pools[0], v_pool=pools[1], tokens=n,
                slots=order[(at // case["block"]).long()] * case["block"] + at % case["block"],
                positions=(first + at).to(torch.int32),
                q_weight=(1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dtype),
                k_weight=(1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dtype),
                cos_sin=torch.cat([angle.cos(), angle.sin()], 1).float().contiguous(),
                q_out=torch.empty(n, hq, d, dtype=dtype, device="cuda"),
                k_back=torch.empty(n, hkv, d, dtype=dtype, device="cuda"),
                v_back=torch.empty(n, hkv, d, dtype=dtype, device="cuda"))


def _prepare_attention(case, gen):
    lens, live, steps = _lengths(case)
    S, dtype = case["block"], ACT[case["act"]]
    held = live if case["packed_blocks"] else lens
    need = [-(-x // S) for x in held]
    blocks = sum(need) + 3
    order = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32)
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    slots = torch.full((off[-1],), -1, dtype=torch.int32, device="cuda")
    ids = torch.full((off[-1],), -1, dtype=torch.int32, device="cuda")
    taken = 0
    for r, (n, a, m) in enumerate(zip(lens, live, steps)):
        if a == n:
            keep = torch.arange(n, device="cuda")
        else:                                 # the newest always, the first four, the others as their score falls
            score = torch.rand(n - m, generator=gen, device="cuda")
            score[:4] += 2.0
            score[max(0, n - m - 64):] += 1.0
            kept = score.topk(a - m).indices.sort().values
            keep = torch.cat([kept, torch.arange(n - m, n, device="cuda")])
        at = torch.arange(a, device="cuda") if case["packed_blocks"] else keep
        slots[off[r]:off[r] + a] = order[taken + at // S] * S + (at % S).to(torch.int32)
        ids[off[r]:off[r] + a] = keep.to(torch.int32)
        taken += need[r]
    q_off = [0]
    for m in steps:
        q_off.append(q_off[-1] + m)
    dev = dict(dtype=torch.int32, device="cuda")
    total = q_off[-1]
    pool = [_pool_rows(gen, case, blocks * S, like) for like in ("k", "v")]
    at = torch.arange(total, **dev)
    back = torch.repeat_interleave(torch.tensor([n - b for n, b in zip(lens, q_off[1:])], **dev), torch.tensor(steps, device="cuda"))
    return dict(q=_values(gen, total, case["hq"], case["d"], dtype, "q"), k_pool=pool[0].view(blocks * S, -1), v_pool=pool[1].view(blocks * S, -1),
                tokens=off[-1], num_requests=torch.tensor([len(lens)], **dev), tt_offsets=torch.tensor(off, **dev),
                cache_slots=slots, cache_ids=ids, cache_len=torch.tensor(live, **dev), q_offsets=torch.tensor(q_off, **dev),
                positions=at + back, out=torch.empty(total, case["hq"], case["d"], dtype=dtype, device="cuda"),
                lse=torch.empty(total, case["hq"], dtype=torch.float32, device="cuda"),
                max_query_len=max(steps), max_live=max(live))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = _prepare_write(case, gen) if case["op"] == "write" else _prepare_attention(case, gen)
    s["case"] = case
    if own:                                   # the handle and the workspace a serving program keeps
        s["lib"] = _Context(s, case)
    return s


# ---- one pass ------------------------------------------------------------------------------------
def run(state):
    if state["case"]["op"] == "write":
        return (_own_write if own else _plain_write)(state)
    return (_own_attention if own else _plain_attention)(state)


def _own_write(s):
    c, lib = s["case"], s["lib"]
    lib.vt.vtoken_write_tokens(lib.ctx, heads=lib.heads, layer=0, max_tokens=s["tokens"], q=s["q"], k=s["k"], v=s["v"],
                               positions=s["positions"], slots=s["slots"], q_out=s["q_out"], q_weight=s["q_weight"],
                               k_weight=s["k_weight"], eps=EPS, cos_sin=s["cos_sin"], max_position=s["cos_sin"].shape[0],
                               rot_dim=c["rot"], interleaved=c["interleaved"], q_stride=s["q"].stride(0),
                               k_stride=s["k"].stride(0), v_stride=s["v"].stride(0))
    if c["kv"] != "fp4":
        return s["q_out"], s["k_pool"], s["v_pool"]
    lib.vt.vtoken_read_tokens(lib.ctx, heads=lib.heads, layer=0, max_tokens=s["tokens"], slots=s["slots"],
                              out_k=s["k_back"], out_v=s["v_back"])
    return s["q_out"], s["k_back"], s["v_back"]


def _own_attention(s):
    c, lib = s["case"], s["lib"]
    lib.vt.vtoken_attention(lib.ctx, heads=lib.heads, layer=0, num_requests=s["num_requests"], q_offsets=s["q_offsets"],
                            positions=s["positions"], q=s["q"], max_query_tokens=s["q"].shape[0],
                            max_query_len=s["max_query_len"], tt_offsets=s["tt_offsets"], cache_slots=s["cache_slots"],
                            cache_ids=s["cache_ids"], cache_len=s["cache_len"], out=s["out"], lse=s["lse"],
                            sm_scale=c["d"] ** -0.5, window=c["window"], sinks=c["sinks"], workspace=lib.workspace,
                            workspace_bytes=lib.workspace_bytes)
    return s["out"], s["lse"]


def _plain_write(s):
    c = s["case"]
    half = c["rot"] // 2
    cs = s["cos_sin"][s["positions"].long()].unsqueeze(1)
    cos, sin = cs[..., :half], cs[..., half:]

    def heads(x, w):
        x = x.float()
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
        r = x[..., :c["rot"]]
        a, b = (r[..., 0::2], r[..., 1::2]) if c["interleaved"] else (r[..., :half], r[..., half:])
        turned = (a * cos - b * sin, b * cos + a * sin)
        turned = torch.stack(turned, -1).flatten(-2) if c["interleaved"] else torch.cat(turned, -1)
        return torch.cat([turned, x[..., c["rot"]:]], -1).to(ACT[c["act"]])
    q, k = heads(s["q"], s["q_weight"]), heads(s["k"], s["k_weight"])
    at, n = s["slots"].long(), s["tokens"]
    if c["kv"] != "fp4":
        s["k_pool"][at] = k.view(n, -1)
        s["v_pool"][at] = s["v"].reshape(n, -1)
        return q, s["k_pool"], s["v_pool"]
    s["k_pool"][at] = _quantise(k.float())
    s["v_pool"][at] = _quantise(s["v"].float())
    return (q, _dequantise(s["k_pool"][at], c["hkv"], c["d"]).to(ACT[c["act"]]),
            _dequantise(s["v_pool"][at], c["hkv"], c["d"]).to(ACT[c["act"]]))


def _plain_attention(s):
    """All requests at once, padded to the longest: scores, mask, softmax, product."""
    c = s["case"]
    R, L, M, hq, hkv, d = c["requests"], s["max_live"], s["max_query_len"], c["hq"], c["hkv"], c["d"]
    at = torch.arange(L, device="cuda")
    entry = (s["tt_offsets"][:-1].long().unsqueeze(1) + at).clamp(max=s["cache_slots"].shape[0] - 1)     # [R, L]
    there = at < s["cache_len"].unsqueeze(1)
    ids = torch.where(there, s["cache_ids"][entry], torch.full_like(entry, 1 << 30, dtype=torch.int32))
    slots = torch.where(there, s["cache_slots"][entry], 0).long().flatten()
    if c["kv"] == "fp4":
        k, v = (_dequantise(s[p][slots], hkv, d) for p in ("k_pool", "v_pool"))
    else:
        k, v = (s[p][slots].float() for p in ("k_pool", "v_pool"))
    k, v = (x.view(R, L, hkv, d).transpose(1, 2) for x in (k, v))                                        # [R, hkv, L, d]
    row = torch.arange(M, device="cuda")
    many = (s["q_offsets"][1:] - s["q_offsets"][:-1]).unsqueeze(1)
    query = (s["q_offsets"][:-1].long().unsqueeze(1) + row).clamp(max=s["q"].shape[0] - 1)               # [R, M]
    pos = s["positions"][query]
    q = s["q"][query.flatten()].float().view(R, M, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(R, hkv, -1, d)
    score = (q @ k.transpose(-1, -2)).view(R, hq, M, L) * d ** -0.5
    sees = ids.unsqueeze(1) <= pos.unsqueeze(2)                                                          # [R, M, L]
    if c["window"]:
        sees &= (ids.unsqueeze(1) > pos.unsqueeze(2) - c["window"]) | (ids.unsqueeze(1) < c["sinks"])
    score = score.masked_fill_(~sees.unsqueeze(1), -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3.0e38)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p.view(R, hkv, -1, L) @ v).view(R, hq, M, d) / total.clamp(min=1e-38)
    lse = (total.log() + top).squeeze(-1)
    mine = (row < many).flatten()
    out = out.permute(0, 2, 1, 3).reshape(R * M, hq, d)[mine].to(ACT[c["act"]])
    return out, lse.permute(0, 2, 1).reshape(R * M, hq)[mine].contiguous()


# ---- the definitions in 64 bits ------------------------------------------------------------------
def _grid64(x):
    """Nearest of the sixteen values of the 4-bit grid, by distance; of two equally near the one with the even code."""
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    a = x.abs().clamp(max=6.0)
    up = torch.searchsorted(grid, a.contiguous()).clamp(max=7)
    dn = (up - 1).clamp(min=0)
    du, dd = grid[up] - a, a - grid[dn]
    pick = torch.where((dd < du) | ((dd == du) & (dn % 2 == 0)), dn, up)
    return torch.copysign(grid[pick], x)


def _scale64(x):
    """Nearest 8-bit scale (3 mantissa bits, steps of 2^-9 at the bottom, 448 at most) of non-negative 64-bit values."""
    e = torch.floor(torch.log2(x.clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(max=448.0)


def _held64(x):
    """What a row of 16-bit values stands for once it is held in 4 bits."""
    n, h, d = x.shape
    g = x.double().view(n, h, d // GROUP, GROUP)
    s = _scale64(g.abs().amax(-1, keepdim=True) / 6.0)
    return torch.where(s > 0, _grid64(g / s.clamp(min=2.0 ** -9)) * s, 0.0).view(n, h, d)


def _exact_write(case, s):
    half, rot = case["rot"] // 2, case["rot"]
    cs = s["cos_sin"].double()[s["positions"].long()]
    z = torch.complex(cs[:, :half], cs[:, half:]).unsqueeze(1)

    def heads(x, w):
        x = x.double()
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["d"] + EPS) * w.double()
        out = x.clone()
        if case["interleaved"]:
            y = torch.view_as_real(torch.view_as_complex(x[..., :rot].reshape(*x.shape[:2], half, 2).contiguous()) * z)
            out[..., :rot] = y.flatten(-2)
        else:
            y = torch.complex(x[..., :half], x[..., half:rot]) * z
            out[..., :half], out[..., half:rot] = y.real, y.imag
        return out
    q, k = heads(s["q"], s["q_weight"]), heads(s["k"], s["k_weight"])
    at = s["slots"].long()
    if case["kv"] == "fp4":
        return q, _held64(k.to(ACT[case["act"]])), _held64(s["v"])
    pools = [torch.zeros(s[p].shape, dtype=torch.float64, device="cuda") for p in ("k_pool", "v_pool")]
    pools[0][at], pools[1][at] = k.flatten(1), s["v"].double().flatten(1)
    return q, pools[0], pools[1]


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


def exact(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] == "write":
        return _exact_write(case, _prepare_write(case, gen))
    s = _prepare_attention(case, gen)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    off, q_off, live = s["tt_offsets"].tolist(), s["q_offsets"].tolist(), s["cache_len"].tolist()
    for r in range(case["requests"]):
        here = slice(off[r], off[r] + live[r])
        k, v = (_rows64(case, s[p], s["cache_slots"][here]) for p in ("k_pool", "v_pool"))
        ids = s["cache_ids"][here]
        for a in range(q_off[r], q_off[r + 1], 1024):
            b = min(a + 1024, q_off[r + 1])
            pos = s["positions"][a:b].unsqueeze(1)
            hidden = ids > pos
            if case["window"]:
                hidden |= (ids <= pos - case["window"]) & (ids >= case["sinks"])
            for h in range(hkv):
                g = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
                x = torch.einsum("mgd,ld->gml", s["q"][a:b, g].double(), k[:, h]) / math.sqrt(d)
                x.masked_fill_(hidden, -math.inf)
                z = torch.logsumexp(x, -1)
                w = torch.exp(x - z.unsqueeze(-1)).nan_to_num(0.0)
                out[a:b, g] = torch.einsum("gml,ld->mgd", w, v[:, h])
                lse[a:b, g] = z.transpose(0, 1)
    return out, lse
