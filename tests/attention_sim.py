"""Problems and 64-bit references for the attention step: token writes, 4-bit rows, attention over a slot cache.
Everything here is written from the definitions in the header, in numpy and float64."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
KINDS = {"bf16": 0, "fp16": 1, "fp4": 2}


def torch_dtype(act):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16}[act]


def unit(act):
    """Unit roundoff of the 16-bit type: 8 and 11 significant bits."""
    return 2.0 ** -8 if act == "bf16" else 2.0 ** -11


def to64(t):
    return t.detach().cpu().double().numpy()


def round16(x, act):
    """float64 -> nearest 16-bit value (through the type's own spacing), as float64."""
    bits, emin = (8, -126) if act == "bf16" else (11, -14)
    m, e = np.frexp(x)
    e = np.maximum(e - 1, emin)
    step = np.ldexp(1.0, e - (bits - 1))
    return np.where(np.isfinite(x), np.rint(x / step) * step, x)


# ---- 4-bit rows ----------------------------------------------------------------------------------
def scale_values():
    b = np.arange(128)
    e, f = b >> 3, b & 7
    v = np.where(e > 0, (1 + f / 8.0) * np.exp2(e - 7.0), f * 2.0 ** -9)
    v[127] = np.nan
    return v


def quantise_rows(x, exponent=0):
    """float64 [n, heads, d] -> uint8 rows, by search over the tables of values."""
    n, h, d = x.shape
    x = x * 2.0 ** -exponent
    g = x.reshape(n, h, d // 16, 16)
    table = scale_values()[:127]
    odd = ~np.isfinite(g).all(-1)
    top = np.abs(np.where(np.isfinite(g), g, 0)).max(-1) / 6.0
    sc = nearest_even(table, np.minimum(top, 448.0))
    s = table[sc]
    ratio = np.where(s[..., None] > 0, np.where(odd[..., None], 0, np.where(np.isfinite(g), g, 0)) / np.where(s > 0, s, 1)[..., None], 0)
    code = nearest_even(GRID, np.minimum(np.abs(ratio), 6.0)).astype(np.uint8) | (np.signbit(ratio).astype(np.uint8) << 3)
    sc = np.where(odd, 127, sc).astype(np.uint8)
    code = np.where(odd[..., None], 0, code).reshape(n, h, d).astype(np.uint8)
    row = np.zeros((n, row_bytes("fp4", h, d)), np.uint8)
    row[:, :h * d // 2] = (code[..., 0::2] | (code[..., 1::2] << 4)).reshape(n, -1)
    row[:, h * d // 2:h * d // 2 + h * d // 16] = sc.reshape(n, -1)
    return row


def nearest_even(table, x):
    """Index of the nearest entry of an ascending table; of two equally near the even index."""
    up = np.clip(np.searchsorted(table, x), 0, len(table) - 1)
    dn = np.maximum(up - 1, 0)
    du, dd = table[up] - x, x - table[dn]
    return np.where((dd < du) | ((dd == du) & (dn % 2 == 0)), dn, up)


def dequantise_rows(row, h, d, exponent=0):
    row = np.asarray(row)
    n = row.shape[0]
    c = row[:, :h * d // 2].reshape(n, h, d // 2)
    code = np.stack([c & 15, c >> 4], -1).reshape(n, h, d)
    val = GRID[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = scale_values()[row[:, h * d // 2:h * d // 2 + h * d // 16].reshape(n, h, d // 16) & 127]
    return val * np.repeat(s, 16, -1) * 2.0 ** exponent


def row_bytes(kv, h, d):
    return -(-h * (d // 2 + d // 16) // 16) * 16 if kv == "fp4" else h * d * 2


# ---- a cache on the device ------------------------------------------------------------------------
class Cache:
    """K and V pools with random rows in every slot of interest, poison everywhere else."""

    def __init__(self, rng, kv, act, hq, hkv, d, slots, used, layers=2, block=16, max_requests=8, max_tokens=4096,
                 k_exponent=0, v_exponent=0, poison=True, scale=1.0):
        import torch
        from paper_2608_13263_b200 import binding as vt
        self.kv, self.act, self.hq, self.hkv, self.d, self.block, self.layers = kv, act, hq, hkv, d, block, layers
        self.k_exponent, self.v_exponent = k_exponent, v_exponent
        self.dev = torch.device("cuda:0")
        self.slots = -(-slots // block) * block
        self.layer = layers - 1
        self.k64, self.v64 = {}, {}
        used = np.asarray(used, np.int64)
        rb = row_bytes(kv, hkv, d)
        pools = []
        for name, exponent in (("k64", k_exponent), ("v64", v_exponent)):
            x = rng.standard_normal((len(used), hkv, d)) * scale * 2.0 ** exponent
            if kv == "fp4":
                host = np.full((layers, self.slots, rb), 0xff if poison else 0, np.uint8)     # scale bytes 0xff: NaN
                rows = quantise_rows(round16(x, "fp16" if exponent == 0 else "bf16"), exponent)
                host[self.layer, used] = rows
                x = dequantise_rows(rows, hkv, d, exponent)
                pool = torch.from_numpy(host).to(self.dev)
            else:
                pool = torch.full((layers, self.slots, hkv * d), float("nan") if poison else 0.0, dtype=torch_dtype(act), device=self.dev)
                rows = torch.from_numpy(x.reshape(len(used), -1)).to(self.dev).to(torch_dtype(act))
                pool[self.layer, torch.from_numpy(used).to(self.dev)] = rows
                x = to64(rows).reshape(len(used), hkv, d)
            setattr(self, name, dict(zip(used.tolist(), x)))
            pools.append(pool)
        self.k_pool, self.v_pool = pools
        self.heads = vt.Heads(hq, hkv, d, KINDS[kv], KINDS[act], k_exponent, v_exponent)
        geo = (1, rb, 1) if kv == "fp4" else (hkv, d, 2)
        self.ctx = vt.vtoken_create(layers, self.slots // block, block, geo[0], geo[1], self.k_pool, self.v_pool, max_requests,
                                    max_tokens, max_tokens, 4, elem_bytes=geo[2])
        self.max_requests, self.max_tokens = max_requests, max_tokens

    def flags(self):
        from paper_2608_13263_b200 import binding as vt
        return vt.vtoken_read_counts(self.ctx)["error_flags"]

    def close(self):
        from paper_2608_13263_b200 import binding as vt
        vt.vtoken_destroy(self.ctx)


class Step:
    """Ragged queries over a Cache: tables, inputs, outputs, the 64-bit result."""

    def __init__(self, rng, cache, ids, slots, positions, window=0, sinks=0, q_pad=0, gap=0, identity=False, q_scale=1.0,
                 max_query_len=None):
        """ids, slots: per request, active tokens; positions: per request, of its query tokens; gap: unused entries
        behind every request's cache; q_pad: unused elements behind every token of q and out."""
        import torch
        self.c, self.ids, self.slots, self.positions, self.window, self.sinks = cache, ids, slots, positions, window, sinks
        R = len(ids)
        dev = cache.dev
        self.offsets = np.zeros(R + 1, np.int32)
        for r in range(R):
            self.offsets[r + 1] = self.offsets[r] + len(ids[r]) + gap
        T = max(1, int(self.offsets[-1]))
        s, i = np.full(T, 1 << 30, np.int32), np.full(T, 7, np.int32)
        for r in range(R):
            o = self.offsets[r]
            s[o:o + len(ids[r])], i[o:o + len(ids[r])] = slots[r], ids[r]
        q_off = np.concatenate([[0], np.cumsum([len(p) for p in positions])]).astype(np.int32)
        self.q_off, self.n = q_off, int(q_off[-1])
        pad = lambda a, n: np.concatenate([a, np.full(n - len(a), 1 << 30)]).astype(np.int32)      # noqa: E731
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)                            # noqa: E731
        self.num_requests = up(np.array([R], np.int32))
        self.tt_offsets = up(pad(self.offsets, cache.max_requests + 1))
        self.cache_slots = up(pad(s, cache.max_tokens))
        self.cache_ids = None if identity else up(pad(i, cache.max_tokens))
        self.cache_len = up(pad(np.array([len(x) for x in ids]), max(cache.max_requests, R)))
        self.q_offsets = up(pad(q_off, cache.max_requests + 1))
        flat = np.concatenate([np.asarray(p, np.int32) for p in positions] + [np.zeros(0, np.int32)])
        self.pos = up(np.concatenate([flat, np.zeros(1, np.int32)]))
        rows, width = max(1, self.n), cache.hq * cache.d + q_pad
        q = rng.standard_normal((rows, width)) * q_scale
        self.q_all = up(q).to(torch_dtype(cache.act))
        self.out_all = torch.full((rows, width), 77.0, dtype=torch_dtype(cache.act), device=dev)
        self.lse = torch.full((rows, cache.hq), 77.0, dtype=torch.float32, device=dev)
        self.stride = width
        self.max_query_len = max_query_len or max([1] + [len(p) for p in positions])
        self.sm_scale = cache.d ** -0.5

    def run(self, workspace=None, stream=None):
        import torch
        from paper_2608_13263_b200 import binding as vt
        c = self.c
        n = vt.vtoken_attention_workspace_bytes(c.ctx, c.heads, max(1, self.n))
        self.workspace = torch.zeros(max(16, n), dtype=torch.uint8, device=c.dev) if workspace is None else workspace
        self.workspace_bytes = n
        self.call(stream)
        return self

    def call(self, stream=None):
        from paper_2608_13263_b200 import binding as vt
        c = self.c
        vt.vtoken_attention(c.ctx, heads=c.heads, layer=c.layer, num_requests=self.num_requests, q_offsets=self.q_offsets,
                            positions=self.pos, q=self.q_all, max_query_tokens=self.n, max_query_len=self.max_query_len,
                            tt_offsets=self.tt_offsets, cache_slots=self.cache_slots, cache_ids=self.cache_ids,
                            cache_len=self.cache_len, out=self.out_all, lse=self.lse, sm_scale=self.sm_scale,
                            window=self.window, sinks=self.sinks, q_stride=self.stride, out_stride=self.stride,
                            workspace=self.workspace, workspace_bytes=self.workspace_bytes, stream=stream)

    def outputs(self):
        c = self.c
        return to64(self.out_all)[:self.n, :c.hq * c.d].reshape(self.n, c.hq, c.d), to64(self.lse)[:self.n]

    def reference(self):
        """(out, lse, bound of |out| error, bound of lse error), float64."""
        c = self.c
        q = to64(self.q_all)[:self.n, :c.hq * c.d].reshape(self.n, c.hq, c.d)
        out, lse = np.zeros((self.n, c.hq, c.d)), np.full((self.n, c.hq), -np.inf)
        out_tol, lse_tol = np.zeros((self.n, c.hq, c.d)), np.zeros((self.n, c.hq))
        u = unit(c.act)
        for r in range(len(self.ids)):
            live = [(i, s) for i, s in zip(self.ids[r], self.slots[r]) if 0 <= s < c.slots]
            for j, p in enumerate(self.positions[r]):
                row = int(self.q_off[r]) + j
                seen = [s for i, s in live if i <= p and (not self.window or i > p - self.window or i < self.sinks)]
                if not seen:
                    continue
                k, v = np.stack([c.k64[s] for s in seen]), np.stack([c.v64[s] for s in seen])
                kh, vh = (np.repeat(x, c.hq // c.hkv, 1) for x in (k, v))
                with np.errstate(all="ignore"):
                    s = np.einsum("hd,lhd->hl", q[row], kh) * self.sm_scale
                    top = s.max(-1, keepdims=True)
                    e = np.exp(s - top)
                    z = e.sum(-1, keepdims=True)
                    out[row] = np.einsum("hl,lhd->hd", e / z, vh)
                    lse[row] = (top + np.log(z))[:, 0]
                    # a 32-bit sum of D exact products, in any order: D * 2^-24 of the sum of their absolute values, twice for
                    # accumulators that cut instead of rounding; it is a relative error of every weight
                    ds = (c.d * 2.0 ** -23 * np.einsum("hd,lhd->hl", np.abs(q[row]), np.abs(kh)) * abs(self.sm_scale)).max(-1)
                    ds = ds + 2.0 ** -20 * (1 + np.abs(s).max(-1))
                    va = np.abs(vh).max(0)
                    # the output's own rounding; weights rounded once to 16 bits (u each); the scores' error on both sides of the quotient
                    out_tol[row] = 1.01 * u * np.abs(out[row]) + (u + 2 * ds[:, None] + 2.0 ** -18) * va + 2.0 ** -24
                    lse_tol[row] = ds + 2.0 ** -20 * (1 + np.abs(lse[row]))
        return out, lse, out_tol, lse_tol

    def check(self):
        out, lse = self.outputs()
        ref, ref_lse, tol, lse_tol = self.reference()
        bad = ~np.isfinite(ref).all(-1)
        assert np.array_equal(np.isnan(out).any(-1) | np.isinf(out).any(-1), bad), "finite where it should not be, or the reverse"
        good = ~bad
        err = np.abs(out - ref)[good]
        assert (err <= tol[good]).all(), f"out off by {err.max()} ({(err / tol[good]).max()} of the bound)"
        gone = np.isneginf(ref_lse)
        assert np.array_equal(np.isneginf(lse), gone)
        ok = good & ~gone
        assert (np.abs(lse[ok] - ref_lse[ok]) <= lse_tol[ok]).all()
        assert (out[gone] == 0).all()
        return out, lse


def spread(rng, lens, keep=1.0, extra=40, block=16):
    """Active ids and slots of requests of the given logical lengths: ids by an eviction that keeps each with
    probability ``keep`` (the newest always), slots by token position in permuted blocks.  Returns ids, slots, slots of the pool."""
    need = [-(-n // block) for n in lens]
    order = rng.permutation(sum(need) + -(-extra // block))
    ids, slots, at = [], [], 0
    for n, b in zip(lens, need):
        mine = order[at:at + b]
        at += b
        i = np.arange(n)
        alive = rng.random(n) < keep
        if n:
            alive[-1] = True
        i = i[alive]
        ids.append(i)
        slots.append(mine[i // block] * block + i % block)
    return ids, slots, len(order) * block
