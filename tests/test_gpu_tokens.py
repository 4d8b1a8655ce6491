"""vtoken_write_tokens and vtoken_read_tokens against their definition in 64 bits: 16-bit rows within the output's rounding,
4-bit rows bit for bit."""
import numpy as np
import pytest

import attention_sim as sim
from attention_sim import KINDS, round16, to64, torch_dtype, unit
from paper_2608_13263_b200 import binding as vt

pytestmark = pytest.mark.gpu

GEOMETRIES = [("bf16", "bf16", 8, 2, 128), ("fp16", "fp16", 7, 1, 128), ("bf16", "bf16", 4, 4, 64), ("bf16", "fp4", 8, 2, 128),
              ("fp16", "fp4", 3, 3, 128), ("fp16", "fp4", 14, 2, 64), ("bf16", "fp4", 1, 1, 64), ("bf16", "bf16", 32, 8, 128)]
IDS = ["-".join(map(str, g)) for g in GEOMETRIES]


class Writer:
    def __init__(self, rng, geometry, n, rot=None, interleaved=False, weights=True, packed=True, in_place=False, layers=2,
                 exponents=(0, 0), scale=1.0, block=16):
        import torch
        self.act, self.kv, self.hq, self.hkv, self.d = geometry
        act, kv, hq, hkv, d = geometry
        self.n, self.rot, self.interleaved, self.weights, self.exponents = n, d if rot is None else rot, interleaved, weights, exponents
        self.dev = dev = torch.device("cuda:0")
        dt = torch_dtype(act)
        up = lambda x, t=None: torch.from_numpy(np.ascontiguousarray(x)).to(dev) if t is None else torch.from_numpy(np.ascontiguousarray(x)).to(dev).to(t)  # noqa: E731
        rows = max(1, n)
        all3 = up(rng.standard_normal((rows, (hq + 2 * hkv) * d + 8)) * scale, dt)
        self.q, self.k, self.v = all3[:, :hq * d], all3[:, hq * d:(hq + hkv) * d], all3[:, (hq + hkv) * d:(hq + 2 * hkv) * d]
        if not packed:
            self.q, self.k, self.v = (x.contiguous() for x in (self.q, self.k, self.v))
        self.qw, self.kw = up(1 + 0.3 * rng.standard_normal(d), dt), up(1 + 0.3 * rng.standard_normal(d), dt)
        self.q64, self.k64, self.v64 = (to64(x) for x in (self.q, self.k, self.v))
        self.top = 5000
        ang = np.outer(np.arange(self.top), 10000.0 ** (-np.arange(max(1, self.rot // 2)) / max(1, self.rot // 2)))
        self.cs = np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)
        self.cos_sin = up(self.cs)
        self.positions = rng.integers(0, self.top, rows).astype(np.int32)
        blocks = -(-rows // block) + 2
        self.slots = rng.permutation(blocks * block)[:rows].astype(np.int32)
        self.layers, self.layer = layers, layers - 1
        self.rb = sim.row_bytes(kv, hkv, d)
        if kv == "fp4":
            self.pools = [torch.full((layers, blocks * block, self.rb), 0x55, dtype=torch.uint8, device=dev) for _ in range(2)]
        else:
            self.pools = [torch.full((layers, blocks * block, hkv * d), 3.0, dtype=dt, device=dev) for _ in range(2)]
        geo = (1, self.rb, 1) if kv == "fp4" else (hkv, d, 2)
        self.heads = vt.Heads(hq, hkv, d, KINDS[kv], KINDS[act], *exponents)
        self.ctx = vt.vtoken_create(layers, blocks, block, geo[0], geo[1], self.pools[0], self.pools[1], 4, 64, 64, 4, elem_bytes=geo[2])
        self.pos_dev, self.slots_dev = up(self.positions), up(self.slots)
        self.q_out = self.q if in_place else torch.full((rows, hq * d), 9.0, dtype=dt, device=dev)
        self.eps = 1e-5

    def args(self):
        return dict(heads=self.heads, layer=self.layer, max_tokens=self.n, q=self.q, k=self.k, v=self.v, positions=self.pos_dev,
                    slots=self.slots_dev, q_out=self.q_out, q_weight=self.qw if self.weights else None,
                    k_weight=self.kw if self.weights else None, eps=self.eps, cos_sin=self.cos_sin, max_position=self.top,
                    rot_dim=self.rot, interleaved=self.interleaved, q_stride=self.q.stride(0), k_stride=self.k.stride(0),
                    v_stride=self.v.stride(0), q_out_stride=self.q_out.stride(0))

    def write(self, **change):
        vt.vtoken_write_tokens(self.ctx, **{**self.args(), **change})

    def turned(self, x, w):
        """[n, heads, d] in float64: normalised and rotated."""
        if self.weights:
            x = x / np.sqrt((x * x).mean(-1, keepdims=True) + np.float64(np.float32(self.eps))) * to64(w)
        else:
            x = x.copy()
        h = self.rot // 2
        if h == 0:
            return x
        cs = self.cs[np.clip(self.positions, 0, self.top - 1)].astype(np.float64)[:, None]
        c, s = cs[..., :h], cs[..., h:]
        ia, ib = (np.arange(0, 2 * h, 2), np.arange(1, 2 * h, 2)) if self.interleaved else (np.arange(h), np.arange(h, 2 * h))
        a, b = x[..., ia].copy(), x[..., ib].copy()
        x[..., ia], x[..., ib] = a * c - b * s, b * c + a * s
        return x

    def expected(self):
        rows = max(1, self.n)
        return (self.turned(self.q64.reshape(rows, self.hq, self.d), self.qw), self.turned(self.k64.reshape(rows, self.hkv, self.d), self.kw),
                self.v64.reshape(rows, self.hkv, self.d))

    def near(self, got, ref):
        # the 16-bit rounding, and a few dozen 32-bit roundings of values up to the head's largest
        tol = 1.01 * unit(self.act) * np.abs(ref) + 2.0 ** -18 * np.abs(ref).max(-1, keepdims=True) + 2.0 ** -25
        assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) / tol).max()

    def check(self, rows=None):
        q, k, v = self.expected()
        rows = np.arange(self.n) if rows is None else rows
        if self.hq and self.q is not None:
            self.near(to64(self.q_out).reshape(-1, self.hq, self.d)[rows], q[rows])
        s = self.slots[rows]
        if self.kv != "fp4":
            self.near(to64(self.pools[0][self.layer])[s].reshape(-1, self.hkv, self.d), k[rows])
            assert np.array_equal(to64(self.pools[1][self.layer])[s].reshape(-1, self.hkv, self.d), v[rows])
        else:
            used = self.hkv * (self.d // 2 + self.d // 16)
            for pool, x, e in ((0, round16(k, self.act), self.exponents[0]), (1, v, self.exponents[1])):
                got = self.pools[pool][self.layer].cpu().numpy()
                assert np.array_equal(got[s][:, :used], sim.quantise_rows(x[rows], e)[:, :used])
                assert (got[:, used:] == 0x55).all()
        # no other row changes
        rest = np.setdiff1d(np.arange(self.pools[0].shape[1]), s)
        for pool in self.pools:
            p = pool.cpu().double().numpy() if self.kv == "fp4" else to64(pool)
            assert (p[self.layer][rest] == (0x55 if self.kv == "fp4" else 3.0)).all()
            assert (p[:self.layer] == (0x55 if self.kv == "fp4" else 3.0)).all()

    def flags(self):
        return vt.vtoken_read_counts(self.ctx)["error_flags"]

    def close(self):
        vt.vtoken_destroy(self.ctx)


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
@pytest.mark.parametrize("n", [1, 2, 3, 17, 130])
def test_write(geometry, n):
    w = Writer(np.random.default_rng(n), geometry, n)
    w.write()
    w.check()
    assert w.flags() == 0
    w.close()


@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[2], GEOMETRIES[3], GEOMETRIES[5]], ids=["16-128", "16-64", "4-128", "4-64"])
@pytest.mark.parametrize("rot,interleaved", [(0, False), (16, False), (48, False), (64, False), (16, True), (48, True), (64, True)])
@pytest.mark.parametrize("weights", [True, False])
def test_rotations(geometry, rot, interleaved, weights):
    w = Writer(np.random.default_rng(rot), geometry, 9, rot=rot, interleaved=interleaved, weights=weights, packed=weights, in_place=interleaved)
    w.write()
    w.check()
    w.close()


def test_interleaved_whole_head():
    for g in (GEOMETRIES[1], GEOMETRIES[4]):
        w = Writer(np.random.default_rng(5), g, 20, interleaved=True)
        w.write()
        w.check()
        w.close()


@pytest.mark.parametrize("exponents,scale", [((0, 0), 1e-4), ((0, 0), 3000.0), ((-9, 12), 1.0), ((30, -30), 1.0)])
def test_ranges_of_4_bit_rows(exponents, scale):
    """Scales that underflow, saturate, and exponents."""
    for weights in (True, False):
        w = Writer(np.random.default_rng(6), GEOMETRIES[3], 40, exponents=exponents, scale=scale, weights=weights)
        w.write()
        w.check()
        w.close()


def test_ties_and_special_values_of_4_bit_rows():
    """Values on every tie of the grid under every kind of scale; zeros; NaN and infinities mark their group."""
    import torch
    w = Writer(np.random.default_rng(7), ("bf16", "fp4", 2, 2, 64), 64, weights=False, rot=0, packed=False)
    grid = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, -5])
    x = np.stack([np.tile(grid, 8) * 2.0 ** (i % 20 - 10) * (1 + (i % 8) / 8) for i in range(64)])
    x[3] = 0
    x[4, 5], x[5, 70], x[6, 16] = np.nan, np.inf, -np.inf
    for t in (w.k, w.v):
        t.copy_(torch.from_numpy(x).to(w.dev))
    w.k64, w.v64 = to64(w.k), to64(w.v)
    w.write()
    got = w.pools[0][w.layer].cpu().numpy()[w.slots][:, :72]
    assert np.array_equal(got, sim.quantise_rows(w.k64.reshape(64, 2, 64))[:, :72])
    assert np.array_equal(w.pools[1][w.layer].cpu().numpy()[w.slots][:, :72], got)
    out = torch.zeros((64, 2, 64), dtype=torch.bfloat16, device=w.dev)
    vt.vtoken_read_tokens(w.ctx, heads=w.heads, layer=w.layer, max_tokens=64, slots=w.slots_dev, out_k=out)
    ref = sim.dequantise_rows(got, 2, 64)
    assert np.array_equal(np.nan_to_num(to64(out), nan=123.0), np.nan_to_num(ref, nan=123.0)) and np.isnan(ref).sum() == 48
    w.close()


@pytest.mark.parametrize("geometry", GEOMETRIES, ids=IDS)
def test_read(geometry):
    import torch
    rng = np.random.default_rng(8)
    act, kv, hq, hkv, d = geometry
    exponents = (-3, 4) if kv == "fp4" else (0, 0)
    c = sim.Cache(rng, kv, act, hq, hkv, d, 96, np.arange(0, 96, 2), k_exponent=exponents[0], v_exponent=exponents[1])
    slots = np.array([0, 94, 10, -1, 2, -7, 50], np.int32)
    s = torch.from_numpy(slots).to(c.dev)
    k = torch.full((7, hkv, d), 5.0, dtype=torch_dtype(act), device=c.dev)
    v = torch.full_like(k, 6.0)
    vt.vtoken_read_tokens(c.ctx, heads=c.heads, layer=c.layer, max_tokens=7, slots=s, out_k=k, out_v=v)
    for got, ref in ((k, c.k64), (v, c.v64)):
        for i, x in enumerate(slots):
            want = np.zeros((hkv, d)) if x < 0 else ref[int(x)]
            assert np.array_equal(to64(got)[i], want), i
    assert c.flags() == 0
    # a count on the device, one output only, a slot outside the pool
    n = torch.tensor([2], dtype=torch.int32, device=c.dev)
    k.fill_(5.0)
    s[1] = 96
    vt.vtoken_read_tokens(c.ctx, heads=c.heads, layer=c.layer, max_tokens=7, num_tokens=n, slots=s, out_k=k)
    assert np.array_equal(to64(k)[0], c.k64[0]) and (to64(k)[1] == 0).all() and (to64(k)[2:] == 5).all()
    assert c.flags() == vt.FLAG_BAD_SLOT
    c.close()


def test_uncached_tokens_bad_slots_and_bad_positions():
    import torch
    for g in (GEOMETRIES[0], GEOMETRIES[3]):
        w = Writer(np.random.default_rng(9), g, 12)
        w.slots_dev[3], w.slots_dev[5] = -1, w.pools[0].shape[1]
        w.pos_dev[7], w.pos_dev[8] = -1, w.top
        w.write()
        assert w.flags() == vt.FLAG_BAD_SLOT | vt.FLAG_BAD_POSITION
        q, _, _ = w.expected()
        got = to64(w.q_out).reshape(12, w.hq, w.d)
        w.near(got[[0, 3, 5, 11]], q[[0, 3, 5, 11]])               # queries of tokens that are not cached
        assert (got[[7, 8]] == 9.0).all()                          # skipped altogether
        p = w.pools[0][w.layer].cpu().double().numpy()
        blank = 0x55 if w.kv == "fp4" else 3.0
        assert (p[w.slots[[3, 5, 7, 8]]] == blank).all() and (p[w.slots[[0, 11]]] != blank).any()
        # the first tokens only, without queries
        w.pools[0].fill_(int(blank))
        w.write(num_tokens=torch.tensor([2], dtype=torch.int32, device=w.dev), q=None, q_out=None, q_stride=0, q_out_stride=0)
        p = w.pools[0][w.layer].cpu().double().numpy()
        assert (p[w.slots[[0, 1]]] != blank).any() and (p[w.slots[2:]] == blank).all()
        w.close()


def test_other_stream_and_graph():
    import torch
    w = Writer(np.random.default_rng(10), GEOMETRIES[7], 40)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    w.write(stream=side)
    side.synchronize()
    w.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w.write(stream=torch.cuda.current_stream())
    w.q_out.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    w.check()
    w.close()


@pytest.mark.parametrize("geometry", [GEOMETRIES[0], GEOMETRIES[3], GEOMETRIES[5]], ids=["16", "4", "4-64"])
def test_checked_build(geometry):
    prev = vt.use_library("checked")
    try:
        w = Writer(np.random.default_rng(11), geometry, 37)
        w.write()
        w.check()
        assert w.flags() == 0
        w.close()
    finally:
        vt.use_library(prev)


def test_refusals():
    w = Writer(np.random.default_rng(12), GEOMETRIES[0], 4)

    def refused(code=vt.EINVAL, **change):
        with pytest.raises(vt.VtokenError) as e:
            w.write(**change)
        assert e.value.code == code
    for name in ("k", "v", "slots", "q_out", "cos_sin", "positions"):
        refused(**{name: None})
    for change in (dict(layer=-1), dict(layer=2), dict(max_tokens=-1), dict(rot_dim=8), dict(rot_dim=144), dict(rot_dim=-16), dict(max_position=0),
                   dict(eps=0.0), dict(eps=float("nan")), dict(q=w.q.data_ptr() + 2), dict(k=w.k.data_ptr() + 8), dict(q_stride=4),
                   dict(k_stride=w.hkv * w.d + 3), dict(q_out=w.q, q_out_stride=0)):
        refused(**change)
    H = vt.Heads
    for heads in (H(8, 3, 128, 0, 0, 0, 0), H(8, 2, 96, 0, 0, 0, 0), H(8, 2, 128, 1, 0, 0, 0), H(8, 2, 128, 2, 0, 99, 0), H(8, 2, 128, 0, 0, 0, 1)):
        refused(heads=heads)
        if heads.num_q_heads % heads.num_kv_heads or heads.head_dim == 96:
            with pytest.raises(vt.VtokenError):
                vt.vtoken_kv_row_bytes(heads)
    assert vt.vtoken_kv_row_bytes(H(8, 2, 128, 2, 0, 0, 0)) == 144 and vt.vtoken_kv_row_bytes(H(1, 1, 64, 2, 1, 0, 0)) == 48
    with pytest.raises(vt.VtokenError):
        vt.vtoken_read_tokens(w.ctx, heads=w.heads, layer=0, max_tokens=3, slots=None, out_k=w.q_out)
    with pytest.raises(vt.VtokenError):
        vt.vtoken_read_tokens(w.ctx, heads=w.heads, layer=0, max_tokens=3, slots=w.slots_dev, out_k=w.q_out.data_ptr() + 2)
    w.write(max_tokens=0)
    assert w.flags() == 0
    w.close()
