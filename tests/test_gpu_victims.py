"""Cutting requests back to a budget, and verification of drafted tokens, against plain Python in 64 bits: whole numbers, equal."""
import numpy as np
import pytest

from paper_2608_13263_b200 import binding as vt

pytestmark = pytest.mark.gpu


def context(max_requests, max_tokens):
    import torch
    pool = torch.zeros(64, dtype=torch.uint8, device="cuda:0")
    ctx = vt.vtoken_create(1, 1, 1, 1, 16, pool, pool, max_requests, max(1, max_tokens), 1, 1, elem_bytes=1)
    return ctx, pool


def up(a, dtype=np.int32):
    import torch
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype))).to("cuda:0")


# ---- select ---------------------------------------------------------------------------------------
class Cut:
    def __init__(self, rng, lens, live=None, gap=0, identity=False, max_requests=None, scores=None):
        """lens: table entries of each request; live: how many of them are active."""
        R = len(lens)
        live = lens if live is None else live
        self.ids = [np.sort(rng.permutation(n)[:a]) if a < n else np.arange(a) for n, a in zip(lens, live)]
        self.offsets = np.concatenate([[0], np.cumsum([n + gap for n in lens])]).astype(np.int32)
        self.lens, self.R = [n + gap for n in lens], R
        T = max(1, int(self.offsets[-1]))
        flat = np.full(T, -7, np.int32)
        for r in range(R):
            flat[self.offsets[r]:self.offsets[r] + len(self.ids[r])] = self.ids[r]
        self.scores = (rng.standard_normal(T) if scores is None else scores(T)).astype(np.float32)
        self.T = T
        self.ctx, self.pool = context(max_requests or max(1, R), T)
        self.dev = dict(num_requests=up([R]), tt_offsets=up(self.offsets), cache_ids=None if identity else up(flat),
                        cache_len=up([len(i) for i in self.ids] or [0]))

    def run(self, budget, sinks=0, recent=0, shared=None, max_victims=None, hint=None, stream=None):
        import torch
        cap = self.T if max_victims is None else max_victims
        self.req, self.tok = (torch.full((cap + 3,), -9, dtype=torch.int32, device="cuda:0") for _ in range(2))
        self.num = torch.full((1,), -9, dtype=torch.int32, device="cuda:0")
        self.inputs = (up(self.scores, np.float32), up(budget if self.R else [0]), None if shared is None else up(shared))
        vt.vtoken_select_victims(self.ctx, **self.dev, scores=self.inputs[0], budget=self.inputs[1], shared_len=self.inputs[2], sinks=sinks,
                                 recent=recent, max_cache_len=hint or max([1] + [len(i) for i in self.ids]), victim_req=self.req,
                                 victim_tok=self.tok, max_victims=cap, num_victims=self.num, stream=stream)
        torch.cuda.synchronize()
        n = int(self.num)
        req, tok = self.req.cpu().numpy(), self.tok.cpu().numpy()
        assert (req[min(cap, n):] == -9).all() and (tok[min(cap, n):] == -9).all()
        return list(zip(req[:n].tolist(), tok[:n].tolist()))

    def reference(self, budget, sinks=0, recent=0, shared=None):
        out = []
        for r in range(self.R):
            ids, n = self.ids[r], len(self.ids[r])
            v = n - max(0, int(budget[r]))
            free = [e for e in range(n) if e < n - recent and e >= (0 if shared is None else shared[r]) and ids[e] >= sinks]

            def rank(e):                                     # lowest first; NaN below all; of equal ones the last
                x = float(self.scores[self.offsets[r] + ids[e]])
                return (0, 0.0, -e) if x != x else (1, x, -e)
            gone = sorted(sorted(free, key=rank)[:max(0, v)])
            out += [(r, int(ids[e])) for e in gone]
        return out

    def check(self, budget, **options):
        hint = options.pop("hint", None)
        got = self.run(budget, hint=hint, **options)
        assert got == self.reference(budget, **options)
        return got

    def close(self, flags=0):
        assert vt.vtoken_read_counts(self.ctx)["error_flags"] == flags
        vt.vtoken_destroy(self.ctx)


@pytest.mark.parametrize("identity", [False, True])
def test_lengths_and_budgets(identity):
    rng = np.random.default_rng(1)
    lens = [0, 1, 2, 31, 32, 33, 511, 512, 513, 1024, 3000, 0, 5]
    c = Cut(rng, lens, None if identity else [n - n // 3 for n in lens], gap=2, identity=identity)
    for budget in ([0] * 13, [n // 2 for n in lens], [1] * 13, [1 << 30] * 13, [-5] * 13, [max(0, n - 1) for n in lens]):
        c.check(budget)
    c.close()


@pytest.mark.parametrize("sinks,recent", [(4, 0), (0, 7), (4, 100), (1000, 3), (0, 1 << 30), (1 << 30, 0)])
def test_what_stays(sinks, recent):
    rng = np.random.default_rng(2)
    lens = [1, 3, 5, 90, 400, 2000]
    c = Cut(rng, lens, [1, 2, 5, 40, 300, 900])
    c.check([n // 4 for n in lens], sinks=sinks, recent=recent)
    c.check([n // 4 for n in lens], sinks=sinks, recent=recent, shared=[0, 5, 2, 17, 250, -3])
    c.close()


@pytest.mark.parametrize("values", ["equal", "few", "zeros", "nan", "extreme"])
def test_ties_and_odd_values(values):
    """Equal scores, both zeros, NaN, infinities, subnormals."""
    rng = np.random.default_rng(3)
    make = dict(equal=lambda n: np.full(n, 0.25), few=lambda n: rng.integers(0, 3, n) / 7.0,
                zeros=lambda n: np.where(rng.random(n) < 0.5, 0.0, -0.0), nan=lambda n: np.where(rng.random(n) < 0.5, np.nan, -np.inf),
                extreme=lambda n: rng.choice([np.inf, -np.inf, np.nan, -np.nan, 1e-45, -1e-45, 0.0, -0.0, 3e38, 1.0, np.nextafter(np.float32(1), 2)], n))
    c = Cut(rng, [10, 700, 1500, 64], scores=lambda n: make[values](n))
    for share in (0.1, 0.5, 0.9):
        c.check([int(share * n) for n in (10, 700, 1500, 64)], sinks=1, recent=2)
    c.close()


@pytest.mark.parametrize("hint", [1, 40000, 1 << 20])
def test_long_requests_over_several_sms(hint):
    """Longer than the keys that one CTA holds; the hint is wrong in both directions."""
    rng = np.random.default_rng(4)
    lens = [70000, 3, 40000, 0, 1000]
    c = Cut(rng, lens, [60000, 3, 40000, 0, 900], scores=lambda n: np.exp(2.5 * rng.standard_normal(n)).round(2))
    c.check([20000, 1, 39999, 0, 100], sinks=4, recent=64, hint=hint)
    c.check([0, 0, 0, 0, 0], hint=hint)
    c.check([59999, 2, 1, 4, 899], shared=[50000, 0, 0, 0, 3], hint=hint)
    c.close()


def test_many_requests():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 90, 3000).tolist()
    c = Cut(rng, lens, [n - n // 4 for n in lens], max_requests=3100)
    c.check([n // 2 for n in lens], sinks=2, recent=3)
    c.close()


def test_no_requests():
    c = Cut(np.random.default_rng(6), [], max_requests=4)
    assert c.run([]) == []
    c.close()


def test_victims_beyond_the_list_are_dropped():
    rng = np.random.default_rng(7)
    c = Cut(rng, [100, 200, 50])
    budget = [10, 20, 30]
    ref = c.reference(budget)
    for cap in (0, 1, 100, len(ref) - 1):
        assert c.run(budget, max_victims=cap) == ref[:cap]
        assert vt.vtoken_read_counts(c.ctx)["error_flags"] == vt.FLAG_CAPACITY
    assert c.run(budget, max_victims=len(ref)) == ref
    c.close()


def test_ids_outside_the_table_are_flagged():
    rng = np.random.default_rng(8)
    c = Cut(rng, [50, 60])
    c.dev["cache_ids"][int(c.offsets[1]) + 30] = 1 << 20
    c.ids[1][30] = 0                                         # (any score; the entry counts as NaN below)
    got = c.run([50, 59])
    assert got == [(1, 1 << 20)]
    c.close(flags=vt.FLAG_BAD_VICTIM)


def test_victims_feed_the_eviction():
    """The list goes straight to vtoken_evict_tokens."""
    import torch
    rng = np.random.default_rng(9)
    c = Cut(rng, [300, 40, 500], [200, 40, 450])
    ref = c.check([100, 10, 440], sinks=3, recent=5)
    keep = torch.zeros(c.T, dtype=torch.uint8, device="cuda:0")
    for r in range(3):
        keep[up(c.offsets[r] + c.ids[r], np.int64)] = 1
    vt.vtoken_evict_tokens(c.ctx, num_victims=c.num, max_victims=c.T, victim_req=c.req, victim_tok=c.tok,
                           num_requests=c.dev["num_requests"], tt_offsets=c.dev["tt_offsets"], tt_len=up(c.lens), keep=keep)
    torch.cuda.synchronize()
    left = keep.cpu().numpy()
    assert [int(left[c.offsets[r]:c.offsets[r + 1]].sum()) for r in range(3)] == [100, 10, 440]
    assert not any(left[c.offsets[r] + t] for r, t in ref)
    c.close()


def test_select_in_a_graph_and_on_a_stream():
    import torch
    rng = np.random.default_rng(10)
    c = Cut(rng, [600, 40, 9000], [500, 40, 8000])
    budget = [100, 10, 4000]
    c.run(budget)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    scores = c.inputs[0]
    with torch.cuda.graph(graph, stream=side):
        vt.vtoken_select_victims(c.ctx, **c.dev, scores=scores, budget=c.inputs[1], max_cache_len=8000, victim_req=c.req,
                                 victim_tok=c.tok, max_victims=c.T, num_victims=c.num, stream=torch.cuda.current_stream())
    for _ in range(2):
        c.scores = rng.standard_normal(c.T).astype(np.float32)
        scores.copy_(torch.from_numpy(c.scores))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        n = int(c.num)
        assert list(zip(c.req[:n].tolist(), c.tok[:n].tolist())) == c.reference(budget)
    c.close()


def test_select_refusals():
    import torch
    c = Cut(np.random.default_rng(11), [30, 40])
    c.run([1, 1])
    good = dict(c.dev, scores=c.inputs[0], budget=c.inputs[1], max_cache_len=40, victim_req=c.req, victim_tok=c.tok, max_victims=70,
                num_victims=c.num)
    for change in (dict(num_requests=None), dict(tt_offsets=None), dict(cache_len=None), dict(scores=None), dict(budget=None),
                   dict(num_victims=None), dict(victim_req=None), dict(victim_tok=None), dict(max_victims=-1), dict(sinks=-1),
                   dict(recent=-1), dict(max_cache_len=0)):
        with pytest.raises(vt.VtokenError) as e:
            vt.vtoken_select_victims(c.ctx, **{**good, **change})
        assert e.value.code == vt.EINVAL, change
    vt.vtoken_select_victims(c.ctx, **{**good, "max_victims": 0, "victim_req": None, "victim_tok": None})
    torch.cuda.synchronize()
    assert int(c.num) == 0
    c.close(flags=vt.FLAG_CAPACITY)


# ---- verify ---------------------------------------------------------------------------------------
KINDS = {"f32": 2, "bf16": 0, "fp16": 1}


def rounded(x, kind):
    """Values of the type, as float64, and the tensor."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x.astype(np.float32))).to({"f32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[kind])
    return t.double().numpy(), t


class Drafted:
    def __init__(self, rng, drafts, vocab, kind="f32", with_q=True, pad=0, q_pad=0, shift=0, sharp=2.0, max_requests=None):
        import torch
        self.drafts, self.V, self.kind, self.R = drafts, vocab, kind, len(drafts)
        self.off = np.concatenate([[0], np.cumsum(drafts)]).astype(np.int32)
        self.D = int(self.off[-1])
        self.max_requests = max_requests or max(1, self.R)
        rows = self.D + self.max_requests

        def table(n, width):
            x = np.exp(sharp * rng.standard_normal((max(1, n), vocab)))
            x /= x.sum(1, keepdims=True)
            full = np.full((max(1, n), width), 7.0)
            full[:, :vocab] = x
            v, t = rounded(full, kind)
            flat = torch.full((t.numel() + shift,), 3.0, dtype=t.dtype)
            flat[shift:] = t.flatten()
            return v[:, :vocab].copy(), flat.to("cuda:0")
        self.p, self.p_dev = table(rows, vocab + pad)
        self.q, self.q_dev = table(self.D, vocab + q_pad) if with_q else (None, None)
        self.pad, self.q_pad, self.shift = pad, q_pad, shift
        self.x = np.zeros(self.D, np.int32)
        for i in range(self.D):
            w = self.q[i] if with_q else self.p[i + int(np.searchsorted(self.off, i, "right")) - 1]
            self.x[i] = rng.choice(vocab, p=w / w.sum())
        self.u = rng.random(self.D).astype(np.float32)
        self.w = rng.random(max(1, self.R)).astype(np.float32)
        self.first = rng.integers(0, 1000, max(1, self.R)).astype(np.int32)
        self.ctx, self.pool = context(self.max_requests, 1)

    def args(self):
        import torch
        full = lambda n: torch.full((max(1, n),), -9, dtype=torch.int32, device="cuda:0")            # noqa: E731
        self.out = dict(accepted=full(self.R), next_tokens=full(self.R), out_tokens=full(self.D + self.max_requests), victim_req=full(self.D),
                        victim_tok=full(self.D), num_victims=full(1))
        size = self.p_dev.element_size()
        off = np.concatenate([self.off, np.full(self.max_requests - self.R, self.off[-1], np.int32)])
        return dict(num_requests=up([self.R]), draft_offsets=up(off), max_drafts=self.D, draft_tokens=up(self.x) if self.D else None,
                    prob_type=KINDS[self.kind], vocab=self.V, target_probs=self.p_dev.data_ptr() + self.shift * size,
                    draft_probs=None if self.q is None else self.q_dev.data_ptr() + self.shift * size,
                    target_stride=self.V + self.pad if self.pad else 0, draft_stride=self.V + self.q_pad if self.q_pad else 0,
                    accept_random=up(self.u, np.float32) if self.D else None, sample_random=up(self.w, np.float32), first_id=up(self.first),
                    max_victims=self.D, **self.out)

    def run(self, stream=None, **changed):
        import torch
        self.held = {**self.args(), **changed}
        vt.vtoken_verify_drafts(self.ctx, **self.held, stream=stream)
        torch.cuda.synchronize()
        n = int(self.out["num_victims"])
        get = lambda k: self.out[k].cpu().numpy()                                                     # noqa: E731
        return (get("accepted")[:self.R].tolist(), get("next_tokens")[:self.R].tolist(), get("out_tokens")[:self.D + self.R].tolist(),
                list(zip(get("victim_req")[:n].tolist(), get("victim_tok")[:n].tolist())))

    def reference(self):
        clean = lambda v: np.where((v > 0) & np.isfinite(v), v, 0.0)                                  # noqa: E731
        acc, nxt, out, gone = [], [], [-1] * (self.D + self.R), []
        for r in range(self.R):
            d0, k = int(self.off[r]), self.drafts[r]
            a = k
            for i in range(k):
                x = int(self.x[d0 + i])
                inside = 0 <= x < self.V
                p = clean(self.p[d0 + r + i])[x] if inside else 0.0
                q = (clean(self.q[d0 + i])[x] if inside else 0.0) if self.q is not None else 1.0
                if not float(self.u[d0 + i]) * q < p:
                    a = i
                    break
            p = clean(self.p[d0 + r + a])
            m = p
            if a < k:
                if self.q is not None:
                    m = np.maximum(p - clean(self.q[d0 + a]), 0.0)
                else:
                    m = p.copy()
                    if 0 <= self.x[d0 + a] < self.V:
                        m[self.x[d0 + a]] = 0.0
                if m.sum() == 0:
                    m = p
            c = np.cumsum(m)
            if c[-1] == 0:
                token = -1
            else:
                over = np.nonzero(c > max(0.0, float(self.w[r])) * c[-1])[0]
                token = int(over[0]) if len(over) else int(np.nonzero(m)[0][-1])
                # the draw is nowhere so near a border that the order of a 64-bit sum could matter
                assert len(m) == 1 or np.abs(c - float(self.w[r]) * c[-1])[m > 0].min() > 1e-13 * c[-1] or self.w[r] in (0.0, 1.0)
            acc.append(a)
            nxt.append(token)
            out[d0 + r:d0 + r + a] = self.x[d0:d0 + a].tolist()
            out[d0 + r + a] = token
            gone += [(r, int(self.first[r]) + i) for i in range(a, k)]
        return acc, nxt, out, gone

    def check(self, **changed):
        got = self.run(**changed)
        assert got == self.reference()
        return got

    def close(self, flags=0):
        assert vt.vtoken_read_counts(self.ctx)["error_flags"] == flags
        vt.vtoken_destroy(self.ctx)


@pytest.mark.parametrize("kind", ["f32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 255, 4096, 4097, 33001])
@pytest.mark.parametrize("with_q", [True, False])
def test_vocabularies_and_types(kind, vocab, with_q):
    rng = np.random.default_rng(vocab)
    d = Drafted(rng, [0, 1, 4, 0, 7, 3], vocab, kind, with_q, sharp=0.5 if vocab > 5000 else 1.0)
    acc = d.check()[0]
    assert max(acc) > 0 or vocab > 1
    d.close()


@pytest.mark.parametrize("pad,q_pad,shift", [(3, 0, 0), (0, 5, 0), (8, 8, 0), (0, 0, 1), (4, 12, 8)])
def test_strides_and_alignment(pad, q_pad, shift):
    for kind in ("f32", "bf16"):
        rng = np.random.default_rng(20)
        d = Drafted(rng, [2, 5, 0], 9000, kind, pad=pad, q_pad=q_pad, shift=shift)
        d.check()
        d.close()


@pytest.mark.parametrize("drafts", [[40, 33, 32, 0], [100], [1] * 300, [0] * 50, [9, 0, 17] * 40])
@pytest.mark.parametrize("with_q", [True, False])
def test_numbers_of_drafts(drafts, with_q):
    rng = np.random.default_rng(21)
    d = Drafted(rng, drafts, 50, with_q=with_q, sharp=0.3)
    if with_q:                                               # the same distribution: most are accepted
        for r in range(d.R):
            a = int(d.off[r])
            d.p[a + r:a + r + drafts[r]] = d.q[a:a + drafts[r]]
        d.p_dev = rounded(d.p, "f32")[1].to("cuda:0")
        d.u *= 0.99
    acc = d.check()[0]
    assert not with_q or sum(acc) == d.D
    d.u = rng.random(d.D).astype(np.float32) * 0 + 0.999
    d.p[:, :] = rng.random(d.p.shape)
    d.p[:, :25] = 0
    d.p /= d.p.sum(1, keepdims=True)
    d.p, t = rounded(d.p, "f32")
    d.p_dev = t.to("cuda:0")
    d.check()
    d.close()


def test_random_numbers_at_their_ends():
    rng = np.random.default_rng(22)
    for u, w in ((0.0, 0.0), (1.0, 1.0), (0.0, 1.0), (np.float32(1 - 2.0 ** -24), np.float32(1 - 2.0 ** -24))):
        d = Drafted(rng, [3, 2, 0, 4], 6000)
        d.u[:], d.w[:] = u, w
        if w == 1.0 or w == 0.0:
            d.p[:, -5:] = 0
            d.p[:, :3] = 0
            d.p_dev = rounded(d.p, "f32")[1].to("cuda:0")
        d.check()
        d.close()
    d = Drafted(rng, [3, 1], 100)
    d.u[:] = np.nan                                          # refuses
    d.w[:] = np.nan                                          # counts as 0
    acc, nxt, _, _ = d.run()
    d.w[:] = 0
    assert (acc, nxt) == d.reference()[:2] and acc == [0, 0]
    d.close()


def test_rows_without_mass_and_odd_probabilities():
    """Zeros, NaN, infinities and negative numbers count as no mass; the same rows on both sides leave the target's row."""
    rng = np.random.default_rng(23)
    d = Drafted(rng, [2, 2, 2, 2, 1], 500)
    d.p[0:3] = 0                                             # nothing to draw from
    d.p[3] = d.q[2]                                          # nothing left over: drawn from the target's row
    d.u[2] = 1.0
    d.p[6, ::3] = np.nan
    d.p[6, 1::7] = -1.0
    d.q[4, ::5] = np.inf
    d.u[4] = 1.0
    d.x[6] = 500                                             # outside the vocabulary
    d.x[8] = -1
    d.p_dev, d.q_dev = rounded(d.p, "f32")[1].to("cuda:0"), rounded(d.q, "f32")[1].to("cuda:0")
    acc, nxt, _, _ = d.check()
    assert nxt[0] == -1 and acc[0] == 0 and acc[3] == 0 and acc[4] == 0
    d.close()


def test_a_small_surplus_is_not_lost():
    """Differences far below the probabilities: the 64-bit difference decides, not one rounded to 32 bits."""
    rng = np.random.default_rng(24)
    V = 20000
    d = Drafted(rng, [1], V)
    d.q[0] = np.float32(1.0 / V)
    d.p[0] = d.q[0]
    for i in (5, 7001, 19999):
        d.p[0, i] = np.nextafter(np.float32(d.p[0, i]), np.float32(1))
    d.u[:] = 1.0
    d.x[0] = 3
    for w, token in ((0.1, 5), (0.5, 7001), (0.9, 19999)):
        d.w[:] = w
        d.p_dev, d.q_dev = rounded(d.p, "f32")[1].to("cuda:0"), rounded(d.q, "f32")[1].to("cuda:0")
        assert d.check()[1] == [token]
    d.close()


def test_offsets_and_victims_are_clipped():
    rng = np.random.default_rng(25)
    d = Drafted(rng, [3, 4, 5], 64)
    d.u[:] = 1.0
    ref = d.reference()
    for cap in (0, 1, 7):
        acc, nxt, out, gone = d.run(max_victims=cap)
        assert (acc, nxt, out) == ref[:3] and gone == ref[3][:cap]
        assert vt.vtoken_read_counts(d.ctx)["error_flags"] == vt.FLAG_CAPACITY
    bad = d.args()
    bad["draft_offsets"] = up([0, 3, 7, 1 << 20])
    vt.vtoken_verify_drafts(d.ctx, **bad)
    assert vt.vtoken_read_counts(d.ctx)["error_flags"] == vt.FLAG_CAPACITY
    d.close()


def test_verify_without_optional_outputs_and_in_a_graph():
    import torch
    rng = np.random.default_rng(26)
    d = Drafted(rng, [3, 0, 5, 2], 12000, max_requests=9)
    ref = d.check()
    args = d.args()
    for k in ("out_tokens", "victim_req", "victim_tok", "num_victims", "first_id"):
        args[k] = None
    args["max_victims"] = 0
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        vt.vtoken_verify_drafts(d.ctx, **args, stream=torch.cuda.current_stream())
    for _ in range(2):
        d.out["accepted"].fill_(-9)
        d.out["next_tokens"].fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        assert (d.out["accepted"][:4].tolist(), d.out["next_tokens"][:4].tolist()) == ref[:2]
        args["sample_random"].copy_(up(rng.random(4), np.float32))
        d.w = args["sample_random"].cpu().numpy()
        ref = d.reference()
    d.close()


def test_sampling_alone():
    """No drafts at all: the draft arrays are not needed."""
    rng = np.random.default_rng(27)
    d = Drafted(rng, [0, 0, 0], 40000, "bf16")
    d.check(draft_offsets=None)
    d.close()


def test_verify_refusals():
    rng = np.random.default_rng(28)
    d = Drafted(rng, [3, 2], 64)
    good = d.args()
    for change in (dict(num_requests=None), dict(target_probs=None), dict(sample_random=None), dict(accepted=None), dict(next_tokens=None),
                   dict(draft_offsets=None), dict(draft_tokens=None), dict(accept_random=None), dict(prob_type=3), dict(prob_type=-1),
                   dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(max_drafts=-1), dict(target_stride=63), dict(draft_stride=1),
                   dict(first_id=None), dict(victim_req=None), dict(victim_tok=None), dict(num_victims=None), dict(max_victims=-1),
                   dict(target_probs=good["target_probs"] + 2), dict(draft_probs=good["draft_probs"] + 1)):
        with pytest.raises(vt.VtokenError) as e:
            vt.vtoken_verify_drafts(d.ctx, **{**good, **change})
        assert e.value.code == vt.EINVAL, change
    d.close()
