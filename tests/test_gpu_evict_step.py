"""The serving loop of examples/evict_step.py: shared prompts, drafted steps, scores, verification, eviction to a budget and repacks
together, against a plain copy of what its caches have to hold, in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest

import attention_sim as sim
from test_gpu_decode_step import turned

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load_example():
    spec = importlib.util.spec_from_file_location("evict_step", os.path.join(ROOT, "examples", "evict_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("kv", ["bf16", "fp16", "fp4"])
def test_the_loop_keeps_its_books(kv):
    import torch
    from paper_2608_13263_b200 import binding as vt
    s = load_example().Server(kv, groups=2, members=3, prompt=48, capacity=320, budget=90, recent=8)
    act = "fp16" if kv == "fp16" else "bf16"
    rng = np.random.default_rng(3)
    R, hq, hkv, d, u, vocab = s.R, s.hq, s.hkv, s.d, sim.unit(act), 50
    qw, kw, cs = sim.to64(s.q_weight), sim.to64(s.k_weight), s.cos_sin.cpu().double().numpy()
    alive = [dict() for _ in range(R)]                          # per request: id -> key, value
    score = [dict() for _ in range(R)]
    real = [s.prompt] * R

    def rows(x, pos):
        k, v = sim.round16(turned(x[:, hq:hq + hkv], kw, pos, cs), act), x[:, hq + hkv:]
        return [sim.dequantise_rows(sim.quantise_rows(y), hkv, d) for y in (k, v)] if kv == "fp4" else [k, v]

    def draw(n):
        qkv = torch.from_numpy(rng.standard_normal((n, (hq + 2 * hkv) * d))).to(s.dev).to(s.act)
        return qkv, sim.to64(qkv).reshape(n, hq + 2 * hkv, d)
    qkv, x = draw(2 * s.prompt)
    s.prompts(qkv)
    for r in range(R):
        g = r // s.members
        k, v = rows(x[g * s.prompt:(g + 1) * s.prompt], np.arange(s.prompt))
        alive[r] = {i: (k[i], v[i]) for i in range(s.prompt)}
        score[r] = {i: 0.0 for i in range(s.prompt)}
    next_id = [s.prompt] * R
    for step in range(36):
        n = [1, 4, 3, 2][step % 4]
        qkv, x = draw(R * n)
        out, lse = s.step(qkv, n)
        got, x = sim.to64(out), x.reshape(R, n, hq + 2 * hkv, d)
        for r in range(R):
            pos = real[r] + np.arange(n)
            q = turned(x[r, :, :hq], qw, pos, cs)
            k, v = rows(x[r], pos)
            for t in range(n):
                alive[r][next_id[r] + t] = (k[t], v[t])
                score[r][next_id[r] + t] = 0.0
            new = dict.fromkeys(alive[r], 0.0)
            for t in range(n):
                seen = [i for i in alive[r] if i <= next_id[r] + t]
                K, V = (np.repeat(np.stack([alive[r][i][j] for i in seen]), hq // hkv, 1) for j in (0, 1))
                sc = np.einsum("hd,lhd->hl", q[t], K) * d ** -0.5
                w = np.exp(sc - sc.max(-1, keepdims=True))
                w /= w.sum(-1, keepdims=True)
                ref = np.einsum("hl,lhd->hd", w, V)
                # as in the loop without sharing: one rounding of queries and keys, of weights and output
                ds = (2.1 * u * np.einsum("hd,lhd->hl", np.abs(q[t]), np.abs(K)) * d ** -0.5).max(-1)
                tol = 1.01 * u * np.abs(ref) + (u + np.expm1(2 * ds)[:, None] + 1e-5) * np.abs(V).max(0)
                assert (np.abs(got[r * n + t] - ref) <= tol).all(), (step, r, t)
                for i, y in zip(seen, w.sum(0)):
                    new[i] += y
                worst = np.expm1(2 * ds.max()) + 1e-4            # relative, of every weight
            for i in new:
                score[r][i] = s.decay * score[r][i] + new[i]
            next_id[r] += n
        have = s.scores.cpu().double().numpy().reshape(R, s.cap)
        for r in range(R):
            for i, y in score[r].items():
                assert abs(have[r, i] - y) <= 3 * worst * y + 1e-6, (step, r, i)
                score[r][i] = have[r, i]                         # (so that errors do not pile up)
        if n > 1:                                                # the drafts behind the first token
            k = n - 1
            target = rng.random((R, n, vocab)) ** 4
            target /= target.sum(-1, keepdims=True)
            draft = rng.random((R, k, vocab)) ** 4
            draft /= draft.sum(-1, keepdims=True)
            t32, d32 = target.astype(np.float32), draft.astype(np.float32)
            tokens = rng.integers(0, vocab, (R, k)).astype(np.int32)
            accept, sample = rng.random(R * k).astype(np.float32), rng.random(R).astype(np.float32)
            up = lambda a: torch.from_numpy(a).to(s.dev)                                      # noqa: E731
            accepted, _ = s.verify(up(tokens), up(t32), up(d32), up(accept), up(sample))
            for r in range(R):
                a = 0
                while a < k and np.float64(accept[r * k + a]) * np.float64(d32[r, a, tokens[r, a]]) < np.float64(t32[r, a, tokens[r, a]]):
                    a += 1
                assert int(accepted[r]) == a
                for i in range(next_id[r] - (k - a), next_id[r]):
                    del alive[r][i], score[r][i]
                real[r] += 1 + a
        else:
            s.place += 1
            real = [p + 1 for p in real]
        if step % 12 == 11:
            s.cut_back()
            for r in range(R):
                order = sorted(alive[r])
                free = [i for e, i in enumerate(order) if e >= s.prompt and e < len(order) - s.recent]
                gone = sorted(free, key=lambda i: (np.float32(score[r][i]), -i))[:max(0, len(order) - 90)]
                for i in gone:
                    del alive[r][i], score[r][i]
            assert s.flags == 0
            left = s.keep.cpu().numpy().reshape(R, s.cap)
            for r in range(R):
                assert np.nonzero(left[r])[0].tolist() == sorted(alive[r])
    assert vt.vtoken_read_counts(s.ctx)["error_flags"] == 0
    assert int(s.cache_len.max()) <= 90 + 30
    s.close()
