"""The example's serving loop (append, write, attention, eviction, repack) against the same attention without a cache: every
step's output is compared with softmax over the window's tokens, computed in 64 bits from what the cache has to hold."""
import importlib.util
import os

import numpy as np
import pytest

import attention_sim as sim

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load_example():
    spec = importlib.util.spec_from_file_location("decode_step", os.path.join(ROOT, "examples", "decode_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def turned(x, weight, positions, cos_sin):
    x = x / np.sqrt((x * x).mean(-1, keepdims=True) + np.float64(np.float32(1e-6))) * weight
    h = x.shape[-1] // 2
    c, s = cos_sin[positions][:, None, :h], cos_sin[positions][:, None, h:]
    return np.concatenate([x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s], -1)


@pytest.mark.parametrize("kv", ["bf16", "fp16", "fp4"])
def test_steps_with_evictions_and_repacks(kv):
    import torch
    from paper_2608_13263_b200 import binding as vt
    dec = load_example().Decoder(kv, requests=3, capacity=256, hq=8, hkv=2, d=128, window=40, sinks=4)
    act = "fp16" if kv == "fp16" else "bf16"
    rng = np.random.default_rng(3)
    hq, hkv, d = dec.hq, dec.hkv, dec.d
    keys, values = [[] for _ in range(dec.R)], [[] for _ in range(dec.R)]
    qw, kw, cs = sim.to64(dec.q_weight), sim.to64(dec.k_weight), dec.cos_sin.cpu().double().numpy()
    u = sim.unit(act)
    for i, n in enumerate([90] + [1] * 30 + [3] * 5 + [1] * 10):
        qkv = torch.from_numpy(rng.standard_normal((dec.R * n, (hq + 2 * hkv) * d))).to(dec.dev).to(dec.act)
        out, _ = dec.step(qkv, n)
        got, x = sim.to64(out), sim.to64(qkv).reshape(dec.R, n, hq + 2 * hkv, d)
        for r in range(dec.R):
            pos = np.arange(len(keys[r]), len(keys[r]) + n)
            q = turned(x[r, :, :hq], qw, pos, cs)
            k = sim.round16(turned(x[r, :, hq:hq + hkv], kw, pos, cs), act)
            v = x[r, :, hq + hkv:]
            if kv == "fp4":
                k, v = (sim.dequantise_rows(sim.quantise_rows(y), hkv, d) for y in (k, v))
            keys[r] += list(k)
            values[r] += list(v)
            for t in range(n):
                p = int(pos[t])
                seen = [j for j in range(p + 1) if j > p - dec.window or j < dec.sinks]
                K, V = (np.repeat(np.stack([y[r][j] for j in seen]), hq // hkv, 1) for y in (keys, values))
                s = np.einsum("hd,lhd->hl", q[t], K) * d ** -0.5
                w = np.exp(s - s.max(-1, keepdims=True))
                w /= w.sum(-1, keepdims=True)
                ref = np.einsum("hl,lhd->hd", w, V)
                # queries and keys carry one 16-bit rounding each: the scores are off by 2 u sum |q k| scale at most, the weights by
                # twice that; then weights and output are rounded once
                ds = (2.1 * u * np.einsum("hd,lhd->hl", np.abs(q[t]), np.abs(K)) * d ** -0.5).max(-1)
                tol = 1.01 * u * np.abs(ref) + (u + np.expm1(2 * ds)[:, None] + 1e-5) * np.abs(V).max(0)
                assert (np.abs(got[r * n + t] - ref) <= tol).all(), (i, r, t)
        if i % 12 == 11:
            dec.evict_and_repack()
    assert vt.vtoken_read_counts(dec.ctx)["error_flags"] == 0
    assert int(dec.cache_len.sum()) < dec.R * 100
    dec.close()
