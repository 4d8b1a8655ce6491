"""Decode steps over a token-evicted paged KV cache, on one layer: every step the new tokens get slots, their projections are
normalised, rotated and written into the cache, the queries attend through the cached slot arrays; in between the oldest tokens
of the window are evicted and the survivors repacked.

    python examples/decode_step.py [--kv bf16|fp16|fp4] [--steps N]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_13263_b200 import binding as vt  # noqa: E402


class Decoder:
    """One layer's cache of ``requests`` sequences with the tables and buffers a serving loop keeps on the device."""

    def __init__(self, kv="bf16", requests=4, capacity=512, hq=8, hkv=2, d=128, block=16, window=64, sinks=4, seed=0):
        self.act = torch.float16 if kv == "fp16" else torch.bfloat16
        act_kind = vt.KV_FP16 if kv == "fp16" else vt.KV_BF16
        kind = {"bf16": vt.KV_BF16, "fp16": vt.KV_FP16, "fp4": vt.KV_FP4}[kv]
        self.R, self.cap, self.hq, self.hkv, self.d, self.S = requests, capacity, hq, hkv, d, block
        self.window, self.sinks = window, sinks
        self.heads = vt.Heads(hq, hkv, d, kind, act_kind, 0, 0)
        row = vt.vtoken_kv_row_bytes(self.heads)
        per = capacity // block
        self.NB = 2 * requests * per
        dev = self.dev = torch.device("cuda:0")
        i32 = dict(dtype=torch.int32, device=dev)
        self.k_pool = torch.zeros(1, self.NB * block, row, dtype=torch.uint8, device=dev)
        self.v_pool = torch.zeros_like(self.k_pool)
        # rows are bytes to the relocation, whatever they hold
        self.ctx = vt.vtoken_create(1, self.NB, block, 1, row, self.k_pool, self.v_pool, requests, requests * capacity,
                                    self.NB, self.NB, elem_bytes=1)
        self.num_requests = torch.tensor([requests], **i32)
        self.tt_offsets = torch.arange(requests + 1, **i32) * capacity
        self.tt_slots = torch.full((requests * capacity,), -1, **i32)
        self.keep = torch.zeros(requests * capacity, dtype=torch.uint8, device=dev)
        self.tt_len, self.phys_len = torch.zeros(requests, **i32), torch.zeros(requests, **i32)
        self.blocks = [list(range(r * per, (r + 1) * per)) for r in range(requests)]
        self.free = list(range(requests * per, self.NB))
        self.dirty = torch.zeros(requests, dtype=torch.uint8, device=dev)
        self.cache_slots, self.cache_ids = torch.full_like(self.tt_slots, -1), torch.full_like(self.tt_slots, -1)
        self.cache_len, self.cache_seen = torch.zeros(requests, **i32), torch.zeros(requests, **i32)
        angle = torch.outer(torch.arange(capacity, device=dev, dtype=torch.float64),
                            10000.0 ** (-torch.arange(d // 2, device=dev, dtype=torch.float64) / (d // 2)))
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
        gen = torch.Generator(device=dev).manual_seed(seed)
        self.q_weight = (1 + 0.1 * torch.randn(d, generator=gen, device=dev)).to(self.act)
        self.k_weight = (1 + 0.1 * torch.randn(d, generator=gen, device=dev)).to(self.act)
        self.workspace_bytes = vt.vtoken_attention_workspace_bytes(self.ctx, self.heads, requests * capacity)
        self.workspace = torch.zeros(self.workspace_bytes, dtype=torch.uint8, device=dev)
        self._tables()

    def _tables(self):
        i32 = dict(dtype=torch.int32, device=self.dev)
        off = [0]
        for b in self.blocks:
            off.append(off[-1] + len(b))
        self.bt_offsets = torch.tensor(off, **i32)
        self.bt_blocks = torch.zeros(self.NB, **i32)
        self.bt_blocks[:off[-1]] = torch.tensor([x for b in self.blocks for x in b], **i32)

    def step(self, qkv, n):
        """``n`` new tokens of every request; qkv: [R * n, (hq + 2 hkv) * d].  Returns [R * n, hq, d] and the lse."""
        R, hq, hkv, d = self.R, self.hq, self.hkv, self.d
        first = self.tt_len.clone()
        new_len = self.tt_len + n
        vt.vtoken_sync_new_tokens(self.ctx, num_requests=self.num_requests, tt_offsets=self.tt_offsets, tt_slots=self.tt_slots,
                                  keep=self.keep, tt_len=self.tt_len, phys_len=self.phys_len, bt_offsets=self.bt_offsets,
                                  bt_blocks=self.bt_blocks, new_len=new_len)
        positions = (first.unsqueeze(1) + torch.arange(n, device=self.dev, dtype=torch.int32)).reshape(-1).contiguous()
        entry = (self.tt_offsets[:-1].unsqueeze(1) + positions.view(R, n)).reshape(-1).long()
        q, k, v = qkv[:, :hq * d], qkv[:, hq * d:(hq + hkv) * d], qkv[:, (hq + hkv) * d:]
        q_out = torch.empty(R * n, hq, d, dtype=self.act, device=self.dev)
        stride = qkv.stride(0)
        vt.vtoken_write_tokens(self.ctx, heads=self.heads, layer=0, max_tokens=R * n, q=q, k=k, v=v, positions=positions,
                               slots=self.tt_slots[entry].contiguous(), q_out=q_out, q_weight=self.q_weight, k_weight=self.k_weight,
                               eps=1e-6, cos_sin=self.cos_sin, max_position=self.cap, rot_dim=d, q_stride=stride, k_stride=stride,
                               v_stride=stride)
        vt.vtoken_slot_cache_update(self.ctx, num_requests=self.num_requests, tt_offsets=self.tt_offsets, tt_slots=self.tt_slots,
                                    keep=self.keep, tt_len=self.tt_len, dirty=self.dirty, cache_slots=self.cache_slots,
                                    cache_ids=self.cache_ids, cache_len=self.cache_len, cache_seen=self.cache_seen)
        out = torch.empty_like(q_out)
        lse = torch.empty(R * n, hq, dtype=torch.float32, device=self.dev)
        vt.vtoken_attention(self.ctx, heads=self.heads, layer=0, num_requests=self.num_requests,
                            q_offsets=torch.arange(R + 1, dtype=torch.int32, device=self.dev) * n, positions=positions, q=q_out,
                            max_query_tokens=R * n, max_query_len=n, tt_offsets=self.tt_offsets, cache_slots=self.cache_slots,
                            cache_ids=self.cache_ids, cache_len=self.cache_len, out=out, lse=lse, sm_scale=d ** -0.5,
                            window=self.window, sinks=self.sinks, workspace=self.workspace, workspace_bytes=self.workspace_bytes)
        return out, lse

    def evict_and_repack(self):
        """Tokens that the window has passed leave the cache (all but the first ones); the survivors are packed."""
        i32 = dict(dtype=torch.int32, device=self.dev)
        req, tok = [], []
        for r, n in enumerate(self.tt_len.tolist()):
            gone = range(self.sinks, max(self.sinks, n - self.window))
            req += [r] * len(gone)
            tok += list(gone)
        if not req:
            return
        victims = dict(num_victims=torch.tensor([len(req)], **i32), max_victims=len(req), victim_req=torch.tensor(req, **i32))
        vt.vtoken_evict_tokens(self.ctx, victim_tok=torch.tensor(tok, **i32), num_requests=self.num_requests,
                               tt_offsets=self.tt_offsets, tt_len=self.tt_len, keep=self.keep, **victims)
        vt.vtoken_slot_cache_mark(self.ctx, dirty=self.dirty, num_requests=self.num_requests, **victims)
        new = dict(new_bt_offsets=torch.zeros(self.R + 1, **i32), new_bt_blocks=torch.zeros(self.NB, **i32),
                   new_tt_slots=torch.zeros_like(self.tt_slots), freed_blocks=torch.zeros(self.NB, **i32),
                   req_status=torch.zeros(self.R, **i32), counts=torch.zeros(8, **i32))
        free = torch.zeros(self.NB, **i32)
        free[:len(self.free)] = torch.tensor(self.free, **i32)
        vt.vtoken_plan(self.ctx, num_requests=self.num_requests, bt_offsets=self.bt_offsets, bt_blocks=self.bt_blocks,
                       tt_offsets=self.tt_offsets, tt_slots=self.tt_slots, keep=self.keep, free_blocks=free,
                       num_free=torch.tensor([len(self.free)], **i32), **new)
        vt.vtoken_repack(self.ctx)
        vt.vtoken_apply_moves(self.ctx, num_requests=self.num_requests, tt_offsets=self.tt_offsets, tt_slots=self.tt_slots,
                              keep=self.keep, phys_len=self.phys_len, new_tt_slots=new["new_tt_slots"],
                              req_status=new["req_status"], new_bt_offsets=new["new_bt_offsets"])
        vt.vtoken_slot_cache_mark(self.ctx, dirty=self.dirty, req_status=new["req_status"], num_requests=self.num_requests)
        counts = vt.vtoken_read_counts(self.ctx)
        off, blocks = new["new_bt_offsets"].tolist(), new["new_bt_blocks"].tolist()
        self.free = self.free[counts["num_free_consumed"]:] + new["freed_blocks"].tolist()[:counts["num_freed"]]
        self.blocks = [blocks[off[r]:off[r + 1]] for r in range(self.R)]
        for b in self.blocks:                       # room for the tokens to come
            while len(b) < self.cap // self.S and self.free:
                b.append(self.free.pop(0))
        self._tables()

    def close(self):
        vt.vtoken_destroy(self.ctx)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--kv", choices=("bf16", "fp16", "fp4"), default="bf16")
    ap.add_argument("--steps", type=int, default=100)
    a = ap.parse_args()
    dec = Decoder(a.kv)
    gen = torch.Generator(device="cuda").manual_seed(1)
    width = (dec.hq + 2 * dec.hkv) * dec.d
    draw = lambda n: torch.randn(dec.R * n, width, generator=gen, device="cuda").to(dec.act)     # noqa: E731
    out, _ = dec.step(draw(100), 100)               # the prompts
    for i in range(a.steps):
        out, lse = dec.step(draw(1), 1)
        if i % 20 == 19:
            dec.evict_and_repack()
    flags = vt.vtoken_read_counts(dec.ctx)["error_flags"]
    print(f"{a.kv}: {a.steps} steps of {dec.R} requests, {int(dec.cache_len.sum())} tokens cached, "
          f"mean lse {float(lse.mean()):.3f}, flags {flags}")
    dec.close()


if __name__ == "__main__":
    main()
