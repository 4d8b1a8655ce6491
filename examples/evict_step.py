"""A serving loop that evicts by attention weight, on one layer: groups of requests behind a shared prompt draft tokens, attend
(the prompt's rows are read once a group), have their drafts verified, and lose the rejected ones; every few steps each request is
cut back to a budget by the attention weight that its tokens received, and the survivors are repacked around the shared blocks.

    python examples/evict_step.py [--kv bf16|fp16|fp4] [--steps N]
"""
import argparse
import os
import sys

import torch

sys.path[:0] = [os.path.dirname(os.path.abspath(__file__)), os.path.dirname(os.path.dirname(os.path.abspath(__file__)))]
from decode_step import Decoder  # noqa: E402
from paper_2608_13263_b200 import binding as vt  # noqa: E402


class Server(Decoder):
    """The Decoder's tables for ``groups`` x ``members`` requests, each group behind a prompt of ``prompt`` tokens (whole blocks)."""

    def __init__(self, kv="bf16", groups=2, members=3, prompt=64, capacity=512, budget=120, recent=16, decay=0.9, **options):
        super().__init__(kv, requests=groups * members, capacity=capacity, window=0, sinks=0, **options)
        assert prompt % self.S == 0
        i32 = dict(dtype=torch.int32, device=self.dev)
        self.members, self.prompt, self.recent, self.decay = members, prompt, recent, decay
        self.num_groups = torch.tensor([groups], **i32)
        self.group_offsets = torch.arange(groups + 1, **i32) * members
        self.shared_len = torch.full((self.R,), prompt, **i32)
        self.budget = torch.full((self.R,), budget, **i32)
        self.protect = torch.zeros(self.NB, dtype=torch.uint8, device=self.dev)
        self.scores = torch.zeros(self.R * capacity, device=self.dev)
        self.place = torch.zeros(self.R, **i32)                 # position of each request's next token: rejected drafts have none
        self.victim_req, self.victim_tok = (torch.zeros(self.R * capacity, **i32) for _ in range(2))
        self.num_victims = torch.zeros(1, **i32)
        rows = self.R * capacity
        self.shared_bytes = vt.vtoken_attention_shared_workspace_bytes(self.ctx, self.heads, rows)
        self.weights_bytes = vt.vtoken_token_weights_workspace_bytes(self.ctx, self.heads, rows)
        self.workspace = torch.zeros(max(self.shared_bytes, self.weights_bytes), dtype=torch.uint8, device=self.dev)

    def _write(self, qkv, positions, slots):
        n, hq, hkv, d = qkv.shape[0], self.hq, self.hkv, self.d
        q, k, v = qkv[:, :hq * d], qkv[:, hq * d:(hq + hkv) * d], qkv[:, (hq + hkv) * d:]
        q_out, stride = torch.empty(n, hq, d, dtype=self.act, device=self.dev), qkv.stride(0)
        vt.vtoken_write_tokens(self.ctx, heads=self.heads, layer=0, max_tokens=n, q=q, k=k, v=v, positions=positions, slots=slots,
                               q_out=q_out, q_weight=self.q_weight, k_weight=self.k_weight, eps=1e-6, cos_sin=self.cos_sin,
                               max_position=self.cap, rot_dim=d, q_stride=stride, k_stride=stride, v_stride=stride)
        return q_out

    def prompts(self, qkv):
        """The prompts' rows, [groups * prompt, (hq + 2 hkv) * d], written once a group; every member's tables begin with them."""
        P, per = self.prompt, self.prompt // self.S
        at = torch.arange(P, dtype=torch.int32, device=self.dev)
        for g in range(self.R // self.members):
            first = g * self.members
            blocks = self.blocks[first][:per]
            slots = torch.tensor(blocks, dtype=torch.int32, device=self.dev)[(at // self.S).long()] * self.S + at % self.S
            self._write(qkv[g * P:(g + 1) * P], at, slots)
            self.protect[blocks] = 1
            for r in range(first, first + self.members):
                if r != first:                                  # its own first blocks go back
                    self.free += self.blocks[r][:per]
                    self.blocks[r] = blocks + self.blocks[r][per:]
                self.tt_slots[r * self.cap:r * self.cap + P] = slots
                self.keep[r * self.cap:r * self.cap + P] = 1
        self.tt_len.fill_(P)
        self.phys_len.fill_(P)
        self.place.fill_(P)
        self._tables()

    def step(self, qkv, n):
        """``n`` new tokens of every request (one and its drafts): attention, and the weight that every cached token received."""
        ids = (self.tt_len.unsqueeze(1) + torch.arange(n, device=self.dev, dtype=torch.int32)).reshape(-1).contiguous()
        places = (self.place.unsqueeze(1) + torch.arange(n, device=self.dev, dtype=torch.int32)).reshape(-1).contiguous()
        vt.vtoken_sync_new_tokens(self.ctx, num_requests=self.num_requests, tt_offsets=self.tt_offsets, tt_slots=self.tt_slots,
                                  keep=self.keep, tt_len=self.tt_len, phys_len=self.phys_len, bt_offsets=self.bt_offsets,
                                  bt_blocks=self.bt_blocks, new_len=self.tt_len + n)
        entry = (self.tt_offsets[:-1].unsqueeze(1) + ids.view(self.R, n)).reshape(-1).long()
        q = self._write(qkv, places, self.tt_slots[entry].contiguous())
        vt.vtoken_slot_cache_update(self.ctx, num_requests=self.num_requests, tt_offsets=self.tt_offsets, tt_slots=self.tt_slots,
                                    keep=self.keep, tt_len=self.tt_len, dirty=self.dirty, cache_slots=self.cache_slots,
                                    cache_ids=self.cache_ids, cache_len=self.cache_len, cache_seen=self.cache_seen)
        out, lse = torch.empty_like(q), torch.empty(self.R * n, self.hq, device=self.dev)
        common = dict(heads=self.heads, layer=0, num_requests=self.num_requests, positions=ids, q=q, max_query_tokens=self.R * n,
                      q_offsets=torch.arange(self.R + 1, dtype=torch.int32, device=self.dev) * n, max_query_len=n,
                      tt_offsets=self.tt_offsets, cache_slots=self.cache_slots, cache_ids=self.cache_ids, cache_len=self.cache_len,
                      lse=lse, sm_scale=self.d ** -0.5, workspace=self.workspace)
        vt.vtoken_attention_shared(self.ctx, out=out, num_groups=self.num_groups, group_offsets=self.group_offsets,
                                   shared_len=self.shared_len, workspace_bytes=self.shared_bytes, **common)
        vt.vtoken_token_weights(self.ctx, decay=self.decay, prev=self.scores, scores=self.scores, workspace_bytes=self.weights_bytes,
                                **common)
        return out, lse

    def verify(self, drafts, target, draft, accept, sample):
        """The last step's n - 1 drafts, [R, n - 1], against target [R, n, vocab] and draft [R, n - 1, vocab] probabilities: the rejected
        ones leave the cache.  Returns accepted [R], the next tokens [R]."""
        i32 = dict(dtype=torch.int32, device=self.dev)
        R, k = drafts.shape
        accepted, tokens = torch.zeros(R, **i32), torch.zeros(R, **i32)
        vt.vtoken_verify_drafts(self.ctx, num_requests=self.num_requests, draft_offsets=torch.arange(R + 1, **i32) * k, max_drafts=R * k,
                                draft_tokens=drafts, prob_type=vt.PROB_F32, vocab=target.shape[-1], target_probs=target,
                                draft_probs=draft, accept_random=accept, sample_random=sample, first_id=self.tt_len - k,
                                accepted=accepted, next_tokens=tokens, victim_req=self.victim_req, victim_tok=self.victim_tok,
                                max_victims=R * k, num_victims=self.num_victims)
        self._evict(R * k)
        self.place += 1 + accepted
        return accepted, tokens

    def cut_back(self):
        """Every request back to its budget by the weight its tokens received; the survivors are packed around the shared blocks."""
        vt.vtoken_slot_cache_update(self.ctx, num_requests=self.num_requests, tt_offsets=self.tt_offsets, tt_slots=self.tt_slots,
                                    keep=self.keep, tt_len=self.tt_len, dirty=self.dirty, cache_slots=self.cache_slots,
                                    cache_ids=self.cache_ids, cache_len=self.cache_len, cache_seen=self.cache_seen)
        most = self.victim_req.shape[0]
        vt.vtoken_select_victims(self.ctx, num_requests=self.num_requests, tt_offsets=self.tt_offsets, cache_ids=self.cache_ids,
                                 cache_len=self.cache_len, scores=self.scores, budget=self.budget, shared_len=self.shared_len,
                                 recent=self.recent, max_cache_len=self.cap, victim_req=self.victim_req, victim_tok=self.victim_tok,
                                 max_victims=most, num_victims=self.num_victims)
        self._evict(most)
        self._repack()

    def _evict(self, most):
        victims = dict(num_victims=self.num_victims, max_victims=most, victim_req=self.victim_req, num_requests=self.num_requests)
        vt.vtoken_evict_tokens(self.ctx, victim_tok=self.victim_tok, tt_offsets=self.tt_offsets, tt_len=self.tt_len, keep=self.keep, **victims)
        vt.vtoken_slot_cache_mark(self.ctx, dirty=self.dirty, **victims)

    def _repack(self):
        i32 = dict(dtype=torch.int32, device=self.dev)
        total = sum(len(b) for b in self.blocks)
        new = dict(new_bt_offsets=torch.zeros(self.R + 1, **i32), new_bt_blocks=torch.zeros(total, **i32),
                   new_tt_slots=torch.zeros_like(self.tt_slots), freed_blocks=torch.zeros(total, **i32),
                   req_status=torch.zeros(self.R, **i32), counts=torch.zeros(8, **i32))
        free = torch.zeros(self.NB, **i32)
        free[:len(self.free)] = torch.tensor(self.free, **i32)
        vt.vtoken_plan_partial(self.ctx, num_requests=self.num_requests, bt_offsets=self.bt_offsets, bt_blocks=self.bt_blocks,
                               tt_offsets=self.tt_offsets, tt_slots=self.tt_slots, keep=self.keep, free_blocks=free,
                               num_free=torch.tensor([len(self.free)], **i32), protect=self.protect, util=(1, 1), **new)
        vt.vtoken_repack(self.ctx)
        vt.vtoken_apply_moves(self.ctx, num_requests=self.num_requests, tt_offsets=self.tt_offsets, tt_slots=self.tt_slots,
                              keep=self.keep, phys_len=self.phys_len, new_tt_slots=new["new_tt_slots"],
                              req_status=new["req_status"], new_bt_offsets=new["new_bt_offsets"])
        vt.vtoken_slot_cache_mark(self.ctx, dirty=self.dirty, req_status=new["req_status"], num_requests=self.num_requests)
        counts = vt.vtoken_read_counts(self.ctx)
        self.flags = counts["error_flags"]
        off, blocks = new["new_bt_offsets"].tolist(), new["new_bt_blocks"].tolist()
        self.free = self.free[counts["num_free_consumed"]:] + new["freed_blocks"].tolist()[:counts["num_freed"]]
        self.blocks = [blocks[off[r]:off[r + 1]] for r in range(self.R)]
        for b in self.blocks:                       # room for the tokens to come
            while len(b) < self.cap // self.S and self.free:
                b.append(self.free.pop(0))
        self._tables()

    def _tables(self):
        i32 = dict(dtype=torch.int32, device=self.dev)
        off = [0]
        for b in self.blocks:
            off.append(off[-1] + len(b))
        self.bt_offsets = torch.tensor(off, **i32)
        self.bt_blocks = torch.tensor([x for b in self.blocks for x in b], **i32)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--kv", choices=("bf16", "fp16", "fp4"), default="bf16")
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    server, vocab, drafts = Server(a.kv), 1000, 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    width = (server.hq + 2 * server.hkv) * server.d
    draw = lambda n: torch.randn(n, width, generator=gen, device="cuda").to(server.act)      # noqa: E731
    server.prompts(draw(2 * server.prompt))
    taken = 0
    for i in range(a.steps):
        server.step(draw(server.R * (drafts + 1)), drafts + 1)
        target = torch.softmax(2 * torch.randn(server.R, drafts + 1, vocab, generator=gen, device="cuda"), -1)
        draft = torch.softmax(torch.log(target[:, :drafts]) + 0.5 * torch.randn(server.R, drafts, vocab, generator=gen, device="cuda"), -1)
        tokens = torch.multinomial(draft.view(-1, vocab), 1, generator=gen).view(server.R, drafts).to(torch.int32)
        accepted, _ = server.verify(tokens, target, draft.contiguous(), torch.rand(server.R * drafts, generator=gen, device="cuda"),
                                    torch.rand(server.R, generator=gen, device="cuda"))
        taken += int(accepted.sum())
        if i % 20 == 19:
            server.cut_back()
    flags = vt.vtoken_read_counts(server.ctx)["error_flags"]
    print(f"{a.kv}: {a.steps} steps of {server.R} requests, {taken} drafts accepted, {int(server.cache_len.sum())} tokens cached, flags {flags}")
    server.close()


if __name__ == "__main__":
    main()
