"""Drafted decoding of a batch of uneven requests over a paged 8-bit KV cache.

One layer of random weights (what it says means nothing) run as a server would run a
model.  The draft is the model itself as a set block decoder: one block forward over the
last token and k masks gives k marginals, a token is drawn from each of them, and the next
forward checks the drawn ones against the model's own next-token distribution, so that
what comes out is distributed as plain next-token decoding.  A turn is

    sbd_linear, sbd_qk_norm_rope            the rows' queries, keys and values
    sbd_block_attention_q8                  the block: the last token and k masks
    sbd_linear                              the head; drawn: the drafted tokens
    (the same projections)                  the last token and the drafted ones
    sbd_tree_attention_q8                   each sees the cache, itself and its ancestors
    sbd_linear, sbd_verify_tree             how many of them hold, and the token after them
    sbd_block_tables, sbd_cache_append_path_q8
                                            pages and slots for those, keys and values into them

    python examples/drafted_decode.py --requests 16 --turns 8
"""
from __future__ import annotations

import argparse
import os
import sys
import time

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2509_04185_gb300 as sbd  # noqa: E402


class DraftedDecoder:
    def __init__(self, requests, n_pages, max_pages, *, page=64, k=7, q_heads=8, kv_heads=2, head_dim=128, hidden=256,
                 vocab=2000, tau=1.0, seed=0):
        self.B, self.page, self.k, self.tau = requests, page, k, tau
        self.heads, self.vocab, self.turns = (q_heads, kv_heads, head_dim), vocab, 0
        self.gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, generator=self.gen, device="cuda") * shape[-1] ** -0.5).bfloat16()

        self.embed = torch.randn((vocab + 1, hidden), generator=self.gen, device="cuda").bfloat16()   # the last: a mask
        self.w_qkv = weight((q_heads + 2 * kv_heads) * head_dim, hidden)
        self.w_out, self.w_head = weight(hidden, q_heads * head_dim), weight(vocab, hidden)
        self.q_norm, self.k_norm = (1 + 0.1 * weight(2, head_dim)).unbind()
        half = torch.arange(head_dim // 2, dtype=torch.float64, device="cuda") / (head_dim // 2)
        self.inv_freq = (1e4 ** -half).float()
        self.cache = [torch.zeros(n_pages, kv_heads, page, head_dim, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
        self.scale = [torch.zeros(n_pages, kv_heads, device="cuda") for _ in range(2)]
        self.table = torch.full((requests, max_pages), -1, dtype=torch.int32, device="cuda")
        self.free = torch.arange(n_pages, dtype=torch.int32, device="cuda")
        self.n_free = torch.full((1,), n_pages, dtype=torch.int32, device="cuda")
        self.length = torch.zeros(requests, dtype=torch.int32, device="cuda")     # tokens in the cache
        self.last = torch.zeros(requests, dtype=torch.int32, device="cuda")       # the last token, not in the cache yet
        self.chain = torch.arange(-1, k, dtype=torch.int32, device="cuda").repeat(requests, 1)

    def _linear(self, x, w):
        flat = x.reshape(-1, x.shape[-1])
        y = torch.cat([sbd.sbd_linear(flat[i:i + 512], w) for i in range(0, len(flat), 512)])
        return y.view(*x.shape[:-1], len(w))

    def _project(self, tokens, positions):
        """Hidden rows, and queries, keys and values of tokens [.., n] at their positions."""
        q, kv, d = self.heads
        x = self.embed[tokens.long()]
        y = self._linear(x, self.w_qkv).view(*tokens.shape, q + 2 * kv, d)
        return x, sbd.sbd_qk_norm_rope(y[..., :q, :], y[..., q:q + kv, :], y[..., q + kv:, :], positions, self.inv_freq,
                                       self.q_norm, self.k_norm)

    def _logits(self, x, out):
        return self._linear(x + self._linear(out.flatten(2), self.w_out), self.w_head)

    def admit(self, prompts):
        """Takes in a prompt [n] int32 for every request: all but its last token enter the cache."""
        lens = torch.tensor([len(p) - 1 for p in prompts], dtype=torch.int32, device="cuda")
        self.table, self.length, _, slots, self.n_free = sbd.sbd_block_tables(
            self.length, lens, self.table, self.free, self.n_free, self.page, int(lens.sum()))
        if not torch.equal(self.length, lens):
            raise RuntimeError("the cache is full")
        if len(slots):
            tokens = torch.cat([p[:-1] for p in prompts]).cuda()
            positions = torch.cat([torch.arange(len(p) - 1, dtype=torch.int32) for p in prompts]).cuda()
            _, (_, keys, values) = self._project(tokens, positions)
            sbd.sbd_cache_append_q8(keys, values, slots, *self.cache, *self.scale)
        self.last = torch.stack([p[-1] for p in prompts]).cuda()

    def turn(self):
        """One drafted turn of every request: (tokens [B, k + 1] int32, count [B] int32 of them that count)."""
        B, n = self.B, self.k + 1
        positions = (self.length[:, None] + torch.arange(n, dtype=torch.int32, device="cuda")).contiguous()
        rows = torch.full((B, n), self.vocab, dtype=torch.int32, device="cuda")
        rows[:, 0] = self.last
        x, (q, keys, values) = self._project(rows, positions)
        out = sbd.sbd_block_attention_q8(q, *self.cache, *self.scale, self.table, self.length, keys, values, n_causal=1)
        draft = self._logits(x, out)
        # Row i + 1 of the block is the marginal that node i's child is drawn from.
        draft = torch.cat([draft[:, 1:], draft[:, :1]], 1)
        ids = torch.arange(B * n, dtype=torch.int32, device="cuda")
        noise = sbd.sbd_gumbel_philox(ids, self.vocab, 1, 2 * self.turns).view(B, n, self.vocab)
        rows[:, 1:] = (draft[:, :-1].float() / (self.tau or 1.0) + (noise[:, :-1] if self.tau else 0.0)).argmax(-1)

        x, (q, keys, values) = self._project(rows, positions)
        out = sbd.sbd_tree_attention_q8(q, *self.cache, *self.scale, self.table, self.length, keys, values, self.chain)
        target = self._logits(x, out)
        uniform = torch.rand((B, n), generator=self.gen, device="cuda")
        gumbel = sbd.sbd_gumbel_philox(ids[:B].contiguous(), self.vocab, 1, 2 * self.turns + 1)
        path, tokens, logprob, count = sbd.sbd_verify_tree(target, draft, self.chain, rows, uniform, gumbel, self.tau)

        wanted = self.length + count
        self.table, self.length, start, slots, self.n_free = sbd.sbd_block_tables(
            self.length, wanted, self.table, self.free, self.n_free, self.page, B * n)
        sbd.sbd_cache_append_path_q8(keys, values, path, start, slots, *self.cache, *self.scale)
        if not torch.equal(self.length, wanted):
            raise RuntimeError("the cache is full")
        self.last = tokens.gather(1, count[:, None].long() - 1)[:, 0]
        self.turns += 1
        self.seen = dict(rows=rows, target=target, draft=draft, uniform=uniform, gumbel=gumbel, path=path, logprob=logprob,
                         keys=keys, values=values)
        return tokens, count


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--turns", type=int, default=8)
    ap.add_argument("--k", type=int, default=7)
    ap.add_argument("--prompt", type=int, default=1000, help="longest prompt")
    a = ap.parse_args()
    gen = torch.Generator().manual_seed(1)
    lens = torch.randint(2, a.prompt + 2, (a.requests,), generator=gen).tolist()
    most = -(-(a.prompt + 2 + a.turns * (a.k + 1)) // 64)
    server = DraftedDecoder(a.requests, n_pages=a.requests * most, max_pages=most, k=a.k)
    server.admit([torch.randint(0, server.vocab, (n,), dtype=torch.int32, generator=gen) for n in lens])
    for turn in range(a.turns):
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        tokens, count = server.turn()
        torch.cuda.synchronize()
        print(f"turn {turn}: {(time.perf_counter() - t0) * 1e6:.0f} us, {count.float().mean().item():.2f} tokens a request, "
              f"{int(server.n_free)} pages free, request 0: {tokens[0, :int(count[0])].tolist()}")
    assert sbd.sbd_device_error() == 0


if __name__ == "__main__":
    main()
