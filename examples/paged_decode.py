"""Set Block Decoding of a batch of uneven requests over a paged 8-bit KV cache.

One layer of random weights (what it says means nothing) run as a server would
run a model: requests come with prompts of their own lengths, every block of k
tokens is decoded until no mask is left, and a request that has ended gives its
pages back to the next one.  A block is

    sbd_block_tables            pages and slots for the tokens that enter the cache
    sbd_linear                  the fused projection of the rows
    sbd_block_attention_q8      the previous block's rows (causal, first iteration
                                only) and the block's, over the cache; a request just
                                taken in has no previous block, and is in a call apart
    sbd_cache_append_q8         the previous block's keys and values, straight from
                                the fused projection
    sbd_head_entropy_sample, sbd_eb_select
                                which masks become tokens; again from the projection
                                until there is none left

    python examples/paged_decode.py --requests 16 --blocks 4
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

MASK = -1


class PagedDecoder:
    def __init__(self, requests, n_pages, max_pages, *, page=64, k=8, q_heads=8, kv_heads=2, head_dim=128,
                 hidden=256, vocab=2000, gamma=0.5, seed=0):
        self.B, self.page, self.k, self.gamma = requests, page, k, gamma
        self.heads, self.vocab = (q_heads, kv_heads, head_dim), vocab
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, generator=gen, device="cuda") * shape[-1] ** -0.5).bfloat16()

        def ints(*shape):
            return torch.zeros(shape, dtype=torch.int32, device="cuda")

        self.embed = torch.randn((vocab + 1, hidden), generator=gen, device="cuda").bfloat16()   # the last: a mask
        self.position = torch.randn((1024, hidden), generator=gen, device="cuda").bfloat16()
        self.w_qkv = weight((q_heads + 2 * kv_heads) * head_dim, hidden)
        self.w_out, self.w_head = weight(hidden, q_heads * head_dim), weight(vocab, hidden)
        self.cache = [torch.zeros(n_pages, kv_heads, page, head_dim, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
        self.scale = [torch.zeros(n_pages, kv_heads, device="cuda") for _ in range(2)]
        self.table = torch.full((requests, max_pages), -1, dtype=torch.int32, device="cuda")
        self.free = torch.arange(n_pages, dtype=torch.int32, device="cuda")
        self.n_free = torch.full((1,), n_pages, dtype=torch.int32, device="cuda")
        self.length = ints(requests)                # tokens in the cache
        self.alive = torch.zeros(requests, dtype=torch.bool, device="cuda")
        # The block of each request that is not in the cache yet; a row of masks: there is none.
        self.last = torch.full((requests, k), MASK, dtype=torch.int32, device="cuda")
        self.forwards = 0

    def _resize(self, target, max_new):
        """The cache's pages for `target` tokens a request; the slots of the new ones."""
        self.table, self.length, start, slots, self.n_free = sbd.sbd_block_tables(
            self.length, target, self.table, self.free, self.n_free, self.page, max_new)
        return start, slots

    def _project(self, tokens, at):
        """Hidden rows and the fused projection's heads of tokens [T] at places `at` [T] of their requests."""
        q, kv, d = self.heads
        x = self.embed[torch.where(tokens == MASK, self.vocab, tokens).long()] + self.position[at.long() % 1024]
        y = torch.cat([sbd.sbd_linear(x[i:i + 512], self.w_qkv) for i in range(0, len(x), 512)])
        return x, y.view(len(x), q + 2 * kv, d)

    def admit(self, prompts):
        """Takes in {request: prompt [n] int32}: its keys and values enter the cache.  A place
        whose request has ended has no block waiting, unless the caller writes one to `last`."""
        target = self.length.clone()
        for b, p in prompts.items():
            if bool(self.alive[b]):
                raise ValueError(f"request {b} is still running")
            target[b] = len(p)
        order = sorted(prompts)
        tokens = torch.cat([prompts[b] for b in order]).cuda()
        _, slots = self._resize(target, len(tokens))
        _, qkv = self._project(tokens, torch.cat([torch.arange(len(prompts[b])) for b in order]).cuda())
        q, kv, _ = self.heads
        sbd.sbd_cache_append_q8(qkv[:, q:q + kv], qkv[:, q + kv:], slots, *self.cache, *self.scale)
        for b in order:
            self.alive[b] = self.length[b] == target[b]   # (a prompt that found no pages is not taken in)
        return self.alive.clone()

    def finish(self, requests):
        """Ends requests: their pages are free."""
        target = self.length.clone()
        for b in requests:
            target[b] = 0
            self.alive[b] = False
            self.last[b] = MASK
        self._resize(target, 0)

    def _rows(self, at, rows, n_causal):
        """Hidden rows, keys, values and attention of rows [b, n] of the requests `at`, of
        which the first n_causal are the block before."""
        q, kv, d = self.heads
        b, n = rows.shape
        length = self.length[at].contiguous()
        x, qkv = self._project(rows.reshape(-1), (length[:, None] + torch.arange(n, device="cuda")).reshape(-1))
        qkv = qkv.view(b, n, q + 2 * kv, d)
        keys, values = qkv[:, :, q:q + kv], qkv[:, :, q + kv:]
        out = sbd.sbd_block_attention_q8(
            qkv[:, :, :q].contiguous(), *self.cache, *self.scale, self.table[at].contiguous(), length,
            keys.contiguous(), values.contiguous(), n_causal=n_causal)
        return x.view(b, n, -1), keys, values, out

    def _store_block(self, at, pending, keys, values):
        """The previous block's keys and values, of the requests `at` that had one, enter the
        cache.  A request that finds no page ends here."""
        runs = self.alive & pending
        target = self.length + self.k * runs.int()
        _, slots = self._resize(target, self.B * self.k)
        live = runs[at]
        if not bool(live.all()):
            keys, values = keys[live], values[live]
        sbd.sbd_cache_append_q8(keys, values, slots, *self.cache, *self.scale)
        refused = (self.length != target).nonzero()[:, 0].tolist()
        if refused:
            self.finish(refused)

    def decode_block(self):
        """The next k tokens of every request [B, k] int32 (of ended ones too: their rows mean nothing)."""
        B, k, (q, _, d) = self.B, self.k, self.heads
        tokens = torch.full((B, k), MASK, dtype=torch.int32, device="cuda")
        masked = torch.ones((B, k), dtype=torch.uint8, device="cuda")
        everyone = slice(None)
        pending = (self.last != MASK).all(1)
        some, every = bool(pending.any()), bool(pending.all())
        while True:
            if some:                                # the first time: who has a block waiting, and who has none
                at = everyone if every else pending.nonzero()[:, 0]
                hidden, keys, values, out = self._rows(at, torch.cat([self.last, tokens], 1)[at], k)
                parts = [(at, hidden[:, k:], out[:, k:])]
                if not every:
                    rest = (~pending).nonzero()[:, 0]
                    hidden, _, _, out = self._rows(rest, tokens[rest], 0)
                    parts.append((rest, hidden, out))
                self._store_block(at, pending, keys[:, :k], values[:, :k])
                some = False
            else:
                hidden, _, _, out = self._rows(everyone, tokens, 0)
                parts = [(everyone, hidden, out)]
            h = torch.empty((B, k, self.embed.shape[1]), dtype=torch.bfloat16, device="cuda")
            for at, hidden, out in parts:
                flat = out.reshape(-1, q * d)
                y = torch.cat([sbd.sbd_linear(flat[i:i + 512], self.w_out) for i in range(0, len(flat), 512)])
                h[at] = hidden + y.view(hidden.shape)
            entropy, token = sbd.sbd_head_entropy_sample(h, self.w_head, masked, None, 0.0)
            sbd.sbd_eb_select(entropy, token, self.gamma, masked, tokens)
            self.forwards += 1
            if not bool(masked.any()):
                self.last = torch.where(self.alive[:, None], tokens, MASK)
                return tokens


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--k", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=1000, help="longest prompt")
    a = ap.parse_args()
    gen = torch.Generator().manual_seed(1)
    lens = torch.randint(1, a.prompt + 1, (a.requests,), generator=gen).tolist()
    most = -(-(a.prompt + (a.blocks + 1) * a.k) // 64)
    server = PagedDecoder(a.requests, n_pages=a.requests * most, max_pages=most, k=a.k)
    taken = server.admit({b: torch.randint(0, server.vocab, (n,), dtype=torch.int32, generator=gen) for b, n in enumerate(lens)})
    print(f"{int(taken.sum())} of {a.requests} requests, {sum(lens)} prompt tokens, {int(server.n_free)} pages free")
    for block in range(a.blocks):
        torch.cuda.synchronize()
        t0, f0 = time.perf_counter(), server.forwards
        tokens = server.decode_block()
        torch.cuda.synchronize()
        n = server.forwards - f0
        print(f"block {block}: {n} forwards, {(time.perf_counter() - t0) / n * 1e6:.0f} us each, "
              f"{int(server.n_free)} pages free, request 0: {tokens[0].tolist()}")
    assert sbd.sbd_device_error() == 0


if __name__ == "__main__":
    main()
