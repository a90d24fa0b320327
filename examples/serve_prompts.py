"""Prompts in chunks, single tokens and parallel samples in one batch, over a paged cache.

A small model with random weights (two layers, rotary positions, grouped heads) serves requests
whose prompts come in chunks of a token budget, beside requests that already decode a token a
step. Its matrix products are torch's; the rest is this library's: pages and slots for the new
tokens (map_slots), rotary positions with the write into the cache (rope_kv; for the 8-bit
cache append_kv_fp8 writes), attention of the ragged batch (chunk_attention), several samples of
a request that share its pages and the end of requests (fork_sequences, copy_pages).

    python examples/serve_prompts.py
"""

import os
import sys

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import torch  # noqa: E402

from paper_2609_04010_gb300 import binding as b  # noqa: E402


class Server:
    def __init__(self, batch, layers=2, num_q_heads=8, num_kv_heads=2, head_dim=64, vocab=512, page_size=16,
                 max_pages=40, num_pages=None, window=0, eight_bit=False, seed=0):
        self.B, self.L, self.Hq, self.H, self.D, self.P = batch, layers, num_q_heads, num_kv_heads, head_dim, page_size
        self.window, self.eight_bit = window, eight_bit
        g = torch.Generator(device="cuda").manual_seed(seed)
        dm, kv = num_q_heads * head_dim, num_kv_heads * head_dim

        def weight(*shape):
            return (torch.randn(shape, device="cuda", generator=g) / shape[0] ** 0.5).bfloat16()
        self.embed = torch.randn((vocab, dm), device="cuda", generator=g).bfloat16()
        self.wqkv = [weight(dm, dm + 2 * kv) for _ in range(layers)]
        self.wo = [weight(dm, dm) for _ in range(layers)]
        self.head = weight(dm, vocab)
        freq, self.factor = b.rope_frequencies(head_dim // 2, 10000.0, "yarn", 4.0, original_max=128)
        self.turns = b.rope_turns(freq)
        N = num_pages or batch * max_pages
        if eight_bit:
            self.caches = [b.new_kv_cache_fp8(N, num_kv_heads, page_size, head_dim) for _ in range(layers)]
        else:
            shape = (N, num_kv_heads, page_size, head_dim)
            self.caches = [tuple(torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
                           for _ in range(layers)]
        i32 = dict(dtype=torch.int32, device="cuda")
        self.table = torch.full((batch, max_pages), -1, **i32)
        self.free, self.free_count = torch.arange(N, **i32), torch.tensor([N], **i32)
        self.shares, self.kv_len = torch.zeros(N, **i32), torch.zeros(batch, **i32)
        self.status = b.new_workspace(256)  # of cache writes and page copies
        self.attn_ws, self.attn_rows = None, 0
        self.waiting = [[] for _ in range(batch)]  # tokens that a sequence has yet to bring

    def submit(self, prompts):
        for i, tokens in prompts.items():
            self.waiting[i] = list(tokens)

    def step(self, budget=128):
        """Brings up to `budget` waiting tokens, at least one of each waiting sequence. Returns the
        logits after each sequence's last token (rows of sequences that bring none are None)."""
        take, left = [], budget
        for w in self.waiting:
            take.append(min(len(w), max(1, left)) if w else 0)
            left -= take[-1]
        tokens = [t for w, n in zip(self.waiting, take) for t in w[:n]]
        self.waiting = [w[n:] for w, n in zip(self.waiting, take)]
        new = torch.tensor(take, dtype=torch.int32, device="cuda")
        x = self.embed[torch.tensor(tokens, device="cuda")]
        where = b.map_slots(new, self.kv_len, self.table, self.P, self.shares.numel(), self.free, self.free_count,
                            len(tokens))
        self._refused(where["flags"], "no pages for new tokens")
        self._room(len(tokens))
        for layer in range(self.L):
            x = self._layer(layer, x, where)
        self._check()
        ends = where["row_start"][1:].long() - 1
        logits = (x[ends.clamp_min(0)] @ self.head).float()
        return [logits[i] if n else None for i, n in enumerate(take)]

    def _room(self, rows):
        """The workspace of every layer's attention, which also holds its status, for steps of `rows` tokens."""
        if rows > self.attn_rows:
            q = torch.empty(rows, self.Hq, self.D, dtype=torch.bfloat16, device="cuda")
            starts = torch.zeros(self.B + 1, dtype=torch.int32, device="cuda")
            a = b.chunk_attn_args(q, self.caches[0], self.table, starts, self.kv_len, q)
            self.attn_ws, self.attn_rows = b.new_chunk_attn_workspace(a), rows

    def _refused(self, flags, what):
        if bool(flags.any()):
            raise RuntimeError(f"{what}: sequences {flags.nonzero().flatten().tolist()}")

    def _check(self):
        for ws, what in ((self.status, "cache writes or page copies"), (self.attn_ws, "attention")):
            code, flags = b.read_device_status(ws) if ws is not None else (0, 0)
            if code:
                raise RuntimeError(f"{what}: status {code}, flags {flags}")

    def _layer(self, layer, x, where):
        q, k, v = (x @ self.wqkv[layer]).unflatten(-1, (-1, self.D)).split([self.Hq, self.H, self.H], 1)
        cache = self.caches[layer]
        if self.eight_bit:
            q, k = b.rope_kv(q, k, None, where["positions"], self.turns, factor=self.factor)
            b.append_kv_fp8(k, v, where["slots"], *cache, self.status)
        else:
            q, _ = b.rope_kv(q, k, v, where["positions"], self.turns, where["slots"], *cache, factor=self.factor,
                             in_place=True, status_ws=self.status)
        out, _ = b.chunk_attention(q, cache, self.table, where["row_start"], self.kv_len, window=self.window,
                                   ws=self.attn_ws)
        return x + out.flatten(1) @ self.wo[layer]

    def fork(self, parent):
        """Sequence i goes on from sequence parent[i] (-1: it ends)."""
        res = b.fork_sequences(torch.tensor(parent, dtype=torch.int32, device="cuda"), self.kv_len, self.table,
                               self.shares, self.free, self.free_count, self.P)
        b.copy_pages(res["copies"], [x for cache in self.caches for x in cache], self.status)
        self._refused(res["flags"], "not forked")
        self._check()
        self.waiting = [list(self.waiting[q]) if q >= 0 else [] for q in parent]
        return res


def main():
    torch.manual_seed(0)
    s = Server(batch=6)
    s.submit({0: torch.randint(0, 512, (300,)).tolist(), 1: torch.randint(0, 512, (37,)).tolist()})
    rows = [None] * 6  # the logits after each sequence's last token
    while any(s.waiting):
        rows = [new if new is not None else old for new, old in zip(s.step(budget=100), rows)]
        print("tokens held:", s.kv_len.tolist())
    # two more samples of request 0 and one of request 1
    parent = [0, 1, 0, 0, 1, -1]
    s.fork(parent)
    rows = [rows[q] if q >= 0 else None for q in parent]
    for _ in range(8):
        sampled = {i: [int(torch.multinomial(torch.softmax(r, -1), 1))] for i, r in enumerate(rows) if r is not None}
        s.submit(sampled)
        rows = s.step()
        print({i: t[0] for i, t in sampled.items()})
    s.fork([-1] * 6)
    print("pages left:", int(s.free_count), "of", s.shares.numel(), "status:", b.read_device_status(s.status))


if __name__ == "__main__":
    main()
