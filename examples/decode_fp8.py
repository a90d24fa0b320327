"""Block decoding over the 8-bit KV cache, with penalties and a token mask.

A one-layer model with random weights serves a batch of ragged prompts. Its matrix products
are torch's; everything between them is this library's: pages and slots for the new tokens
(map_slots), their keys and values (append_kv_fp8), the block's attention
(verify_attention_fp8), the constraints on both models' logits (adjust_logits), the drafts
(sample_block), the acceptance (accept_block) and the cache's roll-back (commit_kv).

With one layer, a prompt's keys and values need no attention, so prefill only writes them. A
deeper model would run each layer's attention over the prompt, at most 64 tokens a call here.

    python examples/decode_fp8.py
"""

import os
import sys

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import torch  # noqa: E402

from paper_2609_04010_gb300 import binding as b  # noqa: E402


class Decoder:
    def __init__(self, batch, gamma, num_q_heads=8, num_kv_heads=2, head_dim=64, vocab=512,
                 page_size=16, max_pages=32, num_pages=None, seed=0):
        self.B, self.G, self.Hq, self.H, self.D = batch, gamma, num_q_heads, num_kv_heads, head_dim
        self.V, self.P, self.seed = vocab, page_size, seed
        dev, dm = "cuda", num_q_heads * head_dim
        g = torch.Generator(device=dev).manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, device=dev, generator=g) / shape[0] ** 0.5).bfloat16()

        self.embed = torch.randn((vocab, dm), device=dev, generator=g).bfloat16()
        self.wqkv = weight(dm, dm + 2 * num_kv_heads * head_dim)
        self.head, self.draft_head = weight(dm, vocab), weight(dm, vocab)
        self.place = torch.randn((gamma, dm), device=dev, generator=g).bfloat16()
        num_pages = num_pages or batch * max_pages
        self.cache, self.scale = b.new_kv_cache_fp8(num_pages, num_kv_heads, page_size, head_dim)
        self.table = torch.full((batch, max_pages), -1, dtype=torch.int32, device=dev)
        self.free = torch.arange(num_pages, dtype=torch.int32, device=dev)
        self.free_count = torch.tensor([num_pages], dtype=torch.int32, device=dev)
        self.kv_len = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.history = torch.zeros(batch, max_pages * page_size, dtype=torch.int32, device=dev)
        self.reserved = 0  # tokens past kv_len whose pages the table holds
        self.status = b.new_workspace(256)
        self.steps = 0

    def _project(self, tokens):
        x = self.embed[tokens.long()]
        q, k, v = (x @ self.wqkv).split([self.Hq * self.D, self.H * self.D, self.H * self.D], -1)
        # k and v stay column ranges of the projection: append_kv_fp8 takes their row stride
        return x, q.contiguous().view(*tokens.shape, self.Hq, self.D), \
            k.unflatten(-1, (self.H, self.D)), v.unflatten(-1, (self.H, self.D))

    def _write(self, num_new, tokens):
        """Keys and values of a packed ragged batch of tokens."""
        where = b.map_slots(num_new, self.kv_len, self.table, self.P, self.cache.shape[0], self.free,
                            self.free_count, tokens.numel(), self.reserved)
        x, q, k, v = self._project(tokens)
        b.append_kv_fp8(k, v, where["slots"], self.cache, self.scale, self.status)
        return where, x, q

    def prefill(self, prompts):
        """prompts: lists of at least two tokens. The last one starts the first block."""
        n = torch.tensor([len(p) - 1 for p in prompts], dtype=torch.int32, device="cuda")
        packed = torch.tensor([t for p in prompts for t in p[:-1]], dtype=torch.int32, device="cuda")
        where, _, _ = self._write(n, packed)
        for i, p in enumerate(prompts):
            self.history[i, :len(p) - 1] = torch.tensor(p[:-1], dtype=torch.int32)
        self.last = torch.tensor([p[-1] for p in prompts], dtype=torch.int32, device="cuda")
        self.prompt_len = n
        return where

    def step(self, temperature, repetition=None, frequency=None, presence=None, allowed=None):
        """One block per sequence. allowed: int32 bit words [batch][gamma][ceil(vocab / 32)]."""
        B, G = self.B, self.G
        rules = dict(history=self.history, history_len=self.kv_len.clone(), prompt_len=self.prompt_len,
                     repetition=repetition, frequency=frequency, presence=presence)
        # drafts, all drawn at once: their rows know the history only
        u = b.philox_uniforms(self.seed + 1, 2 * B * G, 2 * B * G * self.steps).view(2, B, G)
        x = self.embed[self.last.long()][:, None] + self.place
        # a draft row j is for block token j, whose mask is that of the row before
        shifted = None if allowed is None else torch.cat([allowed[:, :1], allowed[:, :-1]], 1).contiguous()
        drafter = b.adjust_logits((x @ self.draft_head).float(), allowed=shifted, **rules)
        block = b.sample_block(drafter, temperature, u[0])["block_tokens"]
        block[:, 0] = self.last
        # the verifier's pass over the block
        new = torch.full((B,), G, dtype=torch.int32, device="cuda")
        where, x, q = self._write(new, block.view(-1))
        out, lse = b.verify_attention_fp8(q.view(B, G, self.Hq, self.D), self.cache, self.scale,
                                          self.table, self.kv_len)
        target = ((out.view(B, G, -1) + x.view(B, G, -1)) @ self.head).float()
        raw = target.clone()
        b.adjust_logits(target, block_tokens=block, allowed=allowed, out=target, **rules)
        got = b.accept_block(target, drafter, block, temperature, u[1])
        held = self.kv_len.clone()
        b.commit_kv(self.kv_len, got["num_accepted"], self.table, self.P, G, self.free, self.free_count)
        self.reserved = G
        # emitted tokens but the last get their places; the last starts the next block
        n = got["num_accepted"] + 1
        at = torch.arange(G, device="cuda")[None]
        row, col = torch.nonzero(at < n[:, None], as_tuple=True)
        self.history[row, rules["history_len"].long()[row] + col] = got["out_tokens"][row, col]
        self.last = got["out_tokens"].gather(1, n.long()[:, None])[:, 0].contiguous()
        self.steps += 1
        return dict(where=where, block=block, q=q, out=out, lse=lse, raw=raw, target=target,
                    drafter=drafter, kv_len=held, history_len=rules["history_len"], **got)


def main():
    torch.manual_seed(0)
    d = Decoder(batch=6, gamma=8)
    d.prefill([torch.randint(0, d.V, (n,)).tolist() for n in (2, 17, 33, 64, 100, 211)])
    t = torch.tensor([0.0, 0.0, 0.7, 0.7, 1.0, 1.0], device="cuda")
    rep = torch.full((6,), 1.3, device="cuda")
    even = torch.full((6, 8, (d.V + 31) // 32), 0x55555555, dtype=torch.int32, device="cuda")
    for i in range(8):
        r = d.step(t, repetition=rep, presence=rep - 1, allowed=even)
        for s in range(6):
            print(i, s, r["out_tokens"][s, :int(r["num_emitted"][s])].tolist())
    code, flags = b.read_device_status(d.status)
    print("tokens held:", d.kv_len.tolist(), "pages left:", int(d.free_count), "status:", code)


if __name__ == "__main__":
    main()
