"""A decoder in 8 bits that serves batches: an example of the language-model operators used together.

Every projection is a `Linear8`, keys and values live in paged `KVCache`s, prompts of unequal length go through
in one ragged batch and then decode a token at a time.  Norms, gates and residual sums are plain torch.

    python -m paper_2203_12091_gb300.decoder        # random weights, prints tokens per second
"""
from __future__ import annotations

import time

import torch

from . import llm


def rms_norm(x, weight, eps=1e-5):
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + eps) * weight).to(x.dtype)


class Layer:
    """Grouped-head attention and a gated MLP, each behind a norm and added to its input."""

    def __init__(self, width, heads, kv_heads, dim, hidden, gen, n_pages, page):
        def weights(n, k):
            return llm.Linear8.from_float(torch.randn(n, k, generator=gen, device=gen.device) * k ** -0.5)
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.qkv, self.out = weights((heads + 2 * kv_heads) * dim, width), weights(width, heads * dim)
        self.gate_up, self.down = weights(2 * hidden, width), weights(width, hidden)
        self.norm1, self.norm2 = (torch.ones(width, device=gen.device) for _ in range(2))
        self.cache = llm.KVCache.empty(n_pages, kv_heads, page, dim, gen.device)

    def __call__(self, x, pages, lens, starts, cos, sin):
        T, h, g = x.shape[0], self.heads, self.kv_heads
        qkv = self.qkv(rms_norm(x, self.norm1)).view(T, h + 2 * g, self.dim)  # (its views go to the kernels as they are)
        q = llm.kv_append(self.cache, pages, lens, qkv[:, h:h + g], qkv[:, h + g:], q=qkv[:, :h], starts=starts, cos=cos, sin=sin)
        a = llm.kv_attention(self.cache, pages, lens, q, starts=starts)
        x = x + self.out(a.view(T, h * self.dim))
        gate, up = self.gate_up(rms_norm(x, self.norm2)).chunk(2, -1)
        return x + self.down(torch.nn.functional.silu(gate) * up)


class Decoder:
    """`max_seqs` sequences of up to `max_tokens` tokens each; every sequence has its own pages of each layer's cache."""

    def __init__(self, vocab=1000, width=512, layers=2, heads=8, kv_heads=2, dim=64, hidden=1024, max_seqs=8, max_tokens=512, page=32,
                 dtype=torch.bfloat16, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        per_seq = -(-max_tokens // page)
        self.dtype, self.max_tokens = dtype, max_tokens
        self.embed = torch.randn(vocab, width, generator=gen, device=device).to(dtype)
        self.layers = [Layer(width, heads, kv_heads, dim, hidden, gen, max_seqs * per_seq, page) for _ in range(layers)]
        self.norm = torch.ones(width, device=device)
        self.head = llm.Linear8.from_float(torch.randn(vocab, width, generator=gen, device=device) * width ** -0.5)
        self.pages = torch.randperm(max_seqs * per_seq, generator=gen, device=device).int().view(max_seqs, per_seq)
        half = dim // 2
        angle = torch.arange(max_tokens, device=device).double()[:, None] * 10000.0 ** (-torch.arange(half, device=device).double() / half)
        self.cos, self.sin = angle.cos().float(), angle.sin().float()

    def forward(self, tokens, lens, starts=None):
        """Logits float32 [T, vocab] of new tokens [T]: lens int32 [B] tokens of each sequence with them, starts as in
        `llm.kv_append`."""
        x, pages = self.embed[tokens], self.pages[:lens.shape[0]]
        for layer in self.layers:
            x = layer(x, pages, lens, starts, self.cos, self.sin)
        return self.head(rms_norm(x, self.norm), torch.float32)

    def generate(self, prompts, count):
        """The `count` likeliest next tokens, one after the other, of each prompt (lists of tokens): int64 [B, count]."""
        dev, vocab = self.embed.device, self.embed.shape[0]
        if not 1 <= len(prompts) <= self.pages.shape[0] or count < 1 or any(not 1 <= len(p) <= self.max_tokens - count for p in prompts):
            raise ValueError("generate: no sequence or too many, an empty prompt, no token wanted, or more tokens than max_tokens")
        if any(not 0 <= t < vocab for p in prompts for t in p):
            raise ValueError(f"generate: tokens are 0 to {vocab - 1}")
        sizes = torch.tensor([len(p) for p in prompts], dtype=torch.int32)
        starts = torch.cat([torch.zeros(1, dtype=torch.int32), sizes.cumsum(0).int()]).to(dev)
        lens = sizes.to(dev)
        logits = self.forward(torch.tensor([t for p in prompts for t in p], device=dev), lens, starts)
        token = logits[starts[1:].long() - 1].argmax(-1)
        out = [token]
        for _ in range(count - 1):
            lens = lens + 1
            token = self.forward(token, lens).argmax(-1)
            out.append(token)
        return torch.stack(out, 1)


def main():
    model = Decoder(vocab=32000, width=2048, layers=8, heads=16, kv_heads=4, dim=128, hidden=5632, max_seqs=32, max_tokens=1024, page=64)
    prompts = [[(7 * i + j) % 32000 for j in range(200 + 17 * i)] for i in range(32)]
    model.generate(prompts, 4)
    torch.cuda.synchronize()
    at = time.perf_counter()
    model.generate(prompts, 64)
    torch.cuda.synchronize()
    took = time.perf_counter() - at
    print(f"{sum(map(len, prompts))} prompt tokens and 32 x 64 new ones in {took * 1e3:.1f} ms")


if __name__ == "__main__":
    main()
