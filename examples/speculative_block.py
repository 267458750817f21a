"""Speculative decoding with a paged cache: what a program runs block after block.

A small attention model with random weights stands for the target, a table of next-token logits
for the drafter.  One block:

1. the drafter proposes gamma tokens on each of K paths (psd.draft, or tokens of its own rows);
2. the target scores the root and every path in one pass: psd.kv_append puts the new keys (normed,
   turned by their position) and values into the paged cache, psd.attention lets each row see the
   cache and its own path;
3. psd.verify races target and drafts under the key (K paths), or psd.verify_given accepts and
   rejects from given random numbers (one path);
4. psd.kv_keep moves the accepted path's keys and values behind the cache, psd.advance commits
   the tokens.

The keyed text is the target's own: it is the same whatever the drafter proposes.

    python examples/speculative_block.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_21858_amd import psd  # noqa: E402

DEV = "cuda"


class Target:
    """Layers of attention over a paged cache, without the rest of a real model."""

    def __init__(self, vocab=500, layers=2, heads=8, kv_heads=2, dim=64, page=16, pages=512, dtype=torch.float32, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.width = heads * dim
        self.heads, self.kv_heads, self.dim, self.dtype = heads, kv_heads, dim, dtype

        def weights(*shape):
            return (torch.randn(shape, device=DEV, generator=g) * shape[0] ** -0.5).to(dtype)

        self.embed = torch.randn((vocab, self.width), device=DEV, generator=g).to(dtype)
        self.qkv = [weights(self.width, (heads + 2 * kv_heads) * dim) for _ in range(layers)]
        self.out = [weights(self.width, self.width) for _ in range(layers)]
        self.unembed = 2.5 * weights(self.width, vocab)
        self.norm = torch.ones(dim, device=DEV, dtype=dtype)
        angle = torch.arange(4096, device=DEV)[:, None] * 10000.0 ** (-torch.arange(dim // 2, device=DEV) * 2.0 / dim)
        self.cos, self.sin = angle.cos(), angle.sin()
        shape = (layers, pages, page, kv_heads, dim)
        self.k, self.v = torch.empty(shape, device=DEV, dtype=dtype), torch.empty(shape, device=DEV, dtype=dtype)
        self.cache = [psd.make_cache(self.k[i], self.v[i]) for i in range(layers)]
        self.all_layers = psd.make_cache(self.k, self.v)
        self.ws = {}

    def workspace(self, seqs):
        n = psd.attention_workspace_bytes(self.cache[0], seqs, self.heads)
        if n not in self.ws:
            self.ws[n] = torch.zeros(n, dtype=torch.uint8, device=DEV)
        return self.ws[n]

    def __call__(self, tokens, seqs, positions=None, mask=None):
        """Logits of packed rows of new tokens; their keys and values go into the cache."""
        H, G, D = self.heads, self.kv_heads, self.dim
        x = self.embed[tokens.long()]
        ws = self.workspace(seqs)
        for layer, cache in enumerate(self.cache):
            y = torch.nn.functional.rms_norm(x, (self.width,)) @ self.qkv[layer]
            q, k, v = (t.unflatten(1, (-1, D)) for t in y.split((H * D, G * D, G * D), 1))
            q = psd.kv_append(cache, seqs, k, v, q=q, cos=self.cos, sin=self.sin, positions=positions, q_norm=self.norm,
                              k_norm=self.norm)
            a = psd.attention(cache, seqs, q, ws, mask=mask)["out"]
            x = x + a.flatten(1) @ self.out[layer]
        return torch.nn.functional.rms_norm(x, (self.width,)) @ self.unembed


def path_mask(K, gamma, B):
    """Each row of 1 + K gamma new tokens sees the root and its own path so far (int32 bits)."""
    n = 1 + K * gamma
    see = torch.zeros((n, -(-n // 32) * 32), dtype=torch.int64)
    see[:, 0] = 1
    for k in range(K):
        at = 1 + k * gamma
        see[at:at + gamma, at:at + gamma] = torch.ones((gamma, gamma), dtype=torch.int64).tril()
    words = (see.view(n, -1, 32) << torch.arange(32)).sum(-1)
    words = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
    return words.repeat(B, 1).contiguous().to(DEV)


class Loop:
    """Texts, their pages and their lengths on the device."""

    def __init__(self, target, prompts, max_len, n_new, params, gamma):
        B, m = prompts.shape
        self.target, self.params, self.gamma, self.B, self.max_len, self.n = target, params, gamma, B, max_len, n_new
        self.text = torch.full((B, max_len), -1, dtype=torch.int32, device=DEV)
        self.text[:, :m] = prompts
        self.length = torch.full((B,), m, dtype=torch.int64, device=DEV)
        self.start = torch.empty((B,), dtype=torch.int64, device=DEV)
        self.prefix = torch.empty((B, params.ctx_window), dtype=torch.int32, device=DEV)
        self.active = torch.empty((1,), dtype=torch.int32, device=DEV)
        page = target.k.shape[2]
        width = -(-(max_len + n_new) // page)
        self.table = torch.arange(B * width, dtype=torch.int32, device=DEV).flip(0).view(B, width).contiguous()
        self.kv_len = torch.empty((B,), dtype=torch.int32, device=DEV)
        self.seqs = self.sequences(n_new, max_len + n_new)
        # the prompts' keys and values, all but the last token's: it is the first block's root
        if m > 1:
            self.kv_len.fill_(m - 1)
            target(prompts[:, :-1].reshape(-1), self.sequences(m - 1, m))
        psd.advance(params, gamma, max_len, self.text, self.length, self.prefix, self.start, self.active)

    def sequences(self, n, max_kv):
        first = torch.arange(self.B + 1, dtype=torch.int32, device=DEV) * n
        return psd.make_seqs(first, self.kv_len, self.table, self.B * n, n, max_kv)

    def score(self, drafts, mask, depth):
        """Target logits [B][n][V] of the root and the drafts [B][n - 1]."""
        root = self.text.gather(1, (self.start - 1)[:, None])
        self.kv_len.copy_(self.start - 1 + self.n)
        positions = ((self.start - 1)[:, None] + depth).to(torch.int32).view(-1).contiguous()
        logits = self.target(torch.cat((root, drafts), 1).view(-1), self.seqs, positions, mask)
        return logits.view(self.B, self.n, -1)

    def commit(self, out, keep):
        """Keep the accepted drafts' keys and values (new tokens keep[b], the root first), commit the tokens."""
        psd.kv_keep(self.target.all_layers, self.seqs, keep.to(torch.int32).contiguous(), out["out_len"])
        psd.advance(self.params, self.gamma, self.max_len, self.text, self.length, self.prefix, self.start, self.active,
                    out["out_tokens"], out["out_len"])


def keyed(target, drafter, prompts, max_len, key=7, K=4, gamma=4):
    """K paths under the key.  Returns the texts and the mean number of tokens a block commits."""
    B, m = prompts.shape
    V = target.embed.shape[0]
    params = psd.make_params(key, V, K, m, 1.0, 1.0, dtype=target.dtype)
    ws = psd.new_workspace(params, B, gamma)
    loop = Loop(target, prompts, max_len, 1 + K * gamma, params, gamma)
    mask = path_mask(K, gamma, B)
    steps = torch.arange(gamma, device=DEV)
    depth = torch.cat((torch.zeros(1, device=DEV, dtype=torch.int64), (steps + 1).repeat(K)))
    index = torch.arange(K, device=DEV)[:, None] * gamma
    rows = torch.cat((torch.zeros((K, 1), device=DEV, dtype=torch.int64), 1 + index + steps), 1)  # [K][gamma + 1] of the new tokens
    blocks = 0
    committed = 0
    while True:
        drafts = torch.zeros((B, K, gamma), dtype=torch.int32, device=DEV)
        last = loop.text.gather(1, (loop.start - 1)[:, None]).expand(B, K)
        for s in range(gamma):
            logits = drafter[last.long()][:, :, None].contiguous()
            psd.draft(params, ws, loop.prefix, loop.start, gamma, s, logits, drafts)
            last = drafts[:, :, s]
        logits = loop.score(drafts.view(B, -1), mask, depth)
        out = psd.verify(params, ws, loop.prefix, loop.start, logits[:, rows].contiguous(), draft_tokens=drafts, target_rows=K)
        # the accepted drafts' path: the first one that holds the tokens before the last
        same = (drafts == out["out_tokens"][:, None, :gamma]).long().cumprod(2).sum(2)
        path = (same >= (out["out_len"] - 1)[:, None]).long().argmax(1)
        committed += int(out["out_len"].sum())
        loop.commit(out, rows[path])
        blocks += 1
        if int(loop.active) == 0:
            return loop.text, committed / (blocks * B)


def given(target, drafter, prompts, max_len, seed=0, gamma=4):
    """One path, accepted and rejected from given random numbers.  Returns as keyed()."""
    B, m = prompts.shape
    V = target.embed.shape[0]
    params = psd.make_params(0, V, 1, m, 1.0, 1.0, dtype=target.dtype)
    ws = psd.new_verify_given_workspace(params, B, gamma)
    loop = Loop(target, prompts, max_len, 1 + gamma, params, gamma)
    g = torch.Generator(device=DEV).manual_seed(seed)
    depth = torch.arange(gamma + 1, device=DEV)
    blocks = 0
    committed = 0
    while True:
        drafts = torch.zeros((B, gamma), dtype=torch.int32, device=DEV)
        rows = torch.empty((B, gamma, V), dtype=target.dtype, device=DEV)
        last = loop.text.gather(1, (loop.start - 1)[:, None])[:, 0]
        for s in range(gamma):
            rows[:, s] = drafter[last.long()]
            last = torch.multinomial(torch.softmax(rows[:, s].float(), -1), 1, generator=g)[:, 0].to(torch.int32)
            drafts[:, s] = last
        logits = loop.score(drafts, None, depth)
        u = torch.rand((B, gamma), device=DEV, generator=g)
        e = torch.empty((B, V), device=DEV).exponential_(generator=g).clamp_(min=1e-30)
        out = psd.verify_given(params, ws, logits.contiguous(), rows, drafts, u, e)
        committed += int(out["out_len"].sum())
        loop.commit(out, depth.expand(B, -1))
        blocks += 1
        if int(loop.active) == 0:
            return loop.text, committed / (blocks * B)


def good_drafter(target):
    """Next-token logits by the last token alone: the target's own after that token."""
    return (torch.nn.functional.rms_norm(target.embed, (target.width,)) @ target.unembed).contiguous()


def main():
    target = Target()
    prompts = torch.randint(0, 500, (8, 6), dtype=torch.int32, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    good = good_drafter(target)
    poor = torch.randn(good.shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))
    a, rate_a = keyed(target, good, prompts, 100)
    b, rate_b = keyed(target, poor, prompts, 100)
    print(f"keyed, 4 paths: {rate_a:.2f} tokens a block with the good drafter, {rate_b:.2f} with the poor one; "
          f"same text: {bool(torch.equal(a, b))}")
    _, rate = given(target, good, prompts, 100)
    print(f"given random numbers, 1 path: {rate:.2f} tokens a block")


if __name__ == "__main__":
    main()
