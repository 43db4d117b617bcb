"""A verifier on the GPU for the closed loop: a small attention model whose choices are steered to a known continuation.

The paper's simulated verifier (Section 4.1, "Simulated Ablations") accepts a drafted token exactly when it equals the ground-truth token at its position.
Here that happens where a serving engine does it: the rows [last token, draft nodes] of the whole batch go through the layers (sd_rotate, sd_attend), their logits
decide (sd_accept), and the accepted rows stay in the cache (sd_commit).  Weights are random; the logit of the token that really follows is raised above
all others, so that what is accepted is known.
"""
from __future__ import annotations

from typing import Dict, Sequence

import numpy as np
import torch

import paper_2411_04975_b200 as sfx

STEER = 1e4                # added to the logit of the token that follows: above any that the random weights give


class Verifier:
    def __init__(self, n: int, max_tokens: int, max_draft: int, vocab: int, *, layers: int = 2, q_heads: int = 8, kv_heads: int = 2, head: int = 64,
                 width: int = 256, page: int = 64, base: float = 10000.0, seed: int = 0, dtype=torch.bfloat16, device=None):
        self.n, self.M, self.vocab, self.layers, self.q_heads, self.kv_heads, self.head = n, max_draft, vocab, layers, q_heads, kv_heads, head
        self.device = dev = torch.device("cuda", torch.cuda.current_device()) if device is None else device
        g = torch.Generator(device=dev)
        g.manual_seed(seed)

        def weight(*shape):
            return (torch.randn(*shape, device=dev, generator=g) * shape[-2] ** -0.5).to(dtype)

        self.embed = torch.randn(vocab, width, device=dev, generator=g).to(dtype)
        self.qkv = [weight(width, (q_heads + 2 * kv_heads) * head) for _ in range(layers)]
        self.out = [weight(q_heads * head, width) for _ in range(layers)]
        self.unembed = weight(width, vocab)
        self.norms = [(1 + 0.1 * torch.randn(2, head, device=dev, generator=g)).to(dtype) for _ in range(layers)]
        self.freq, self.turned = sfx.rotary_frequencies(head, base, device=dev)
        pages = -(-(max_tokens + max_draft + 1) // page)
        self.table = torch.randperm(n * pages, device=dev, generator=g).to(torch.int32).view(n, pages)
        self.k_cache, self.v_cache = (torch.zeros(layers, n * pages, page, kv_heads, head, dtype=dtype, device=dev) for _ in range(2))
        self.cached = torch.zeros(n, dtype=torch.int32, device=dev)

    def forward(self, ids: torch.Tensor, offsets: torch.Tensor, mask=None, cached=None) -> torch.Tensor:
        """Rows of tokens through the layers (their keys and values go to the cache behind what is there); the last layer's output."""
        x = self.embed[ids]
        cached = self.cached if cached is None else cached
        Q, H, D = self.q_heads, self.kv_heads, self.head
        for layer in range(self.layers):
            qkv = (x @ self.qkv[layer]).view(-1, Q + 2 * H, D)
            k, v = self.k_cache[layer], self.v_cache[layer]
            q = sfx.sd_rotate(qkv[:, :Q], qkv[:, Q:Q + H], qkv[:, Q + H:], k, v, self.table, offsets, cached, self.freq, mask=mask,
                              q_weight=self.norms[layer][0], k_weight=self.norms[layer][1], scale=self.turned)
            x = x + sfx.sd_attend(q, k, v, self.table, offsets, cached, mask=mask).view(-1, Q * D) @ self.out[layer]
        return x

    def start(self, slots: Sequence[int], prompts: Sequence[np.ndarray]) -> None:
        """New requests in these slots: all tokens of their prompts but the last go into the cache (the last is the first step's first row)."""
        todo = {s: np.asarray(p[:-1], dtype=np.int64) for s, p in zip(slots, prompts)}
        begin = torch.zeros(self.n, dtype=torch.int32)
        step = sfx.MAX_DRAFT + 1                                  # rows that a request can have in a call: a chain of so many
        for at in range(0, max((len(p) for p in todo.values()), default=0), step):
            part = {s: p[at:at + step] for s, p in todo.items() if len(p) > at}
            count = np.zeros(self.n + 1, dtype=np.int64)
            for s, p in part.items():
                count[s + 1] = len(p)
            begin[list(part)] = at
            ids = np.concatenate([part[s] for s in sorted(part)])
            self.forward(torch.as_tensor(ids, device=self.device), torch.as_tensor(np.cumsum(count), device=self.device), cached=begin.to(self.device))
        for s, p in todo.items():
            self.cached[s] = len(p)

    def rows(self, out: Dict[str, torch.Tensor], last: torch.Tensor):
        """(ids, offsets, request, depth) of the rows [last token, draft nodes] of sd_speculate's drafts."""
        offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=self.device), (out["n_draft"] + 1).cumsum(0)])
        total = int(offsets[-1])
        row = torch.arange(total, device=self.device)
        request = torch.searchsorted(offsets, row, right=True) - 1
        local = row - offsets[request]
        node = (local - 1).clamp(min=0)
        ids = torch.where(local == 0, last[request].long(), out["tokens"][request, node].long())
        start = self.cached[request].long()
        depth = torch.where(local == 0, 0, out["positions"][request, node].long() - start)
        return ids, offsets, request, depth

    def step(self, out: Dict[str, torch.Tensor], last: torch.Tensor, follows: torch.Tensor) -> Dict[str, torch.Tensor]:
        """Verifies the drafts `out` of a batch in all slots.  last: the requests' last tokens; follows: int64[n, *], the tokens that really come next (-1: nothing more is
        known).  Returns what sd_accept does; the cache and its lengths go on behind the accepted rows."""
        ids, offsets, request, depth = self.rows(out, last)
        mask = out["mask"]
        logits = self.forward(ids, offsets, mask) @ self.unembed
        want = follows[request, depth.clamp(max=follows.shape[1] - 1)]
        logits.scatter_add_(1, want.clamp(min=0)[:, None], torch.where(want >= 0, STEER, 0.0)[:, None].to(logits.dtype))
        got = sfx.sd_accept(logits, offsets, out["tokens"], out["parents"])
        sfx.sd_commit(self.k_cache, self.v_cache, self.table, self.cached, got["path"], out=self.cached)
        return got
