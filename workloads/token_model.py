"""A small decoder of tokens on the library's serving operators: what a program that answers with a language model does at every step.

Each block is  x -> norm -> queries, keys, values (one 8-bit product) -> keys and values into the cache -> attention -> product + shortcut
-> norm -> product, ReLU -> product + shortcut;  behind the last one a norm, the logits, and what is read from them.  All sequences of a batch may begin with the same
tokens (instructions, say): those pass once, and lie in the cache once.

    python -m workloads.token_model          # 16 answers to one shared beginning, on the GPU

Weights are random, as everywhere in `workloads`: the numbers mean nothing, the time does."""
from __future__ import annotations

from dataclasses import dataclass
from typing import Dict, List, Optional

import torch

from paper_2302_00282_amd import tokens as T


@dataclass
class Sizes:
    layers: int = 4
    width: int = 512             # the feed-forward block of `cnn_graphs.matmul_chain`: 512 -> 2048 -> 512
    hidden: int = 2048
    heads: int = 8
    kv_heads: int = 2
    head_dim: int = 64
    vocab: int = 32000
    page: int = 64
    eps: float = 1e-5


def draw(sizes: Sizes, seed: int = 11, device="cuda") -> Dict[str, torch.Tensor]:
    """Weights of the model in float32: He-normal products, norms around one, embeddings of size one."""
    g = torch.Generator(device="cpu").manual_seed(seed)

    def normal(rows, cols):
        return (torch.randn(rows, cols, generator=g) / cols ** 0.5).to(device)

    def gains(n):
        return (torch.rand(n, generator=g) + 0.5).to(device)

    s = sizes
    w = {"embed": torch.randn(s.vocab, s.width, generator=g).to(device), "final.norm": gains(s.width), "logits": 4 * normal(s.vocab, s.width)}
    for i in range(s.layers):
        w.update({f"{i}.norm1": gains(s.width), f"{i}.qkv": normal((s.heads + 2 * s.kv_heads) * s.head_dim, s.width), f"{i}.out": normal(s.width, s.heads * s.head_dim),
                  f"{i}.norm2": gains(s.width), f"{i}.up": normal(s.hidden, s.width), f"{i}.down": normal(s.width, s.hidden)})
    return w


class TokenModel:
    """The weights in 8 bits, a cache per layer, and the pages that its sequences hold.

    The pages of the shared beginning come first, then each sequence's own."""

    def __init__(self, sizes: Sizes, weights: Dict[str, torch.Tensor], n_seqs: int, longest: int, prefix: int = 0):
        s = self.sizes = sizes
        self.norms = {k: v.float().contiguous() for k, v in weights.items() if "norm" in k}
        self.embed = weights["embed"].bfloat16()
        self.layers8 = {k: T.quantize_rows(v) for k, v in weights.items() if "norm" not in k and k != "embed"}
        device = self.embed.device
        front, own = -(-prefix // s.page), -(-longest // s.page)
        self.caches = [T.KVCache.empty(front + n_seqs * own, s.page, s.kv_heads, s.head_dim, device) for _ in range(s.layers)]
        pages = torch.arange(front + n_seqs * own, dtype=torch.int32, device=device)
        self.prefix_table, self.tables = pages[:front], pages[front:].view(n_seqs, own)
        self.prefix, self.lengths = 0, torch.zeros(n_seqs, dtype=torch.int32, device=device)
        self.longest, self.room = longest, own * s.page

    def _product(self, name: str, x: torch.Tensor, norm: Optional[str] = None, **kw) -> torch.Tensor:
        w, scale = self.layers8[name]
        return T.linear(x, w, scale, gamma=None if norm is None else self.norms[norm], eps=self.sizes.eps, **kw)

    def _blocks(self, x: torch.Tensor, slots: torch.Tensor, attend) -> torch.Tensor:
        """Logits (bfloat16 [tokens][vocab]) of the embedded tokens x, whose keys and values go to `slots`; attend(q, cache) is the attention of their queries."""
        s = self.sizes
        for i, cache in enumerate(self.caches):
            qkv = self._product(f"{i}.qkv", x, f"{i}.norm1").view(len(x), s.heads + 2 * s.kv_heads, s.head_dim)
            cache.write(qkv[:, s.heads:s.heads + s.kv_heads], qkv[:, s.heads + s.kv_heads:], slots)
            x = self._product(f"{i}.out", attend(qkv[:, :s.heads], cache).view(len(x), -1), residual=x)
            x = self._product(f"{i}.down", self._product(f"{i}.up", x, f"{i}.norm2", relu=True), residual=x)
        return self._product("logits", x, "final.norm")

    def begin(self, tokens: torch.Tensor) -> torch.Tensor:
        """Takes the tokens (int64 [n]) that all sequences begin with; returns their logits."""
        n, page = len(tokens), self.sizes.page
        if n > len(self.prefix_table) * page:
            raise ValueError(f"{n} tokens in the {len(self.prefix_table)} pages of the shared beginning")
        at = torch.arange(n, device=tokens.device)
        slots = self.prefix_table.long()[at // page] * page + at % page
        table, length = self.prefix_table[None], torch.full((1,), n, dtype=torch.int32, device=tokens.device)
        starts = torch.tensor([0, n], dtype=torch.int32, device=tokens.device)
        self.prefix = n
        return self._blocks(self.embed[tokens], slots, lambda q, cache: T.attention(q, cache, table, length, starts=starts, max_queries=n, max_length=n))

    def append(self, tokens: List[torch.Tensor]) -> torch.Tensor:
        """Takes some more tokens of each sequence (int64, any number of each); returns the logits of all, one sequence behind the other."""
        counts = [len(t) for t in tokens]
        held = self.lengths.tolist()
        if len(counts) != len(held) or max(a + b for a, b in zip(held, counts)) > self.room:
            raise ValueError(f"{counts} more tokens of sequences of {held}, in pages for {self.room} each")
        device, page = self.lengths.device, self.sizes.page
        starts = torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], dtype=torch.int32, device=device)
        seq = torch.repeat_interleave(torch.arange(len(counts), device=device), torch.tensor(counts, device=device))
        at = self.lengths.long()[seq] + torch.arange(len(seq), device=device) - starts.long()[seq]
        self.lengths += starts[1:] - starts[:-1]
        return self._attend(torch.cat(tokens), self.tables.long()[seq, at // page] * page + at % page, starts, max(counts))

    def step(self, tokens: torch.Tensor) -> torch.Tensor:
        """Takes one more token of each sequence (int64 [sequences]); returns their logits.  No look at the device: a step can be captured in a graph.
        Beyond the pages that a sequence has, nothing more of it is stored, and it is answered from what they hold."""
        at, page = self.lengths.long(), self.sizes.page
        there = at < self.room
        place = torch.where(there, at, torch.zeros_like(at))
        slots = torch.where(there, self.tables.long().gather(1, (place // page)[:, None]).squeeze(1) * page + place % page, torch.full_like(at, -1))
        self.lengths += 1
        return self._attend(tokens, slots, None, 1)

    def _attend(self, tokens, slots, starts, most):
        front = dict(prefix_table=self.prefix_table, prefix_length=self.prefix) if self.prefix else {}
        return self._blocks(self.embed[tokens], slots, lambda q, cache: T.attention(q, cache, self.tables, self.lengths, starts=starts, max_queries=most, max_length=self.longest, **front))


def main():
    import time

    sizes, n_seqs, prefix, own, answer = Sizes(), 16, 1000, 24, 32
    model = TokenModel(sizes, draw(sizes), n_seqs, own + answer, prefix)
    g = torch.Generator().manual_seed(5)
    pick = lambda n: torch.randint(0, sizes.vocab, (n,), generator=g).cuda()
    model.begin(pick(prefix))
    counts = [1 + (7 * b) % own for b in range(n_seqs)]
    last = torch.tensor(counts).cumsum(0).cuda() - 1
    logits = model.append([pick(n) for n in counts])[last]
    said = torch.zeros(n_seqs, device="cuda")
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(answer):
        _, entropy, best, token = T.logprobs(logits, top=5)
        said += best[:, 0]
        logits = model.step(token[:, 0].long())
    torch.cuda.synchronize()
    s = time.perf_counter() - began
    print(f"{n_seqs} sequences of {prefix} shared and up to {own} own tokens: {answer} more of each in {s * 1e3:.1f} ms, {n_seqs * answer / s:.0f} tokens/s; "
          f"log probability of the first answer {said[0].item():.2f}, entropy of its next token {entropy[0].item():.3f}")


if __name__ == "__main__":
    main()
