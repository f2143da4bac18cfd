"""The attention block of a decoder out of the decoder operators, and a small serving loop around a stack of them.

    python -m paper_2007_12216_amd.decode --layers 4 --requests 8 --prompt 300 --tokens 32

runs synthetic requests of different lengths, their prompts in one step and then a token a step, on random weights, and prints the time of both."""
from __future__ import annotations

import argparse
import time

import torch

from .decoder import BatchTables, Cache4, CacheAttention, Fp8Linear, QKNormRope


def rotation_angles(positions: int, rotary: int, base: float = 10000.0, device="cuda:0") -> torch.Tensor:
    """float32 [positions][rotary] for QKNormRope: cosines, then sines, of position * base^(-2i / rotary)."""
    turn = torch.outer(torch.arange(positions, dtype=torch.float64), base ** (-2.0 * torch.arange(rotary // 2, dtype=torch.float64) / rotary))
    return torch.cat([turn.cos(), turn.sin()], 1).to(torch.float32).to(device)


class AttentionBlock:
    """Projection to queries, keys and values, their norms and rotation into the layer's own cache, attention over it, projection back: five launches or six.

    qkv: [(q_heads + 2 kv_heads) * head_dim][width] and out: [width][q_heads * head_dim], both Fp8Linear.  Serves one stream at a time."""

    def __init__(self, qkv: Fp8Linear, rope: QKNormRope, cache: Cache4, attention: CacheAttention, out: Fp8Linear):
        q_heads = attention.desc.q_heads
        if qkv.outputs != (q_heads + 2 * cache.kv_heads) * cache.head_dim or out.inputs != q_heads * cache.head_dim:
            raise ValueError(f"projections {qkv.outputs} x {qkv.inputs} and {out.outputs} x {out.inputs} do not fit {q_heads} and {cache.kv_heads} heads of {cache.head_dim}")
        if (rope.desc.q_heads, rope.desc.kv_heads, rope.desc.head_dim) != (q_heads, cache.kv_heads, cache.head_dim):
            raise ValueError(f"a rotation of {rope.desc.q_heads} and {rope.desc.kv_heads} heads of {rope.desc.head_dim} for {q_heads} and {cache.kv_heads} heads of {cache.head_dim}")
        if attention.cache is not cache:
            raise ValueError("the attention must be over the block's cache")
        self.qkv, self.rope, self.cache, self.attention, self.out = qkv, rope, cache, attention, out

    def forward(self, x: torch.Tensor, tables: BatchTables, table: torch.Tensor, max_fresh: int = 0, max_len: int = 0) -> torch.Tensor:
        """x: [tables.n_tokens][width], the step's new tokens as `tables` packs them (its build has been called with `table`).  Returns [n_tokens][width]."""
        q = self.rope.append(self.qkv.forward(x), tables.positions, tables.slots, self.cache)
        return self.out.forward(self.attention.forward(q, table, tables.lens, tables.row_start, max_fresh=max_fresh, max_len=max_len).flatten(1))


class DecodingBatch:
    """Requests that go through a stack of blocks together: block table, free pages and lengths are shared by all layers."""

    def __init__(self, blocks: list[AttentionBlock], n_requests: int, max_len: int):
        cache = blocks[0].cache
        if any((b.cache.pages, b.cache.page_size) != (cache.pages, cache.page_size) for b in blocks):
            raise ValueError("the blocks' caches must have the same pages")
        angles = min(b.rope.desc.max_position for b in blocks)
        if max_len > angles:  # positions without angles are not cached
            raise ValueError(f"angles for {angles} positions, requests of up to {max_len}")
        self.blocks, self.page_size, self.max_len = blocks, cache.page_size, max_len
        self.free = torch.arange(cache.pages, dtype=torch.int32, device=cache.device)
        self.table = torch.full((n_requests, -(-max_len // self.page_size)), -1, dtype=torch.int32, device=cache.device)
        self.cached, self.lens, self.used, self.tables = torch.zeros(n_requests, dtype=torch.int32, device=cache.device), [0] * n_requests, 0, None

    def step(self, x: torch.Tensor, fresh: list[int]) -> torch.Tensor:
        """x: [sum(fresh)][width], the requests' new tokens one request after another.  Returns the same shape behind the last block, each block's result added to its input."""
        if len(fresh) != len(self.lens) or sum(fresh) != x.shape[0] or min(fresh) < 0:
            raise ValueError(f"{x.shape[0]} rows for requests of {fresh} new tokens")
        lens = [n + f for n, f in zip(self.lens, fresh)]
        pages = sum(-(-n // self.page_size) for n in lens)
        if max(lens) > self.max_len or pages > self.free.numel():
            raise ValueError(f"lengths up to {max(lens)} of {self.max_len}, {pages} pages of {self.free.numel()}")
        if self.tables is None or self.tables.n_tokens != x.shape[0]:
            self.tables = BatchTables(len(lens), x.shape[0], self.page_size, self.free.device)
        tables = self.tables.build(self.cached, torch.tensor(fresh, dtype=torch.int32).to(self.free.device), self.free[self.used:], self.table)
        for block in self.blocks:
            x = x + block.forward(x, tables, self.table, max_fresh=max(fresh), max_len=max(lens))
        self.cached.copy_(tables.lens)
        self.lens, self.used = lens, pages
        return x


def random_block(width: int, q_heads: int, kv_heads: int, head_dim: int, pages: int, page_size: int, angles: torch.Tensor, generator: torch.Generator) -> AttentionBlock:
    """Weights of a normal distribution under 1 / sqrt(inputs)."""
    def linear(outputs, inputs):
        w = torch.randn(outputs, inputs, generator=generator) / inputs ** 0.5
        return Fp8Linear.from_weights(w.to(torch.bfloat16).to(angles.device))
    norm = torch.ones(head_dim, dtype=torch.bfloat16, device=angles.device)
    cache = Cache4(pages, page_size, kv_heads, head_dim, device=angles.device)
    return AttentionBlock(linear((q_heads + 2 * kv_heads) * head_dim, width), QKNormRope(q_heads, kv_heads, head_dim, angles, wq=norm, wk=norm, rotary=angles.shape[1]),
                          cache, CacheAttention(cache, q_heads), linear(width, q_heads * head_dim))


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("layers", 4), ("requests", 8), ("prompt", 300), ("tokens", 32), ("width", 2048), ("q-heads", 16), ("kv-heads", 4), ("head-dim", 128), ("page-size", 64)):
        p.add_argument("--" + name, type=int, default=default)
    a = p.parse_args()
    generator = torch.Generator().manual_seed(0)
    prompts = [1 + int(n) for n in torch.randint(a.prompt // 2, a.prompt, (a.requests,), generator=generator)]
    longest = max(prompts) + a.tokens
    pages = sum(-(-(n + a.tokens) // a.page_size) for n in prompts)
    angles = rotation_angles(longest, a.head_dim)
    blocks = [random_block(a.width, a.q_heads, a.kv_heads, a.head_dim, pages, a.page_size, angles, generator) for _ in range(a.layers)]

    def run():
        batch = DecodingBatch(blocks, a.requests, longest)
        x = torch.randn(sum(prompts), a.width, generator=generator).to(torch.bfloat16).cuda()
        torch.cuda.synchronize()
        start = time.perf_counter()
        x = batch.step(x, prompts)
        last = torch.tensor(prompts).cumsum(0) - 1
        x = x[last.to(x.device)]
        torch.cuda.synchronize()
        middle = time.perf_counter()
        for _ in range(a.tokens):
            x = batch.step(torch.nn.functional.normalize(x.float(), dim=1).mul_(a.width ** 0.5).to(torch.bfloat16), [1] * a.requests)
        torch.cuda.synchronize()
        return middle - start, time.perf_counter() - middle, x
    run()  # the first launches
    prompt, tokens, x = run()
    if not torch.isfinite(x).all():
        raise RuntimeError("a result is not finite")
    print(f"{a.requests} requests, {a.layers} layers: prompts of {sum(prompts)} tokens {1e3 * prompt:.2f} ms, then {a.tokens} tokens each, {1e3 * tokens / a.tokens:.3f} ms a step "
          f"({1e6 * tokens / a.tokens / a.layers:.1f} us a layer, {a.requests * a.tokens / tokens:.0f} tokens/s)")


if __name__ == "__main__":
    main()
