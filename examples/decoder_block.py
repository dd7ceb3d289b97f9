"""A decoder block served with LQER linears: prompts, then tokens one by one, each request with an adapter of its own.

    python examples/decoder_block.py

What a step runs, all on one stream and without a synchronisation:

    lqer_rmsnorm_mx            residual + the previous block's output, norm, X_q of q, k and v (and its values for the adapters)
    lqer_linear_forward_q      q, k, v
    lqer_adapters_forward      the requests' adapters on q
    lqer_kv4_append            k and v into the 4-bit cache
    lqer_kv4_attention         the step's queries over it
    lqer_linear_forward        o
    lqer_rmsnorm_mx            residual + o, norm, X_q of gate and up
    lqer_linear_forward_q      gate, up
    lqer_linear_forward        down, from silu(gate) * up

Weights are random; rotary positions and the activation function are torch operations here.
"""
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2402_02446_amd import binding as lqer, synth  # noqa: E402

DEV = "cuda"


class Cache:
    """Pages of one block's keys and values, and which request has which."""

    def __init__(self, pages, kv_heads, page_tokens, head_dim, requests, most_tokens):
        self.pool = lqer.lqer_kv4_pool(pages, kv_heads, page_tokens, head_dim)
        self.page_tokens, self.free = page_tokens, list(range(pages))
        self.table = np.full((requests, -(-most_tokens // page_tokens)), -1, np.int32)
        self.lengths = np.zeros(requests, np.int64)

    def take(self, new):
        """Room for new[b] more tokens of request b: their positions and slots, and what the attention wants to know."""
        positions, slots = [], []
        for b, n in enumerate(new):
            end = self.lengths[b] + n
            for i in range(-(-self.lengths[b] // self.page_tokens), -(-end // self.page_tokens)):
                self.table[b, i] = self.free.pop()
            p = np.arange(self.lengths[b], end)
            positions.append(p)
            slots.append(self.table[b, p // self.page_tokens] * self.page_tokens + p % self.page_tokens)
            self.lengths[b] = end
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.int32)).to(DEV)  # noqa: E731
        return dict(positions=dev(np.concatenate(positions)), slots=dev(np.concatenate(slots)), cu_q=dev(np.cumsum([0] + list(new))),
                    kv_len=dev(self.lengths), table=dev(self.table), max_q=int(max(new)), max_kv=int(self.lengths.max()))


def rotate(x, positions):
    """Rotary positions on [tokens][heads][head_dim]."""
    half = x.shape[-1] // 2
    angle = positions[:, None].float() * 10000.0 ** (-torch.arange(half, device=x.device) / half)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


class Block:
    def __init__(self, hidden=512, mlp=1024, q_heads=8, kv_heads=2, head_dim=64, k=16, adapters=3, adapter_rank=8, seed=0):
        rng = np.random.default_rng(seed)
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self.scale = head_dim ** -0.5

        def layer(K, N):
            W = rng.standard_normal((K, N), dtype=np.float32) * np.float32(K ** -0.5)
            calib = synth.gen_activations(rng, 64, K, synth.gen_outlier_channels(rng, K, k), 30.0)[None]
            return lqer.lqer_build_factors(W, calib, k)
        self.q, self.k, self.v = layer(hidden, q_heads * head_dim), layer(hidden, kv_heads * head_dim), layer(hidden, kv_heads * head_dim)
        self.o = layer(q_heads * head_dim, hidden)
        self.gate, self.up, self.down = layer(hidden, mlp), layer(hidden, mlp), layer(mlp, hidden)
        bf16 = lambda *s: torch.from_numpy(rng.standard_normal(s, dtype=np.float32)).to(DEV).bfloat16()  # noqa: E731
        self.norm1, self.norm2 = 1 + 0.1 * bf16(hidden), 1 + 0.1 * bf16(hidden)
        self.A = bf16(adapters, adapter_rank, hidden) * hidden ** -0.5
        self.B = bf16(adapters, q_heads * head_dim, adapter_rank) * 0.1

    def step(self, x, residual, cache, at, ids):
        """x, residual fp32 [tokens][hidden]: the previous block's output and the stream it is added to; at: what cache.take gave; ids: every
        token's adapter.  Returns this block's x and residual."""
        codes, exps, residual, values = lqer.lqer_rmsnorm_mx(x, self.norm1, residual=residual, values=True)
        q, k, v = (lqer.lqer_linear_forward_q(layer, codes, exps) for layer in (self.q, self.k, self.v))
        lqer.lqer_adapters_forward(values, ids, self.A, self.B, q)
        heads = lambda t: t.view(t.shape[0], -1, self.head_dim)  # noqa: E731
        lqer.lqer_kv4_append(cache.pool, rotate(heads(k), at["positions"]), heads(v), at["slots"])
        out = torch.empty(q.shape[0], self.q_heads, self.head_dim, device=DEV)
        lqer.lqer_kv4_attention(cache.pool, rotate(heads(q), at["positions"]).bfloat16(), at["cu_q"], at["kv_len"], at["table"], at["max_q"],
                                at["max_kv"], self.scale, out=out)
        x = lqer.lqer_linear_forward(self.o, out.flatten(1))
        codes, exps, residual, _ = lqer.lqer_rmsnorm_mx(x, self.norm2, residual=residual)
        gate, up = (lqer.lqer_linear_forward_q(layer, codes, exps) for layer in (self.gate, self.up))
        return lqer.lqer_linear_forward(self.down, torch.nn.functional.silu(gate) * up), residual


def main():
    torch.manual_seed(0)
    block = Block()
    prompts, adapters = [37, 150, 1], torch.tensor([2, -1, 0], dtype=torch.int32, device=DEV)     # request 1 has no adapter
    cache = Cache(64, block.kv_heads, 16, block.head_dim, len(prompts), 256)
    x = torch.randn(sum(prompts), 512, device=DEV)
    ids = adapters.repeat_interleave(torch.tensor(prompts, device=DEV))
    y, residual = block.step(x, torch.zeros_like(x), cache, cache.take(prompts), ids)
    print("prompts:", prompts, "-> block output", tuple(y.shape), "rms %.3f" % float((y + residual).square().mean().sqrt()))
    last = torch.tensor(prompts, device=DEV).cumsum(0) - 1
    x, steps = (y + residual)[last].contiguous(), 32
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(steps):
        y, residual = block.step(x, torch.zeros_like(x), cache, cache.take([1] * len(prompts)), adapters)
        x = torch.tanh(y + residual)
    torch.cuda.synchronize()
    print("%d decode steps of %d requests: %.0f us a step, cached tokens now %s" %
          (steps, len(prompts), (time.perf_counter() - began) / steps * 1e6, cache.lengths.tolist()))


if __name__ == "__main__":
    main()
