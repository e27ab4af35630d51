"""Serves a few requests on a small mixture-of-experts model with random weights: prompts first, then one token each a step, until
all have what they asked for.  Every layer is attention over the paged 4-bit cache, then a MoE layer over the resident experts.

    python examples/serve_moe.py [--steps N]

What is not the library's (projections, norms, rotary positions, the choice of the next token) is plain torch.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2503_06823_amd as P  # noqa: E402

DEVICE = "cuda:0"


class Model:
    """Random weights, four of eight experts resident in every layer."""

    def __init__(self, layers=2, d=512, q_heads=8, kv_heads=2, head_dim=64, d_ff=1024, experts=8, resident=4, top_k=2, vocab=1000, seed=1):
        self.layers, self.d, self.q_heads, self.kv_heads, self.head_dim = layers, d, q_heads, kv_heads, head_dim
        self.d_ff, self.experts, self.resident, self.top_k = d_ff, experts, resident, top_k
        g = torch.Generator(device=DEVICE)
        g.manual_seed(seed)

        def normal(*shape, std):
            return torch.empty(shape, dtype=torch.bfloat16, device=DEVICE).normal_(0.0, std, generator=g)

        self.embedding, self.head = normal(vocab, d, std=1.0), normal(vocab, d, std=d ** -0.5)
        self.blocks = []
        for _ in range(layers):
            slots = torch.full((experts,), -1, dtype=torch.int32, device=DEVICE)
            slots[torch.randperm(experts, generator=g, device=DEVICE)[:resident]] = torch.arange(resident, dtype=torch.int32, device=DEVICE)
            self.blocks.append(dict(
                qkv=normal((q_heads + 2 * kv_heads) * head_dim, d, std=d ** -0.5), out=normal(d, q_heads * head_dim, std=d ** -0.5),
                moe=(normal(experts, d, std=d ** -0.5), None, slots, normal(resident, d_ff, d, std=d ** -0.5),
                     normal(resident, d_ff, d, std=d ** -0.5), normal(resident, d, d_ff, std=d_ff ** -0.5))))
        self.buffers = {}

    def moe(self, block, x):
        T = x.shape[0]
        if T not in self.buffers:  # once per batch size
            self.buffers[T] = P.LayerBuffers.allocate(
                P.make_desc(T, self.d, self.d_ff, self.experts, self.top_k, self.resident, "bf16", "swiglu"), DEVICE)
        return P.layer_forward(self.buffers[T], x, *block["moe"], one_call=True)

    def forward(self, kv, tokens, max_new):
        """Logits [T, vocab] of a step's tokens, for which `kv` has been planned."""
        T, q, k, n = tokens.shape[0], self.q_heads, self.kv_heads, self.head_dim
        x = self.embedding[tokens]
        angle = kv.position[:T, None].float() * 10000.0 ** (-torch.arange(0, n, 2, device=DEVICE) / n)
        cos, sin = angle.cos()[:, None], angle.sin()[:, None]
        for i, block in enumerate(self.blocks):
            heads = (norm(x) @ block["qkv"].t()).view(T, q + 2 * k, n)
            rotate(heads[:, :q + k], cos, sin)
            kv.append(i, heads[:, q:q + k], heads[:, q + k:])
            attended = kv.attend(i, heads[:, :q], torch.empty((T, q, n), dtype=x.dtype, device=DEVICE), max_new)
            x = x + attended.view(T, q * n) @ block["out"].t()
            x = x + self.moe(block, norm(x))
        return norm(x) @ self.head.t()


def norm(x):
    y = x.float()
    return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


def rotate(heads, cos, sin):
    """Rotary positions, in place: halves of a head's row are the two coordinates."""
    a, b = heads.float().chunk(2, -1)
    heads.copy_(torch.cat((a * cos - b * sin, a * sin + b * cos), -1))


def serve(model, prompts, steps, window=0, sinks=0, pages=None):
    """`prompts`: a list of token lists; row r generates steps - r tokens, so that requests end one after the other.  `pages`: of the cache, if
    not enough for all; requests that get none then wait until others have ended.  Returns the tokens of every request and the cache."""
    R, longest = len(prompts), max(map(len, prompts))
    page = 16
    width = -(-(longest + steps) // page)
    kv = P.KvCache.allocate(model.layers, R, longest + steps, pages or R * width, page, model.kv_heads, model.head_dim,
                            max(sum(map(len, prompts)), R), window=window, sinks=sinks, device=DEVICE)
    i32 = dict(dtype=torch.int32, device=DEVICE)
    made = [[] for _ in prompts]
    pending = [list(p) for p in prompts]  # what each request brings to the next step; nothing: it has ended
    while any(pending):
        new = [len(p) for p in pending]
        tokens = torch.tensor(sum(pending, []), dtype=torch.int64, device=DEVICE)
        kv.plan(torch.tensor(new, **i32), len(tokens))
        logits = model.forward(kv, tokens, max(new))
        running = [r for r in range(R) if new[r]]
        chosen = logits[torch.tensor([sum(new[:r + 1]) - 1 for r in running], device=DEVICE)].argmax(-1)
        held = kv.length[1].tolist()
        ended = [0] * R
        for r, t in zip(running, chosen.tolist()):
            if held[r] == 0:  # refused: there was no page for it, and it brings the same tokens again
                continue
            made[r].append(t)
            ended[r] = int(len(made[r]) >= steps - r)
            pending[r] = [] if ended[r] else [t]
        if not any(held[r] for r in running):
            raise RuntimeError(f"{kv.desc.pages} pages are too few: none of requests {running} can go on")
        kv.release(torch.tensor(ended, **i32))
    return made, kv


def main():
    parser = argparse.ArgumentParser()
    parser.add_argument("--steps", type=int, default=24)
    steps = max(parser.parse_args().steps, 6)
    model = Model()
    g = torch.Generator().manual_seed(2)
    prompts = [torch.randint(0, 1000, (n,), generator=g).tolist() for n in (5, 130, 37, 1)]
    serve(model, prompts, steps)  # builds the buffers
    torch.cuda.synchronize()
    begin = time.perf_counter()
    made, kv = serve(model, prompts, steps, window=64, sinks=4)
    torch.cuda.synchronize()
    spent = time.perf_counter() - begin
    head, tail = kv.counters[0].tolist()
    print(f"{sum(map(len, made))} tokens of {len(prompts)} requests in {spent * 1e3:.1f} ms; {tail - head} of {kv.desc.pages} pages are free again")
    for r, m in enumerate(made):
        print(f"request {r}: prompt of {len(prompts[r])}, then {m[:8]}{' ...' if len(m) > 8 else ''}")


if __name__ == "__main__":
    main()
