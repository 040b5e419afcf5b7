"""One step of a small model with quantised weights: every layer as a program runs it with this library.

    python -m paper_2510_06957_amd.decode_step [--tokens 4] [--steps 8]

A token's vector goes through blocks of an 8-bit projection (tst_w8_linear), a ternary layer (tstgemm) and a mixture of experts
(tst_moe), each added to what went in, then through an 8-bit matrix to logits, and tst_logprobs says how likely the most likely next
tokens are.  There is no attention here: a token sees itself alone.  Weights are random; the step is recorded into a graph once and
replayed, the next token being the most likely one.
"""
from __future__ import annotations

import argparse
import math

import torch

import paper_2510_06957_amd as tg


def _norm(x):
    return (x.float() * torch.rsqrt(x.float().pow(2).mean(1, keepdim=True) + 1e-6)).to(x.dtype)


class Model:
    """blocks x (projection width x width, ternary width x width, experts x (width x inner x 3)), vocabulary entries."""

    def __init__(self, blocks=2, width=512, experts=8, inner=256, top_k=2, vocabulary=2000, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def int8(*shape):
            return (torch.randn(shape, generator=g, device="cuda") * 32).round().clamp(-127, 127).to(torch.int8)

        def scale(fan_in, *shape):      # what goes through keeps its size
            return (0.5 + torch.rand(shape, generator=g, device="cuda")) / (32 * math.sqrt(fan_in))

        self.top_k, self.dtype, self.blocks = top_k, dtype, []
        self.embedding = torch.randn((vocabulary, width), generator=g, device="cuda").to(dtype)
        for _ in range(blocks):
            raw = dict(proj=int8(width, width), proj_scale=scale(width, width),
                       ternary=torch.randint(-1, 2, (width, width), generator=g, device="cuda", dtype=torch.int8),
                       router=(torch.randn((experts, width), generator=g, device="cuda") / math.sqrt(width)).to(dtype))
            for name, rows, cols in (("gate", width, inner), ("up", width, inner), ("down", inner, width)):
                raw[name], raw[name + "_scale"] = int8(experts, rows, cols), scale(rows, experts, cols)
            self.blocks.append(dict(
                raw=raw, proj=tg.tst_w8_pack(raw["proj"], raw["proj_scale"]),
                ternary=tg.tcsc_upload(tg.tcsc_build(raw["ternary"].cpu().numpy())),
                moe=tg.tst_moe_pack(*(raw[n] for n in ("router", "gate", "gate_scale", "up", "up_scale", "down", "down_scale")))))
        self.head_raw = (int8(width, vocabulary), scale(width, vocabulary))
        self.head = tg.tst_w8_pack(*self.head_raw)
        self.ternary_scale = math.sqrt(1.5 / width)

    def logits(self, tokens):
        x = self.embedding[tokens]
        for b in self.blocks:
            x = x + tg.tst_w8_linear(_norm(x), b["proj"])
            x = x + (tg.tstgemm(_norm(x).float(), b["ternary"]) * self.ternary_scale).to(self.dtype)
            x = x + tg.tst_moe(_norm(x), b["moe"], self.top_k)[0]
        return tg.tst_w8_linear(_norm(x), self.head)

    def step(self, tokens, top=4):
        """tokens [T] -> (log probabilities, entropy [T], the `top` most likely next tokens [T, top], theirs), of `tokens` themselves
        first."""
        return tg.tst_logprobs(self.logits(tokens), tokens, top=top)


def generate(model, tokens, steps, top=4):
    """[steps, T] most likely tokens, their log probabilities and the entropies, from a step recorded once."""
    model.step(tokens, top)             # what is set up on first use
    torch.cuda.synchronize()
    graph, now = torch.cuda.CUDAGraph(), tokens.clone()
    with torch.cuda.graph(graph):
        _, entropy, ids, of_top = model.step(now, top)
    out = []
    for _ in range(steps):
        graph.replay()
        out.append((ids[:, 0].clone(), of_top[:, 0].clone(), entropy.clone()))
        now.copy_(ids[:, 0])
    return [torch.stack(o) for o in zip(*out)]


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=4)
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args(argv)
    vocabulary = 2000
    if not 1 <= a.tokens <= vocabulary or a.steps < 1:   # an index behind the embedding would end the process on the GPU
        ap.error(f"--tokens takes 1 to {vocabulary}, --steps 1 or more")
    model = Model(vocabulary=vocabulary)
    ids, of_top, entropy = generate(model, torch.arange(a.tokens, device="cuda"), a.steps)
    for s in range(a.steps):
        print(f"step {s}: " + "  ".join(f"{t} (log p {p:.2f}, entropy {h:.2f})" for t, p, h in zip(ids[s].tolist(), of_top[s].tolist(), entropy[s].tolist())))


if __name__ == "__main__":
    main()
