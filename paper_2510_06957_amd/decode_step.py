"""One step of a small model with quantised weights: every layer as a program runs it with this library.

    python -m paper_2510_06957_amd.decode_step [--tokens 4] [--steps 8] [--heads 8 [--prompt 40]]

A token's vector goes through blocks of an 8-bit projection (tst_w8_linear), a ternary layer (tstgemm) and a mixture of experts
(tst_moe), each added to what went in, then through an 8-bit matrix to logits, and tst_logprobs says how likely the most likely next
tokens are.  Weights are random; the step is recorded into a graph once and replayed, the next token being the most likely one.

Without heads a token sees itself alone.  With them each block begins with attention: an 8-bit projection to queries, keys and values, which tst_kv_append rotates
by their positions and keeps in a paged cache of 8-bit codes; a prompt goes through tst_attention at once, each further token through tst_kv_attention over
the cache.
"""
from __future__ import annotations

import argparse
import math

import torch

import paper_2510_06957_amd as tg


def _norm(x):
    return (x.float() * torch.rsqrt(x.float().pow(2).mean(1, keepdim=True) + 1e-6)).to(x.dtype)


class Model:
    """blocks x (projection width x width, ternary width x width, experts x (width x inner x 3)), vocabulary entries.  heads: query heads of
    width / heads entries, four of them (or all) to a head of keys and values; 0: no attention."""

    def __init__(self, blocks=2, width=512, experts=8, inner=256, top_k=2, vocabulary=2000, dtype=torch.bfloat16, seed=0, heads=0):
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
        self.heads, self.kv_heads, self.size = heads, max(1, heads // 4), width // heads if heads else 0
        if heads and (heads % self.kv_heads or not 2 <= self.size <= 256 or self.size % 2):
            raise ValueError("heads must be 1 to 3 or a multiple of 4, of an even number of up to 256 entries")
        for b in self.blocks if heads else ():
            for name, rows, cols in (("qkv", width, (heads + 2 * self.kv_heads) * self.size), ("out", heads * self.size, width)):
                b["raw"][name], b["raw"][name + "_scale"] = int8(rows, cols), scale(rows, cols)
                b[name] = tg.tst_w8_pack(b["raw"][name], b["raw"][name + "_scale"])

    def _attend(self, b, cache, x, memory, offsets, prompt):
        h, g = self.heads, self.kv_heads
        qkv = tg.tst_w8_linear(_norm(x), b["qkv"]).view(-1, h + 2 * g, self.size)
        k, v = qkv[:, h:h + g], qkv[:, h + g:]
        q, k = tg.tst_kv_append(cache, k, v, memory.pages, memory.lens, offsets, Q=qkv[:, :h], cos=memory.cos, sin=memory.sin, keys=True)
        y = tg.tst_attention(q, k, v, offsets) if prompt else tg.tst_kv_attention(q, cache, memory.pages, memory.lens, offsets)
        return tg.tst_w8_linear(y.view(len(x), -1), b["out"])

    def logits(self, tokens, memory=None, offsets=None, prompt=False):
        """tokens [T] -> [T, vocabulary].  memory (of a model with heads): the Memory whose sequences these are the last tokens of, one each or offsets[i] ..
        offsets[i + 1] - 1 of sequence i, counted in memory.lens already; prompt: all that there is of them."""
        x = self.embedding[tokens]
        for i, b in enumerate(self.blocks):
            if memory is not None:
                x = x + self._attend(b, memory.caches[i], x, memory, offsets, prompt)
            x = x + tg.tst_w8_linear(_norm(x), b["proj"])
            x = x + (tg.tstgemm(_norm(x).float(), b["ternary"]) * self.ternary_scale).to(self.dtype)
            x = x + tg.tst_moe(_norm(x), b["moe"], self.top_k)[0]
        return tg.tst_w8_linear(_norm(x), self.head)

    def step(self, tokens, top=4, memory=None):
        """tokens [T] -> (log probabilities, entropy [T], the `top` most likely next tokens [T, top], theirs), of `tokens` themselves
        first."""
        return tg.tst_logprobs(self.logits(tokens, memory), tokens, top=top)


class Memory:
    """What a model with heads keeps of its sequences: a cache for each block, the pages of each sequence, and how many tokens it has."""

    def __init__(self, model, lengths, room, page=32):
        held = [-(-(n + room) // page) for n in lengths]
        pages, at = torch.full((len(lengths), max(held)), -1, dtype=torch.int32), 0
        for i, n in enumerate(held):
            pages[i, :n] = torch.arange(at, at + n)
            at += n
        self.pages, self.lens = pages.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.caches = [tg.tst_kv_cache(at, page, model.kv_heads, model.size) for _ in model.blocks]
        angles = torch.arange(max(lengths) + room, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(model.size // 2, dtype=torch.float64) * 2 / model.size)
        self.cos, self.sin = angles.cos().float().cuda(), angles.sin().float().cuda()


def answer(model, prompts, steps, top=4):
    """prompts: lists of tokens.  The prompts at once, then `steps` tokens for each from a step recorded once: [steps, sequences] most likely tokens, their log
    probabilities and the entropies they were chosen from, beginning with what follows the prompts."""
    lengths, vocabulary = [len(p) for p in prompts], len(model.embedding)
    # a prompt without tokens would be answered from another's last, and an index behind the embedding would end the process on the GPU
    if steps < 1 or not lengths or min(lengths) < 1 or not all(0 <= t < vocabulary for p in prompts for t in p):
        raise ValueError(f"prompts must be lists of at least one token of 0 to {vocabulary - 1}, and steps at least 1")
    memory = Memory(model, lengths, steps + 1)
    offsets = torch.tensor([0] + lengths, dtype=torch.int32).cumsum(0).int().cuda()
    logits = model.logits(torch.tensor([t for p in prompts for t in p], device="cuda"), memory, offsets, prompt=True)
    _, entropy, ids, of_top = tg.tst_logprobs(logits[offsets[1:].long() - 1], top=top)
    now, out = ids[:, 0].long(), [(ids[:, 0], of_top[:, 0], entropy)]
    if steps > 1:
        memory.lens += 1
        model.step(now, top, memory)        # what is set up on first use; the graph appends the same tokens again
        memory.lens -= 1
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            memory.lens += 1
            _, entropy, ids, of_top = model.step(now, top, memory)
        for _ in range(steps - 1):
            graph.replay()
            out.append((ids[:, 0].clone(), of_top[:, 0].clone(), entropy.clone()))
            now.copy_(ids[:, 0])
    return [torch.stack(o) for o in zip(*out)]


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
    ap.add_argument("--heads", type=int, default=0, help="query heads; 0: no attention")
    ap.add_argument("--prompt", type=int, default=40, help="tokens of the longest prompt (with heads)")
    a = ap.parse_args(argv)
    vocabulary = 2000
    if not 1 <= a.tokens <= vocabulary or a.steps < 1:   # an index behind the embedding would end the process on the GPU
        ap.error(f"--tokens takes 1 to {vocabulary}, --steps 1 or more")
    if a.heads not in (0, 2, 4, 8, 16, 32, 64, 128, 256) or not 1 <= a.prompt <= vocabulary - a.tokens + 1:
        ap.error(f"--heads takes 0 and powers of two from 2 to 256, --prompt 1 to {vocabulary - a.tokens + 1}")
    model = Model(vocabulary=vocabulary, heads=a.heads)
    if a.heads:
        prompts = [list(range(i, i + max(1, a.prompt - 3 * i))) for i in range(a.tokens)]
        ids, of_top, entropy = answer(model, prompts, a.steps)
    else:
        ids, of_top, entropy = generate(model, torch.arange(a.tokens, device="cuda"), a.steps)
    for s in range(a.steps):
        print(f"step {s}: " + "  ".join(f"{t} (log p {p:.2f}, entropy {h:.2f})" for t, p, h in zip(ids[s].tolist(), of_top[s].tolist(), entropy[s].tolist())))


if __name__ == "__main__":
    main()
