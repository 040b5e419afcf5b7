"""The example with attention (paper_2510_06957_amd/decode_step.py): prompts, then tokens over the cache, against the same model in 64 bits."""
import math

import numpy as np
import pytest
import torch

import kv_reference as ref

pytestmark = pytest.mark.gpu


def reference(model, sequences, prompts, page=32):
    """Logits in 64 bits of the last tokens: sequences (lists of tokens) of which prompts[i] came at once and the others one by one, over a cache that is kept as the
    definition says.  Codes of 8-bit layers are rounded as the layer rounds them."""
    h, g, size = model.heads, model.kv_heads, model.size

    def norm(x):
        return x * (x.pow(2).mean(1, keepdim=True) + 1e-6).rsqrt()

    def linear(x, W, scale):
        s = x.abs().amax(1, keepdim=True) / 127
        return (x / s).round() @ W.cpu().double() * s * scale.cpu().double()

    pairs = size // 2
    angles = np.arange(4096)[:, None] * 10000.0 ** (-np.arange(pairs) * 2 / size)
    cos, sin = np.cos(angles).astype(np.float32), np.sin(angles).astype(np.float32)
    out = []
    for tokens, prompt in zip(sequences, prompts):
        table = np.arange(-(-len(tokens) // page))[None]
        caches = [ref.Cache(table.shape[1], page, g, size) for _ in model.blocks]
        for first, n in [(0, prompt)] + [(i, 1) for i in range(prompt, len(tokens))]:
            x = model.embedding[torch.tensor(tokens[first:first + n])].cpu().double()
            for cache, b in zip(caches, model.blocks):
                r = {k: t.cpu().double() for k, t in b["raw"].items()}
                qkv = linear(norm(x), b["raw"]["qkv"], r["qkv_scale"]).float().numpy().reshape(n, h + 2 * g, size)
                position = np.arange(first, first + n)
                q, k = (ref.rotate(qkv[:, a:e], position, cos, sin, False) for a, e in ((0, h), (h, h + g)))
                v = qkv[:, h + g:]
                cache.append("k", k, table, 0, first)
                cache.append("v", v, table, 0, first)
                if first:     # further tokens see the codes, a prompt sees itself
                    k, v = (cache.values(name, table, 0, 0, first + n) for name in "kv")
                y = np.stack([ref.attention(q[:, i].astype(np.float64), k[:, i // (h // g)].astype(np.float64), v[:, i // (h // g)].astype(np.float64), position + 1,
                                            1 / math.sqrt(size), 0)[0] for i in range(h)], 1)
                x = x + linear(torch.from_numpy(y.reshape(n, -1)), b["raw"]["out"], r["out_scale"])
                x = x + linear(norm(x), b["raw"]["proj"], r["proj_scale"])
                x = x + norm(x) @ r["ternary"] * model.ternary_scale
                u = norm(x)
                most, ids = (u @ r["router"].t()).topk(model.top_k, dim=1)
                p, z = most.softmax(1), torch.zeros_like(x)
                for t in range(n):
                    for j, e in enumerate(ids[t].tolist()):
                        a, c = (u[t] @ r["gate"][e]) * r["gate_scale"][e], (u[t] @ r["up"][e]) * r["up_scale"][e]
                        z[t] += p[t, j] * ((a * a.sigmoid() * c) @ r["down"][e]) * r["down_scale"][e]
                x = x + z
        out.append(linear(norm(x), *model.head_raw)[-1])
    return torch.stack(out)


def test_prompts_and_steps_are_the_model():
    """fp32 activations.  As without attention, what differs is a code rounded the other way now and then, half a step of 1 / 127 of a token's largest entry in one of 512,
    which moves a logit by less than 1 / 100 of its spread for three such layers; here there are seven, and the cache's codes beside them, of one entry in 64: 1 / 30."""
    from paper_2510_06957_amd.decode_step import Memory, Model
    model = Model(dtype=torch.float32, seed=5, heads=8)
    r = np.random.default_rng(5)
    lengths = [37, 1, 64]
    sequences = [r.integers(0, 2000, n + 18).tolist() for n in lengths]
    memory = Memory(model, lengths, 18)
    offsets = torch.tensor([0, 37, 38, 102], dtype=torch.int32, device="cuda")
    tokens = torch.tensor([t for s, n in zip(sequences, lengths) for t in s[:n]], device="cuda")
    got = [model.logits(tokens, memory, offsets, prompt=True)[[36, 37, 101]]]
    for step in range(18):
        memory.lens += 1
        got.append(model.logits(torch.tensor([s[n + step] for s, n in zip(sequences, lengths)], device="cuda"), memory))
    for step in (0, 1, 18):
        want = reference(model, [s[:n + step] for s, n in zip(sequences, lengths)], lengths)
        assert ((got[step].cpu().double() - want).abs().max(1).values < want.std(1) * math.sqrt(10) / 30).all()


def test_answers_from_a_graph_are_step_by_step():
    from paper_2510_06957_amd.decode_step import Memory, Model, answer
    import paper_2510_06957_amd as tg
    model = Model(seed=6, heads=8)
    prompts = [[5, 900, 1999] * 11, [7], list(range(50))]
    ids, of_top, entropy = answer(model, prompts, 20)
    assert ids.shape == (20, 3)
    lengths = [len(p) for p in prompts]
    memory = Memory(model, lengths, 21)
    offsets = torch.tensor([0, 33, 34, 84], dtype=torch.int32, device="cuda")
    logits = model.logits(torch.tensor(sum(prompts, []), device="cuda"), memory, offsets, prompt=True)[[32, 33, 83]]
    _, h, best, p = tg.tst_logprobs(logits, top=4)
    for s in range(20):
        assert torch.equal(best[:, 0], ids[s]) and torch.equal(p[:, 0], of_top[s]) and torch.equal(h, entropy[s])
        memory.lens += 1
        _, h, best, p = model.step(best[:, 0].long(), memory=memory)


def test_a_model_without_heads_is_what_it_was():
    """The weights that a seed gives do not depend on whether there are heads."""
    from paper_2510_06957_amd.decode_step import Model
    a, b = Model(seed=7), Model(seed=7, heads=4)
    tokens = torch.tensor([3, 1500], device="cuda")
    assert torch.equal(a.logits(tokens), b.logits(tokens))
    with pytest.raises(ValueError):
        Model(heads=6)


def test_the_command(capsys):
    from paper_2510_06957_amd import decode_step
    decode_step.main(["--heads", "8", "--tokens", "3", "--steps", "4", "--prompt", "9"])
    assert len([line for line in capsys.readouterr().out.splitlines() if line.startswith("step ")]) == 4
    for argv in (["--heads", "3"], ["--heads", "512"], ["--heads", "8", "--prompt", "0"], ["--heads", "8", "--prompt", "2000"]):
        with pytest.raises(SystemExit):
            decode_step.main(argv)
