"""The operators with which a token sees the tokens before it, whose speed matters to a program that answers with a quantised
model: appending keys and values to a paged cache of 8-bit codes with the position rotation on the way ("append", with what the
touched blocks then stand for read back), attention of new tokens over that cache ("cached"), and causal attention over whole
prompts packed one behind another ("prompt").

A scale belongs to a block of 16 tokens and a head.  Keys have a few large channels, queries agree with one of the keys they see,
as trained heads do; pages lie in the order an allocator that has run for a while gives them.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 16                                  # tokens that share a scale
LARGEST_PROMPT = 32 * 128 * 8192 ** 2       # heads * head size * sum of squared lengths
LARGEST_CACHED = 175000 * 8 * 128           # tokens * key heads * head size
LARGEST_APPEND = 6912 * 48 * 128            # tokens * all heads * head size


def _append(S, new, lens, heads, kv_heads, size, page, dtype, rotary, interleaved=False):
    # S sequences; each has up to lens tokens behind the call, and up to new of them come with it
    return dict(kind="append", S=S, new=new, lens=lens, heads=heads, kv_heads=kv_heads, size=size, page=page, dtype=dtype, rotary=rotary,
                interleaved=interleaved)


def _cached(S, new, lens, heads, kv_heads, size, page, dtype):
    return dict(kind="cached", S=S, new=new, lens=lens, heads=heads, kv_heads=kv_heads, size=size, page=page, dtype=dtype)


def _prompt(S, lens, heads, kv_heads, size, dtype):
    return dict(kind="prompt", S=S, lens=lens, heads=heads, kv_heads=kv_heads, size=size, dtype=dtype)


def listed():
    cases = {
        # the first token of one answer of a small model: latency
        "append-1": _append(1, 1, 100, 8, 2, 64, 16, "f16", 64),
        # a batch of answers, a token each
        "append-64": _append(64, 1, 8192, 32, 8, 128, 64, "bf16", 128),
        # prompts that have just come in
        "append-prompts": _append(4, 4096, 4096, 32, 8, 128, 64, "bf16", 128),
        # drafts and pieces of prompts, odd sizes, 32 bits, a part of each head rotated in neighbouring pairs
        "append-ragged": _append(7, 61, 700, 10, 5, 80, 32, "f32", 32, True),
        # one token of a short answer: latency
        "cached-1": _cached(1, 1, 200, 32, 8, 128, 64, "f16"),
        # one token behind a whole book
        "cached-1-long": _cached(1, 1, 131072, 32, 8, 128, 64, "bf16"),
        # a batch of answers of all lengths
        "cached-64": _cached(64, 1, 8192, 32, 8, 128, 64, "bf16"),
        # drafts of a few tokens that are to be verified, odd sizes, 32 bits
        "cached-draft-ragged": _cached(11, 5, 1531, 15, 5, 80, 32, "f32"),
        # a question
        "prompt-37": _prompt(1, 37, 32, 8, 128, "bf16"),
        # a batch of prompts of all lengths
        "prompt-packed": _prompt(24, 2048, 32, 8, 128, "bf16"),
        # a document
        "prompt-8192": _prompt(1, 8192, 32, 8, 128, "bf16"),
        # a few short prompts, odd sizes, 32 bits
        "prompt-ragged": _prompt(5, 531, 9, 3, 80, "f32"),
    }
    return [dict(case, name=name) for name, case in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One to 128 sequences of 1 to 131072 tokens (prompts: 1 to 8192), 1 to 16 key heads with 1 to 16 queries' heads each, head sizes of 32
    to 256, pages of 16 to 256 tokens; 1 to 8 new tokens over a cache, 1 to 8192 into one."""
    kind = rng.choice(["append", "cached", "prompt"])
    while True:
        kv_heads = _log_int(rng, 1, 16)
        heads = kv_heads * rng.choice([1, 2, 3, 4, 4, 7, 8, 16])
        size = rng.choice([64, 128, 128, 128, 192, 256, 8 * rng.randint(4, 32)])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        page = rng.choice([16, 32, 64, 128, 256])
        S = _log_int(rng, 1, 128)
        if heads > 64:
            continue
        if kind == "prompt":
            lens = _log_int(rng, 1, 8192)
            if S <= 32 and heads * size * S * lens ** 2 <= LARGEST_PROMPT and S * lens <= 16384:
                return _prompt(S, lens, heads, kv_heads, size, dtype)
        elif kind == "cached":
            lens = _log_int(rng, 1, 131072)
            case = _cached(S, min(lens, rng.choice([1, 1, 1, rng.randint(2, 8)])), lens, heads, kv_heads, size, page, dtype)
            if sum(_lengths(case)[0]) * kv_heads * size <= LARGEST_CACHED:
                return case
        else:
            new = 1 if rng.random() < 0.4 else _log_int(rng, 1, 8192)
            lens = max(new, _log_int(rng, 1, 16384))
            case = _append(S, new, lens, heads, kv_heads, size, page, dtype, rng.choice([size, size, size // 4 * 2]), rng.random() < 0.25)
            all_lens, all_new = _lengths(case)
            if sum(all_new) * (heads + 2 * kv_heads) * size <= LARGEST_APPEND and sum(all_lens) * kv_heads * size <= LARGEST_CACHED:
                return case


def _lengths(case):
    """(lengths behind the call, new tokens) of the sequences: the longest first, then all the way down, as spread as answers are."""
    S, most, new = case["S"], case["lens"], case.get("new", 0)
    lens = [max(1, round(most * (1 - i / S) ** 2)) for i in range(S)]
    n = [max(1, min(lens[i], new - (i * 5 % 7) * new // 8)) if i else min(most, new) for i in range(S)]
    return lens, n


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _keys(n, case, g):
    K = torch.randn((n, case["kv_heads"], case["size"]), generator=g, device="cuda")
    K[:, :, torch.randint(0, case["size"], (2,), generator=g, device="cuda")] *= 4
    return K


def _coded(x, kv_heads, size):
    """Blocks [n, 16, heads, size] -> codes int8 [n, heads, 16, size], scales [n, heads]."""
    x = x.permute(0, 2, 1, 3)
    s = x.abs().amax((2, 3)) / 127
    return (x / s[:, :, None, None]).round().to(torch.int8), s


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 31)
    heads, kv_heads, size, dtype = case["heads"], case["kv_heads"], case["size"], TYPES[case["dtype"]]
    lens, new = _lengths(case)
    if case["kind"] == "prompt":
        starts = _starts(lens)
        T = starts[-1]
        qkv = torch.empty((T, heads + 2 * kv_heads, size), dtype=dtype, device="cuda")      # as one projection leaves them
        K = _keys(T, case, g)
        for a, b in zip(starts, starts[1:]):
            seen = a + (torch.rand(b - a, generator=g, device="cuda") * torch.arange(1, b - a + 1, device="cuda")).long()
            qkv[a:b, :heads] = (torch.randn((b - a, heads, size), generator=g, device="cuda")
                                + 0.6 * K[seen].repeat_interleave(heads // kv_heads, 1)).to(dtype)
        qkv[:, heads:heads + kv_heads] = K.to(dtype)
        qkv[:, heads + kv_heads:] = torch.randn((T, kv_heads, size), generator=g, device="cuda").to(dtype)
        return dict(qkv=qkv, starts=starts, offsets=_int32(starts))
    per_page = case["page"] // BLOCK
    held = [-(-n // case["page"]) for n in lens]
    count = sum(held) + 3                     # some pages belong to nobody
    order = torch.randperm(count, generator=g, device="cuda").to(torch.int32)
    pages = torch.full((len(lens), max(held) + 1), -1, dtype=torch.int32, device="cuda")
    for i, (a, n) in enumerate(zip(_starts(held), held)):
        pages[i, :n] = order[a:a + n]
    d = dict(pages=pages, lens=_int32(lens), offsets=_int32(_starts(new)) if max(new) > 1 else None, T=sum(new))
    for name in "kv":                         # blocks as they lie in the pages, heads first
        codes = torch.empty((count * per_page, kv_heads, BLOCK, size), dtype=torch.int8, device="cuda")
        scale = torch.empty((count * per_page, kv_heads), device="cuda")
        for at in range(0, len(codes), 2048):
            n = min(2048, len(codes) - at)
            x = _keys(n * BLOCK, case, g) if name == "k" else torch.randn((n * BLOCK, kv_heads, size), generator=g, device="cuda")
            codes[at:at + n], scale[at:at + n] = _coded(x.view(n, BLOCK, kv_heads, size), kv_heads, size)
        d[name + "_codes"], d[name + "_scale"] = codes, scale
    seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), torch.tensor(new, device="cuda"))
    if case["kind"] == "cached":
        at = (torch.rand(d["T"], generator=g, device="cuda") * (d["lens"] - torch.tensor(new, device="cuda") + 1)[seq]).long()
        block = pages[seq, at // case["page"]].long() * per_page + at % case["page"] // BLOCK
        key = d["k_codes"][block, :, at % BLOCK].float() * d["k_scale"][block][:, :, None]
        d["Q"] = (torch.randn((d["T"], heads, size), generator=g, device="cuda") + 0.6 * key.repeat_interleave(heads // kv_heads, 1)).to(dtype)
        return d
    qkv = torch.randn((d["T"], heads + 2 * kv_heads, size), generator=g, device="cuda")
    qkv[:, heads:heads + kv_heads] = 1.1 * _keys(d["T"], case, g)     # now and then larger than what is there
    d["qkv"] = qkv.to(dtype)
    rates = 10000.0 ** (-torch.arange(case["rotary"] // 2, dtype=torch.float64, device="cuda") * 2 / case["rotary"])
    angles = torch.arange(max(lens), dtype=torch.float64, device="cuda")[:, None] * rates
    d["cos"], d["sin"] = angles.cos().float(), angles.sin().float()
    # read back: everything of the blocks that the call touched
    back = [n - (n - m) // BLOCK * BLOCK for n, m in zip(lens, new)]
    d["back"], d["back_offsets"] = sum(back), _int32(_starts(back))
    return d


def prepare(case, seed):
    d = _inputs(case, seed)
    state = dict(d, case=case)
    if case["kind"] == "prompt":
        state["bounds"] = list(zip(d["starts"], d["starts"][1:]))
    elif own:
        import paper_2510_06957_amd as tg
        per_page, size = case["page"] // BLOCK, case["size"]
        count = len(d["k_codes"]) // per_page
        cache = tg.tst_kv_cache(count, case["page"], case["kv_heads"], size)
        k = state.pop("k_codes").view(count, per_page, case["kv_heads"], BLOCK, size).transpose(1, 2)
        cache.k_codes[..., :size] = k.reshape(count, case["kv_heads"], case["page"], size)
        v = state.pop("v_codes").view(count, per_page, case["kv_heads"], BLOCK, size).transpose(1, 2)
        cache.v_codes[..., :size, :] = v.transpose(3, 4)
        cache.k_scale.copy_(state.pop("k_scale").view(count, per_page, -1).transpose(1, 2))
        cache.v_scale.copy_(state.pop("v_scale").view(count, per_page, -1).transpose(1, 2))
        state["cache"] = cache
    return state


def _run_own(s):
    import paper_2510_06957_amd as tg
    case = s["case"]
    h, g = case["heads"], case["kv_heads"]
    if case["kind"] == "prompt":
        x = s["qkv"]
        return tg.tst_attention(x[:, :h], x[:, h:h + g], x[:, h + g:], s["offsets"])
    if case["kind"] == "cached":
        return tg.tst_kv_attention(s["Q"], s["cache"], s["pages"], s["lens"], s["offsets"])
    x = s["qkv"]
    Q, K = tg.tst_kv_append(s["cache"], x[:, h:h + g], x[:, h + g:], s["pages"], s["lens"], s["offsets"], Q=x[:, :h], cos=s["cos"], sin=s["sin"],
                            interleaved=case["interleaved"], keys=True)
    return Q, K, *tg.tst_kv_read(s["cache"], s["pages"], s["lens"], s["back"], s["back_offsets"], dtype=x.dtype)


def run(state):
    """prompt, cached: Y.  append: rotated queries and keys, then the values of the blocks that the new tokens went into, keys and values."""
    if own:
        return _run_own(state)
    return {"prompt": _plain_prompt, "cached": _plain_cached, "append": _plain_append}[state["case"]["kind"]](state)


def _softmax_product(z, V):
    """z: logits with -inf where there is nothing to see.  Rows without any are zeros."""
    m = z.amax(-1, keepdim=True)
    e = (z - torch.where(m == -math.inf, torch.zeros_like(m), m)).exp()
    total = e.sum(-1, keepdim=True)
    return (e @ V) / torch.where(total == 0, torch.ones_like(total), total)


def _plain_prompt(s):
    h, g, size = (s["case"][n] for n in ("heads", "kv_heads", "size"))
    Y = torch.empty((len(s["qkv"]), h, size), device="cuda")
    for a, b in s["bounds"]:
        n = b - a
        x = s["qkv"][a:b].float().transpose(0, 1)
        z = (x[:h].reshape(g, h // g * n, size) @ x[h:h + g].transpose(1, 2).contiguous()) * (1 / math.sqrt(size))
        i = torch.arange(n, device="cuda")
        z = torch.where((i[None, :] <= i[:, None]).repeat(h // g, 1), z, -math.inf)
        Y[a:b] = _softmax_product(z, x[h + g:].contiguous()).view(h, n, size).transpose(0, 1)
    return Y.to(s["qkv"].dtype)


def _places(s, offsets, T):
    """(sequence, position) of packed rows that are the last ones of their sequences."""
    lens = s["lens"].long()
    t = torch.arange(T, device="cuda")
    if offsets is None:
        return t, lens - 1
    ends = offsets[1:].long()
    seq = torch.bucketize(t, ends, right=True)
    return seq, lens[seq] - ends[seq] + t


def _block_of(s, seq, at):
    page = s["case"]["page"]
    return s["pages"][seq, at // page].long() * (page // BLOCK) + at % page // BLOCK


def _plain_cached(s):
    case = s["case"]
    h, g, size, S = case["heads"], case["kv_heads"], case["size"], len(s["lens"])
    T, longest = s["T"], case["lens"]
    seq, at = _places(s, s["offsets"], T)
    n = case["new"]
    behind = s["lens"].long()[seq] - 1 - at                     # a row's place from the end, in rows padded to the longest draft
    Q = torch.zeros((S, n, h, size), device="cuda")
    Q[seq, behind] = s["Q"].float()
    j = torch.arange(-(-longest // BLOCK) * BLOCK, device="cuda")
    blocks = s["pages"][:, j[::BLOCK] // case["page"]].long().clamp_(min=0) * (case["page"] // BLOCK) + j[::BLOCK] % case["page"] // BLOCK

    def values(name):                                           # [S, g, longest, size]
        x = s[name + "_codes"][blocks].float() * s[name + "_scale"][blocks][:, :, :, None, None]
        return x.transpose(1, 2).reshape(S, g, -1, size)

    z = (Q.view(S, n, g, h // g, size).permute(0, 2, 1, 3, 4).reshape(S, g, -1, size) @ values("k").transpose(2, 3).contiguous()) * (1 / math.sqrt(size))
    last = s["lens"].long()[:, None] - 1 - torch.arange(n, device="cuda")
    seen = (j <= last[:, :, None])[:, None, :, None].expand(S, g, n, h // g, len(j)).reshape(S, g, -1, len(j))
    Y = _softmax_product(torch.where(seen, z, -math.inf), values("v"))
    Y = Y.view(S, g, n, h // g, size).permute(0, 2, 1, 3, 4).reshape(S, n, h, size)
    return Y[seq, behind].to(s["Q"].dtype)


def _rotated(x, cos, sin, interleaved):
    """x [T, heads, size] in 32 bits; cos, sin [T, pairs]."""
    pairs = cos.shape[1]
    c, s = cos[:, None], sin[:, None]
    y = x.clone()
    a, b = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
    y[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
    y[:, :, b] = x[:, :, b] * c + x[:, :, a] * s
    return y


def _plain_append(s):
    case = s["case"]
    h, g = case["heads"], case["kv_heads"]
    x = s["qkv"].float()
    seq, at = _places(s, s["offsets"], s["T"])
    cos, sin = s["cos"][at], s["sin"][at]
    Q, K = _rotated(x[:, :h], cos, sin, case["interleaved"]), _rotated(x[:, h:h + g], cos, sin, case["interleaved"])
    block = _block_of(s, seq, at)
    starts = torch.arange(s["T"], device="cuda") if s["offsets"] is None else s["offsets"][:-1].long()
    first = at[starts]                                          # of each sequence's new tokens: only its block can hold older ones
    old = block[starts]
    there = first % BLOCK
    for name, y in (("k", K), ("v", x[:, h + g:])):
        codes, scale = s[name + "_codes"], s[name + "_scale"]
        before = scale[old]
        most = torch.zeros_like(scale).index_reduce_(0, block, y.abs().amax(2), "amax")
        seven = torch.full_like(most, 127)
        grown = most / seven
        grown[old] = torch.where((there > 0)[:, None], torch.maximum(before, grown[old]), grown[old])
        scale[block] = grown[block]
        now = scale[old]
        share = torch.where(now > 0, before / now, torch.ones_like(now))
        kept = torch.where((share == 1)[:, :, None, None], codes[old], (codes[old].float() * share[:, :, None, None]).round().to(torch.int8))
        older = torch.arange(BLOCK, device="cuda") < there[:, None]
        codes[old] = torch.where(older[:, None, :, None], kept, codes[old])
        inverse = (torch.ones_like(scale) / scale).clamp(max=torch.finfo(torch.float32).max)[block]
        codes[block, :, at % BLOCK] = (y * inverse[:, :, None]).round().clamp(-127, 127).to(torch.int8)
    seq, at = _places(s, s["back_offsets"], s["back"])
    block = _block_of(s, seq, at)
    back = [s[n + "_codes"][block, :, at % BLOCK].float() * s[n + "_scale"][block][:, :, None] for n in "kv"]
    return tuple(t.to(s["qkv"].dtype) for t in (Q, K, *back))


def work(case):
    x, h, g, size = BYTES[case["dtype"]], case["heads"], case["kv_heads"], case["size"]
    lens, new = _lengths(case)
    if case["kind"] == "prompt":
        return {"bytes": 2 * sum(lens) * (h + g) * size * x, "flops": 4 * h * size * sum(n * (n + 1) // 2 for n in lens)}
    row = 2 * g * (size + 4 / BLOCK)                            # a token's codes and its share of the scales
    if case["kind"] == "cached":
        return {"bytes": sum(lens) * row + 2 * sum(new) * h * size * x,
                "flops": 4 * h * size * sum(m * n - m * (m - 1) // 2 for n, m in zip(lens, new))}
    back = sum(n - (n - m) // BLOCK * BLOCK for n, m in zip(lens, new))
    T = sum(new)
    return {"bytes": T * (2 * h + 3 * g) * size * x + (T + 2 * back) * row + back * 2 * g * size * x + T * 4 * case["rotary"],
            "flops": T * (3 * (h + g) * case["rotary"] + 4 * g * size)}


def _exact_attention(q, k, v, visible):
    """[n, size] rows of one head in 64 bits."""
    z = torch.matmul(q, k.t()) / math.sqrt(q.shape[1])
    return torch.matmul(torch.softmax(z.masked_fill(~visible, -math.inf), 1), v)


def exact(case, seed):
    d = _inputs(case, seed)
    h, g, size = case["heads"], case["kv_heads"], case["size"]
    lens, new = _lengths(case)
    if case["kind"] == "prompt":
        x = d["qkv"].double()
        Y = torch.empty((len(x), h, size), dtype=torch.float64, device="cuda")
        for a, b in zip(d["starts"], d["starts"][1:]):
            visible = torch.ones((b - a, b - a), dtype=torch.bool, device="cuda").tril()
            for i in range(h):
                Y[a:b, i] = _exact_attention(x[a:b, i], x[a:b, h + i // (h // g)], x[a:b, h + g + i // (h // g)], visible)
        return Y
    page, per_page = case["page"], case["page"] // BLOCK

    def tokens(name, i, first, last):                           # [last - first, g, size] of sequence i, from the cache
        p = torch.arange(first, last, device="cuda")
        b = d["pages"][i].long()[p // page] * per_page + p % page // BLOCK
        return torch.mul(d[name + "_codes"][b, :, p % BLOCK].double(), d[name + "_scale"][b].double().unsqueeze(2))

    if case["kind"] == "cached":
        out, at = [], 0
        for i, (n, m) in enumerate(zip(lens, new)):
            k, v, q = tokens("k", i, 0, n), tokens("v", i, 0, n), d["Q"][at:at + m].double()
            visible = torch.ones((m, n), dtype=torch.bool, device="cuda").tril(n - m)
            out.append(torch.stack([_exact_attention(q[:, j], k[:, j // (h // g)], v[:, j // (h // g)], visible) for j in range(h)], 1))
            at += m
        return torch.cat(out)
    # a rotated entry is two products and a sum, each kept in 32 bits, and so are scales, their inverses and what is rounded to a code
    def f32(t):
        return t.float().double()

    Q, K, back = [], [], {"k": [], "v": []}
    at, r = 0, case["rotary"] // 2
    for i, (n, m) in enumerate(zip(lens, new)):
        x = d["qkv"][at:at + m].double()
        at += m
        c, s = (d[t][n - m:n].double().unsqueeze(1) for t in ("cos", "sin"))
        y = x.clone()
        lo, hi = (torch.arange(r) * 2, torch.arange(r) * 2 + 1) if case["interleaved"] else (torch.arange(r), torch.arange(r) + r)
        lo, hi = lo.cuda(), hi.cuda()
        y[:, :h + g, lo] = f32(f32(x[:, :h + g, lo] * c) - f32(x[:, :h + g, hi] * s))
        y[:, :h + g, hi] = f32(f32(x[:, :h + g, hi] * c) + f32(x[:, :h + g, lo] * s))
        Q.append(y[:, :h])
        K.append(y[:, h:h + g])
        first = (n - m) // BLOCK * BLOCK
        for name, rows in (("k", y[:, h:h + g]), ("v", y[:, h + g:])):
            kept = n - m - first                                # older tokens of the first block
            whole = torch.zeros((-(-(n - first) // BLOCK) * BLOCK, g, size), dtype=torch.float64, device="cuda")
            whole[kept:n - first] = rows
            blocks = whole.view(-1, BLOCK, g, size)
            scale = f32(blocks.abs().amax((1, 3)) / 127)
            if kept:
                b = int(d["pages"][i, first // page]) * per_page + first % page // BLOCK
                old = d[name + "_scale"][b].double()
                scale[0] = torch.max(scale[0], old)
            inverse = f32(1 / scale)
            codes = torch.round(f32(blocks * inverse[:, None, :, None])).clamp(-127, 127)
            if kept:
                was = d[name + "_codes"][b, :, :kept].double().transpose(0, 1)
                codes[0, :kept] = torch.round(f32(was * f32(old / scale[0])[None, :, None]))
            back[name].append((codes * scale[:, None, :, None]).view(-1, g, size)[:n - first])
    return tuple(torch.cat(t) for t in (Q, K, back["k"], back["v"]))
