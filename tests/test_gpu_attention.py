"""GPU tests of the cache of keys and values and of attention (include/tst_attention.h), through the binding, against their definitions: codes bit for bit,
attention in 64 bits within bounds of the roundings (tests/kv_reference.py)."""
import math

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2510_06957_amd as tg

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LAST = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}   # half a step of the type, relative
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


def rng(*seed):
    return np.random.default_rng(list(seed))


def cuda(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t if dtype is None else t.to(dtype)).cuda()


def int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def f32(t):
    return t.detach().cpu().float().numpy()


def same(a, b, what=""):
    a, b = np.asarray(a), np.asarray(b)
    assert a.shape == b.shape, what
    bad = ~((a == b) | ((a != a) & (b != b)))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} differ, first at {np.argwhere(bad)[0]}: {a[bad][0]!r}, want {b[bad][0]!r}"


def strided(x, dtype, gap=0, token_gap=0):
    """x [T, heads, size] as a view whose heads and tokens lie `gap` and `token_gap` entries further apart, NaN between."""
    T, h, d = x.shape
    wide = torch.full((T, h * (d + gap) + token_gap), float("nan"), dtype=TYPES[dtype])
    view = wide[:, :h * (d + gap)].view(T, h, d + gap)[:, :, :d] if T else wide.view(T, h, d + gap)[:, :, :d]
    view.copy_(torch.from_numpy(x))
    big = wide.cuda()
    return big[:, :h * (d + gap)].view(T, h, d + gap)[:, :, :d]


class World:
    """Sequences in a cache, here and in the reference."""

    def __init__(self, lens, heads, size, page, seed, spare=2, columns=None):
        self.r = rng(seed, len(lens), heads, size, page)
        self.lens, self.heads, self.size, self.page = list(lens), heads, size, page
        held = [-(-max(n, 0) // page) for n in lens]
        pages = sum(held) + spare
        order = self.r.permutation(pages)
        self.table = np.full((len(lens), max(max(held), 1) if columns is None else columns), -1, np.int32)
        for i, n in enumerate(held):
            self.table[i, :n] = order[sum(held[:i]):sum(held[:i]) + n]
        self.ref = ref.Cache(pages, page, heads, size)
        for n in "kv":
            self.ref.codes[n][:] = self.r.integers(-127, 128, self.ref.codes[n].shape)
            self.ref.scale[n][:] = (0.5 + self.r.random(self.ref.scale[n].shape)) / 64
        self.cache = tg.tst_kv_cache(pages, page, heads, size)
        self.upload()

    def upload(self):
        c, blocks = self.cache, self.page // 16
        c.k_codes[..., :self.size] = cuda(self.ref.codes["k"])
        v = self.ref.codes["v"].reshape(self.ref.pages, self.heads, blocks, 16, self.size)
        c.v_codes[..., :self.size, :] = cuda(v.swapaxes(3, 4))
        c.k_scale.copy_(cuda(self.ref.scale["k"]))
        c.v_scale.copy_(cuda(self.ref.scale["v"]))

    def arrays(self):
        return cuda(self.table), int32(self.lens)

    def download(self):
        """(codes, scale) of "k" and "v", as the reference has them."""
        c = self.cache
        v = c.v_codes[..., :self.size, :].transpose(3, 4).reshape(self.ref.codes["v"].shape)
        return {"k": (c.k_codes[..., :self.size].cpu().numpy(), f32(c.k_scale)), "v": (v.cpu().numpy(), f32(c.v_scale))}

    def assert_cache(self, what=""):
        """Everything but what lies behind a block's last token."""
        for name, (codes, scale) in self.download().items():
            same(scale, self.ref.scale[name], f"{what} {name} scale")
            defined = np.ones(codes.shape[:3], bool)
            for i, n in enumerate(self.lens):
                if n % 16 and self.ref.page_of(self.table, i, n - 1) is not None:
                    defined[self.ref.page_of(self.table, i, n - 1), :, n % self.page:(n + 15) // 16 * 16 - n // self.page * self.page] = False
            same(np.where(defined[..., None], codes, 0), np.where(defined[..., None], self.ref.codes[name], 0), f"{what} {name} codes")
        if self.cache.k_codes.shape[3] > self.size:
            assert not self.cache.k_codes[..., self.size:].any() and not self.cache.v_codes[..., self.size:, :].any()


def starts(new, front=0):
    at = [front]
    for n in new:
        at.append(at[-1] + n)
    return at


def angles(positions, pairs):
    a = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(pairs) / pairs)
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def check_append(lens, new, q_heads, heads, size, page, dtype, pairs, interleaved, seed, gap=0, token_gap=0, offsets=True, grow=1.0, front=0):
    w = World(lens, heads, size, page, seed)
    at = starts(new, front)
    T = at[-1] + front
    r = rng(seed, 1)
    K, V, Q = (r.standard_normal((T, h, size)) * grow for h in (heads, heads, q_heads))
    Kd, Vd, Qd = (strided(x, dtype, gap, token_gap) for x in (K, V, Q))
    K, V, Q = f32(Kd), f32(Vd), f32(Qd)
    pages, lens_d = w.arrays()
    kw = dict(offsets=int32(at) if offsets else None)
    if pairs:
        cos, sin = angles(max(max(lens), 1), pairs)
        kw.update(Q=Qd, cos=cuda(cos), sin=cuda(sin), interleaved=interleaved, keys=True)
    for again in range(2):   # a second time changes nothing
        q_out, k_out = tg.tst_kv_append(w.cache, Kd, Vd, pages, lens_d, **kw)
        if again == 0:
            position = np.full(T, -1)
            for i, n in enumerate(new):
                position[at[i]:at[i + 1]] = np.arange(lens[i] - n, lens[i])
            if pairs:
                K, Q = ref.rotate(K, position, cos, sin, interleaved), ref.rotate(Q, position, cos, sin, interleaved)
            for i, n in enumerate(new):
                if n:
                    w.ref.append("k", K[at[i]:at[i + 1]], w.table, i, lens[i] - n)
                    w.ref.append("v", V[at[i]:at[i + 1]], w.table, i, lens[i] - n)
        w.assert_cache(f"call {again}")
        if pairs:
            for got, want in ((q_out, Q), (k_out, K)):
                assert got.dtype == TYPES[dtype] and got.is_contiguous()
                same(f32(got)[at[0]:at[-1]], f32(torch.from_numpy(want).to(TYPES[dtype]))[at[0]:at[-1]], "rotated")
        else:
            assert q_out is None and k_out is None
    for kind in TYPES:       # what the codes stand for
        k, v = tg.tst_kv_read(w.cache, pages, lens_d, T, offsets=kw["offsets"], dtype=TYPES[kind])
        for got, name in ((k, "k"), (v, "v")):
            want = np.concatenate([w.ref.values(name, w.table, i, lens[i] - n, lens[i]) for i, n in enumerate(new)])
            same(f32(got)[at[0]:at[-1]], f32(torch.from_numpy(want).to(TYPES[kind])), f"read {name}")
    return w


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lens,new,page", [([1], [1], 16), ([16, 17, 33], [1, 1, 1], 16), ([100, 5, 64, 63], [37, 5, 1, 20], 32), ([300], [300], 256),
                                           ([48, 0, 31, 500], [17, 0, 0, 490], 64), ([129] * 70, [1, 3] * 35, 128)])
def test_append(lens, new, page, dtype):
    check_append(lens, new, 6, 3, 64, page, dtype, 32, False, 1)


@pytest.mark.parametrize("size,pairs,interleaved", [(1, 0, False), (2, 1, True), (7, 2, False), (8, 4, True), (33, 16, False), (64, 0, False), (72, 36, False),
                                                     (80, 16, True), (80, 40, False), (96, 48, False), (100, 50, True), (128, 64, True), (128, 32, False),
                                                     (192, 96, False), (200, 100, True), (255, 127, False), (256, 128, False), (256, 128, True)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_append_sizes(size, pairs, interleaved, dtype):
    check_append([70, 19], [33, 2], 10, 5, size, 32, dtype, pairs, interleaved, 2)


@pytest.mark.parametrize("gap,token_gap", [(8, 0), (0, 16), (1, 0), (0, 3), (24, 40)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_of_views(gap, token_gap, dtype):
    check_append([50, 90], [20, 41], 4, 2, 64, 16, dtype, 32, False, 3, gap, token_gap, grow=3.0)


def test_append_without_offsets_and_with_rows_of_no_sequence():
    check_append([17, 64, 1, 250], [1] * 4, 8, 2, 128, 64, "bf16", 64, False, 4, offsets=False)
    check_append([17, 64, 1, 250], [3, 1, 1, 20], 8, 2, 128, 64, "bf16", 64, False, 4, front=5)


def test_append_token_by_token_is_append_with_growing_scales():
    """Each token larger than those before it: every code that was there is rescaled, each time."""
    w = World([0], 2, 64, 16, 5)
    r = rng(5, 2)
    w.table[:] = 1
    pages = cuda(w.table)
    for n in range(1, 17):
        x = (r.standard_normal((1, 2, 64)) * 1.3 ** n).astype(np.float32)
        w.lens = [n]
        tg.tst_kv_append(w.cache, cuda(x), cuda(-x), pages, int32([n]))
        w.ref.append("k", x, w.table, 0, n - 1)
        w.ref.append("v", -x, w.table, 0, n - 1)
        w.assert_cache(f"token {n}")


def test_append_of_entries_that_are_special():
    """Zeros, subnormals, the largest there are, infinities and NaN, in blocks of their own and beside others."""
    w = World([64, 24], 1, 8, 16, 6)
    x = np.ones((64 + 4, 1, 8), np.float32)
    x[:16] = 0
    x[16:32] = np.float32(1e-42)
    x[32:48] = 3.4028234e38
    x[50, 0, 3] = np.nan
    x[65, 0, 0] = -np.inf
    pages, lens = w.arrays()
    tg.tst_kv_append(w.cache, cuda(x), cuda(x[::-1].copy()), pages, lens, int32([0, 64, 68]))
    for i, (a, b, first) in enumerate(((0, 64, 0), (64, 68, 20))):
        w.ref.append("k", x[a:b], w.table, i, first)
        w.ref.append("v", x[::-1][a:b], w.table, i, first)
    assert np.isnan(w.ref.scale["k"]).sum() == 2
    w.assert_cache()
    y = np.full((1, 1, 8), 2, np.float32)      # a block begun anew is rid of the NaN
    w.lens = [49, 24]
    tg.tst_kv_append(w.cache, cuda(y), cuda(y), cuda(w.table[:1]), int32([49]))
    w.ref.append("k", y, w.table, 0, 48)
    w.ref.append("v", y, w.table, 0, 48)
    w.assert_cache()
    assert np.isnan(w.ref.scale["k"]).sum() == 1


def test_append_and_read_where_there_are_no_pages():
    """Pages that are none of the cache's, positions behind the table, more rows than tokens, offsets that do not ascend: nothing else is touched."""
    w = World([40, 70, 3], 2, 64, 16, 7)
    w.table[0, 1] = -5
    w.table[1, 2] = w.ref.pages
    w.table[1, 3] = 2 ** 31 - 1
    r = rng(7, 3)
    new = [40, 70, 8]
    at = starts(new)
    K, V = (r.standard_normal((at[-1], 2, 64)).astype(np.float32) for _ in "kv")
    pages, lens = w.arrays()
    lens[1] = 100                      # behind the table's five columns
    cos, sin = angles(50, 32)
    q, k = tg.tst_kv_append(w.cache, cuda(K), cuda(V), pages, lens, int32(at), Q=cuda(K), cos=cuda(cos), sin=cuda(sin), keys=True)
    position = np.concatenate([np.arange(40), np.arange(30, 100), np.arange(-5, 3)])
    rotated = ref.rotate(K, position, cos, sin, False)
    same(f32(k), rotated)
    same(f32(q), rotated)
    assert np.isnan(rotated[-8:-3]).all() and np.isnan(rotated[40 + 20:40 + 70]).all()
    for i in range(3):
        first = position[at[i]]
        skip = max(-first, 0)
        for name, x in (("k", rotated), ("v", V)):
            w.ref.append(name, x[at[i] + skip:at[i + 1]], w.table, i, first + skip)
    w.lens = [40, 100, 3]
    w.assert_cache()
    k, v = tg.tst_kv_read(w.cache, pages, lens, at[-1], int32(at), dtype=torch.float32)
    for got, name in ((k, "k"), (v, "v")):
        want = np.concatenate([w.ref.values(name, w.table, i, position[at[i]], position[at[i]] + new[i]) for i in range(3)])
        keep = position >= 0
        same(f32(got)[keep], want[keep])
    for wrong in ([0, 80, 20, 118], [-7, 5, 2 ** 31 - 1, 9], [118, 0, 118, 0]):
        before = w.download()
        q, k = tg.tst_kv_append(w.cache, cuda(K), cuda(V), torch.full_like(pages, -1), lens, int32(wrong), Q=cuda(K), cos=cuda(cos), sin=cuda(sin), keys=True)
        tg.tst_kv_read(w.cache, pages, lens, at[-1], int32(wrong))
        after = w.download()
        for name in "kv":
            same(after[name][0], before[name][0])
            same(after[name][1], before[name][1])


# ------------------------------------------------------------------------------------------------------------------------ attention
WEIGHT = {"f32": 2.0 ** -22, "bf16": 2.0 ** -11, "f16": 2.0 ** -11}   # kept of a weight by tst_kv_attention
CUT = {"f32": 2.0 ** -22, "bf16": 2.0 ** -24, "f16": 2.0 ** -24}      # of a query's entry, relative to the largest of its row


def assert_within(got, want, bound, dtype, what=""):
    got = f32(got).astype(np.float64)
    bound = bound + LAST[dtype] * (np.abs(want) + bound) + TINY[dtype]
    assert got.shape == want.shape
    bad = ~((np.abs(got - want) <= bound) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} outside, first at {np.argwhere(bad)[0]}: {got[bad][0]!r}, want {want[bad][0]!r} +- {bound[bad][0]!r}"


def reference_over_cache(w, Q, new, at, scale, dtype, heads=None):
    """Rows of Q float32 [T, q_heads, size]; -> (Y, bound), rows of no sequence 0."""
    T, q_heads, size = Q.shape
    Y, bound = np.zeros(Q.shape), np.zeros(Q.shape)
    group = q_heads // w.heads
    for i, n in enumerate(new):
        if n == 0:
            continue
        length = max(w.lens[i], 0)
        k, v = (w.ref.values(name, w.table, i, 0, length, np.float64) for name in "kv")
        limit = np.maximum(w.lens[i] - n + np.arange(n) + 1, 0)
        for h in range(q_heads) if heads is None else heads:
            y, b = ref.attention(Q[at[i]:at[i + 1], h].astype(np.float64), k[:, h // group], v[:, h // group], limit, scale, WEIGHT[dtype], CUT[dtype])
            Y[at[i]:at[i + 1], h], bound[at[i]:at[i + 1], h] = y, b
    return Y, bound


def queries(w, T, q_heads, size, seed, large=1.0):
    return rng(seed, T, q_heads).standard_normal((T, q_heads, size)) * large


def check_over_cache(lens, new, q_heads, heads, size, page, dtype, seed, large=1.0, gap=0, scale=None, columns=None, **kw):
    w = World(lens, heads, size, page, seed, columns=columns)
    at = starts(new)
    T = at[-1]
    Qd = strided(queries(w, T, q_heads, size, seed, large), dtype, gap)
    pages, lens_d = w.arrays()
    offsets = None if new == [1] * len(lens) else int32(at)
    Y = tg.tst_kv_attention(Qd, w.cache, pages, lens_d, offsets, scale=scale, **kw)
    assert Y.dtype == TYPES[dtype] and Y.shape == Qd.shape
    want, bound = reference_over_cache(w, f32(Qd), new, at, 1 / math.sqrt(size) if scale is None else scale, dtype)
    assert_within(Y, want, bound, dtype, f"lens {lens[:6]} new {new[:6]}")
    assert torch.equal(tg.tst_kv_attention(Qd, w.cache, pages, lens_d, offsets, scale=scale, **kw), Y)
    return w, Qd, Y


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lens,new,page", [([1], [1], 16), ([15, 16, 17, 63, 64, 65], [1] * 6, 16), ([255, 256, 257, 1000], [1] * 4, 64),
                                           ([5000, 3, 700], [1] * 3, 256), ([0, 9, 0], [1] * 3, 32), ([130, 40, 1030], [5, 1, 9], 32), ([700, 64], [64, 64], 128)])
def test_attention_over_the_cache(lens, new, page, dtype):
    check_over_cache(lens, new, 8, 2, 128, page, dtype, 11)


@pytest.mark.parametrize("q_heads,heads", [(1, 1), (5, 5), (3, 1), (7, 1), (14, 2), (16, 1), (17, 1), (48, 3), (64, 1)])
@pytest.mark.parametrize("new", [[1, 1], [2, 7]])
def test_attention_over_the_cache_groups(q_heads, heads, new):
    check_over_cache([301, 90], new, q_heads, heads, 64, 16, "bf16", 12)


@pytest.mark.parametrize("size", [1, 7, 8, 32, 64, 65, 80, 96, 100, 128, 130, 192, 200, 255, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_attention_over_the_cache_sizes(size, dtype):
    check_over_cache([333, 100], [1, 1], 4, 2, size, 32, dtype, 13)
    check_over_cache([333, 100], [30, 4], 4, 2, size, 32, dtype, 14, gap=3)


@pytest.mark.parametrize("large,scale", [(50.0, None), (1e-3, None), (1.0, 0.0), (1.0, -0.3), (1.0, 3.0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_attention_over_the_cache_scales(large, scale, dtype):
    check_over_cache([900, 77], [1, 1], 4, 1, 64, 16, dtype, 15, large=large, scale=scale)


# ------------------------------------------------------------------------------------------------------------------------ prompts
# half a step of a weight in the second product, and what the three bf16 planes of fp32 leave out: products of planes behind the 24th bit, of queries and
# keys (cut) and of weights and values
PROMPT_WEIGHT = {"f32": 2.0 ** -21, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
PROMPT_CUT = {"f32": 2.0 ** -21, "bf16": 0.0, "f16": 0.0}


def prompt_reference(Q, K, V, at, scale, dtype, heads=None, rows=None):
    """(Y, bound); `rows`: of each sequence, all if None."""
    Y, bound = np.zeros(Q.shape), np.zeros(Q.shape)
    group = Q.shape[1] // K.shape[1]
    for a, b in zip(at, at[1:]):
        own = np.arange(b - a) if rows is None else rows[rows < b - a]
        for h in range(Q.shape[1]) if heads is None else heads:
            y, e = ref.attention(Q[a:b, h].astype(np.float64)[own], K[a:b, h // group].astype(np.float64), V[a:b, h // group].astype(np.float64), own + 1, scale,
                                 PROMPT_WEIGHT[dtype], PROMPT_CUT[dtype])
            Y[a + own, h], bound[a + own, h] = y, e
    return Y, bound


def prompt(lens, q_heads, heads, size, dtype, seed, gap=0, token_gap=0, large=1.0):
    r = rng(seed, sum(lens), q_heads, size)
    T = sum(lens)
    return [strided(r.standard_normal((T, h, size)) * (large if i < 2 else 1), dtype, gap, token_gap) for i, h in enumerate((q_heads, heads, heads))]


def check_prompt(lens, q_heads, heads, size, dtype, seed, scale=None, **kw):
    q, k, v = prompt(lens, q_heads, heads, size, dtype, seed, **kw)
    at = starts(lens)
    Y = tg.tst_attention(q, k, v, int32(at), scale=scale)
    assert Y.dtype == TYPES[dtype] and Y.shape == q.shape and Y.is_contiguous()
    want, bound = prompt_reference(f32(q), f32(k), f32(v), at, 1 / math.sqrt(size) if scale is None else scale, dtype)
    assert_within(Y, want, bound, dtype, f"lens {lens[:6]}")
    assert torch.equal(tg.tst_attention(q, k, v, int32(at), scale=scale), Y)


@pytest.mark.parametrize("lens", [[1], [2], [31], [32], [33], [63, 64, 65], [1, 0, 127, 0, 128, 129, 1], [300], [257, 5, 513], [3] * 100])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_prompts(lens, dtype):
    check_prompt(lens, 4, 2, 64, dtype, 21)


@pytest.mark.parametrize("q_heads,heads", [(1, 1), (3, 3), (3, 1), (7, 1), (8, 1), (14, 2), (33, 1), (130, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompts_groups(q_heads, heads, dtype):
    check_prompt([70, 9, 150], q_heads, heads, 64, dtype, 22)


@pytest.mark.parametrize("size", [1, 7, 8, 40, 64, 65, 72, 80, 96, 100, 112, 128, 129, 136, 192, 200, 255, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_prompts_sizes(size, dtype):
    check_prompt([130, 41], 4, 2, size, dtype, 23)
    check_prompt([130, 41], 4, 2, size, dtype, 24, gap=5, token_gap=1)


@pytest.mark.parametrize("large,scale", [(8.0, None), (1e-3, None), (1.0, 0.0), (1.0, -0.3), (1.0, 2.0), (30.0, 0.5)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_prompts_scales(large, scale, dtype):
    check_prompt([200, 33], 4, 1, 64, dtype, 25, large=large, scale=scale)


def test_prompts_of_many_sequences():
    """More sequences than are put in order by their lengths, and as many; the others are 0 to 40 tokens long."""
    for n, long in ((64, 700), (65, 700), (1500, 300)):
        lens = [int(x) for x in rng(26, n).integers(0, 41, n)]
        lens[n // 3] = long
        check_prompt(lens, 2, 1, 64, "bf16", 26)
