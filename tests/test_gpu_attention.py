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


def with_room(pages, page):
    """The table with columns for 16384 tokens more: sequences that may be as long as that are cut into chunks."""
    return torch.cat([pages, torch.full((pages.shape[0], 16384 // page), -1, dtype=torch.int32, device="cuda")], 1)


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
    for _ in range(2):
        assert_within(tg.tst_kv_attention(Qd, w.cache, with_room(pages, page), lens_d, offsets, scale=scale, **kw), want, bound, dtype, f"cut: lens {lens[:6]} new {new[:6]}")
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


@pytest.mark.parametrize("lens,q_heads,heads,size", [([700], 3, 1, 64), ([129, 300, 161], 4, 2, 80), ([1030, 1], 1, 1, 128), ([400] * 3, 7, 1, 100), ([33, 66], 2, 2, 128)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_prompts_whose_keys_are_shared(lens, q_heads, heads, size, dtype):
    """Few rows and many keys."""
    check_prompt(lens, q_heads, heads, size, dtype, 30)
    check_prompt(lens, q_heads, heads, size, dtype, 30, scale=1.5)


@pytest.mark.parametrize("q_heads,heads,size,dtype", [(64, 8, 64, "bf16"), (64, 8, 96, "f16"), (64, 16, 128, "bf16"), (66, 2, 128, "f16"), (64, 64, 64, "f16"), (64, 8, 80, "bf16"),
                                                      (64, 4, 192, "bf16"), (32, 8, 256, "f16")])
@pytest.mark.parametrize("lens", [[1217, 0, 3, 64, 65, 400, 1], [1217, 835]])
def test_prompts_in_whole_tiles(lens, q_heads, heads, size, dtype):
    """Enough rows for the tiles that large calls take, of short prompts and of long ones; a few heads and rows of each sequence against the definition."""
    q, k, v = prompt(lens, q_heads, heads, size, dtype, 27)
    at = starts(lens)
    Y = tg.tst_attention(q, k, v, int32(at))
    few = [0, q_heads // 2 + 1, q_heads - 1]
    rows = np.unique(np.r_[np.arange(0, 70), np.arange(120, 135), np.arange(250, 262), np.arange(1200, 1217)])
    want, bound = prompt_reference(f32(q), f32(k), f32(v), at, 1 / math.sqrt(size), dtype, few, rows)
    seen = np.concatenate([a + rows[rows < b - a] for a, b in zip(at, at[1:])])
    assert_within(Y[torch.from_numpy(seen).cuda()][:, few], want[seen][:, few], bound[seen][:, few], dtype)
    assert torch.equal(tg.tst_attention(q, k, v, int32(at)), Y)
    for off in (1, 4):      # results that lie off 16-byte borders, and off 8-byte ones
        room = torch.full((Y.numel() + 16,), 7.0, dtype=Y.dtype, device="cuda")
        assert torch.equal(tg.tst_attention(q, k, v, int32(at), Y=room[off:off + Y.numel()].view(Y.shape)), Y)
        assert (room[:off] == 7).all() and (room[off + Y.numel():] == 7).all()
    # each sequence by itself, in smaller tiles: the same up to the rounding of its sums
    for a, b in zip(at, at[1:]):
        alone = tg.tst_attention(q[a:b], k[a:b], v[a:b], int32([0, b - a]))
        assert torch.allclose(alone.float(), Y[a:b].float(), rtol=8 * LAST[dtype], atol=0.02)


@pytest.mark.parametrize("q_heads,lens", [(4, [90, 40]), (4, [300, 77]), (64, [1217, 64]), (64, [2100, 64])])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_prompts_what_a_row_does_not_see_does_not_touch_it(dtype, q_heads, lens):
    """Infinities and NaN in keys and values behind a row, in other sequences and in rows of no sequence."""
    heads, size = 2, 64
    T = sum(lens)
    q, k, v = prompt([T + 9], q_heads, heads, size, dtype, 28)
    offsets = int32([5, 5 + lens[0], 5 + T])
    clean = tg.tst_attention(q, k, v, offsets)[5:5 + T]
    k2, v2 = k.clone(), v.clone()
    k2[:5], v2[:5], k2[5 + T:], v2[5 + T:] = float("nan"), float("inf"), float("inf"), float("nan")
    cut = 5 + lens[0] - 27           # from here on the first sequence is spoilt, a channel of a head's values
    k2[cut:5 + lens[0], 1] = float("nan")
    v2[cut + 2, 0, 7], v2[cut + 3, 0, 63], v2[cut + 4, 0, 0], v2[cut + 2, 1] = float("nan"), float("inf"), -float("inf"), float("inf")
    Y = tg.tst_attention(q, k2, v2, offsets)[5:5 + T]
    group, n = q_heads // heads, cut - 5
    assert torch.equal(Y[:n], clean[:n]) and torch.equal(Y[lens[0]:], clean[lens[0]:])
    assert torch.equal(Y[:n + 2, :group], clean[:n + 2, :group])
    spoilt = ~torch.isfinite(Y[:lens[0], :group])
    want = torch.zeros_like(spoilt)
    want[n + 2:, :, 7], want[n + 3:, :, 63], want[n + 4:, :, 0] = True, True, True
    assert torch.equal(spoilt, want)
    assert torch.equal(Y[:lens[0], :group][~want], clean[:lens[0], :group][~want])
    assert torch.isnan(Y[n:lens[0], group:]).all()
    q2 = q.clone()
    q2[5 + 3, 1, 2], q2[5 + 4, 1, 2] = float("nan"), float("inf")
    Y = tg.tst_attention(q2, k, v, offsets)[5:5 + T]
    assert torch.isnan(Y[3, 1]).all() and not torch.isfinite(Y[4, 1]).any()
    Y[3:5, 1] = clean[3:5, 1]
    assert torch.equal(Y, clean)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompts_leave_other_rows_as_they_are(dtype):
    q, k, v = prompt([60], 4, 4, 40, dtype, 29)
    Y = torch.full((60, 4, 40), 7.0, dtype=TYPES[dtype], device="cuda")
    out = tg.tst_attention(q, k, v, int32([11, 30, 30, 49]), Y=Y)
    assert out is Y and (Y[:11] == 7).all() and (Y[49:] == 7).all() and not (Y[11:49] == 7).all(2).any()
    assert torch.equal(tg.tst_attention(q, k, v, int32([11, 30, 30, 49]))[11:49], Y[11:49])
    for wrong in ([49, 30, 11], [-5, 20, 2 ** 31 - 1], [60, 0, 60, 0], [0, 100, 30]):     # nothing outside is touched
        wide = torch.full((80, 4, 40), 7.0, dtype=TYPES[dtype], device="cuda")
        tg.tst_attention(q, k, v, int32(wrong), Y=wide[10:70])
        assert (wide[:10] == 7).all() and (wide[70:] == 7).all()
    Y.fill_(7)
    tg.tst_attention(q, k, v, int32([0]), Y=Y)      # no sequences
    tg.tst_attention(q, k, v, int32([20, 20]), Y=Y)
    assert (Y == 7).all()
    assert tg.tst_attention(q[:0], k[:0], v[:0], int32([0, 0])).shape == (0, 4, 40)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_over_long_caches(dtype):
    """Chunks that are joined, of one sequence and of ragged ones; drafts of rows in two tiles; more sequences than are cut."""
    check_over_cache([20011], [1], 4, 1, 64, 64, dtype, 31)
    check_over_cache([9000, 17, 4097, 0, 1, 6000], [1] * 6, 7, 1, 128, 256, dtype, 32)
    check_over_cache([5000, 800, 64], [3, 40, 64], 4, 1, 96, 16, dtype, 33)
    lens = [int(x) for x in rng(34).integers(0, 300, 1100)]
    check_over_cache(lens, [1] * 1100, 1, 1, 64, 16, dtype, 34)
    check_over_cache(lens[:70] + [4000], [2] * 70 + [31], 2, 1, 64, 32, dtype, 35)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("columns", [100, 1000])
def test_attention_over_the_cache_scales_of_blocks(dtype, columns):
    """Scales of values and keys that differ by many powers of ten between blocks; blocks of zeros."""
    w = World([1500, 333], 2, 64, 32, 36, columns=columns)
    for name, spread in (("k", 3), ("v", 12)):
        w.ref.scale[name] *= (10.0 ** w.r.integers(-spread, 2, w.ref.scale[name].shape)).astype(np.float32)
        w.ref.scale[name][w.r.random(w.ref.scale[name].shape) < 0.1] = 0
    w.upload()
    pages, lens = w.arrays()
    Qd = strided(queries(w, 2, 4, 64, 36), dtype)
    want, bound = reference_over_cache(w, f32(Qd), [1, 1], [0, 1, 2], 0.125, dtype)
    assert_within(tg.tst_kv_attention(Qd, w.cache, pages, lens), want, bound, dtype)
    w.ref.scale["v"][:] = 0
    w.upload()
    assert not tg.tst_kv_attention(Qd, w.cache, pages, lens).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("columns", [100, 1000])
def test_attention_over_the_cache_what_a_row_does_not_see(dtype, columns):
    """Blocks without a scale behind a row; rows that see one, or whose query is none, are NaN."""
    w = World([700, 90, 350], 2, 64, 16, 37, columns=columns)
    new = [40, 1, 3]
    at = starts(new)
    Qd = strided(queries(w, at[-1], 4, 64, 37), dtype)
    pages, lens = w.arrays()
    clean = tg.tst_kv_attention(Qd, w.cache, pages, lens, int32(at))
    want, bound = reference_over_cache(w, f32(Qd), new, at, 0.125, dtype)
    assert_within(clean, want, bound, dtype)
    for name in "kv":
        saved = w.ref.scale[name].copy()
        for scale in (np.nan, np.float32(1e30)):
            w.ref.scale[name][w.table[0, 688 // 16], 1, 0] = scale       # positions 688 .. of head 1: rows 28 .. of the first sequence's 40
            w.upload()
            Y = tg.tst_kv_attention(Qd, w.cache, pages, lens, int32(at))
            assert np.isfinite(scale) or torch.isnan(Y[28:40, 2:]).all()
            Y[28:40, 2:] = clean[28:40, 2:]
            assert torch.equal(Y, clean)
        w.ref.scale[name] = saved
    w.upload()
    Q2 = Qd.clone()
    Q2[3, 1, 5], Q2[40, 2, 0] = float("inf"), float("nan")
    Y = tg.tst_kv_attention(Q2, w.cache, pages, lens, int32(at))
    assert torch.isnan(Y[3, 1]).all() and torch.isnan(Y[40, 2]).all()
    Y[3, 1], Y[40, 2] = clean[3, 1], clean[40, 2]
    assert torch.equal(Y, clean)


@pytest.mark.parametrize("columns", [100, 1000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_over_the_cache_blocks_without_a_scale_whose_tokens_weigh_nothing(dtype, columns):
    """A row that sees one is NaN however far below others its logits lie, also where another wavefront or chunk has those."""
    w = World([1500], 1, 64, 16, 49, columns=columns)
    pages, lens = w.arrays()
    Qd = strided(np.ones((1, 2, 64)), dtype)
    w.ref.codes["k"][w.table[0, 60]] = 127
    w.ref.scale["k"][w.table[0, 60]] = 100.0       # logits of 0.125 * 64 * 12700; the others' are below 130
    w.upload()
    want = f32(tg.tst_kv_attention(Qd, w.cache, pages, lens))
    assert np.isfinite(want).all()
    for block in (0, 3, 61, 70, 93):
        w.ref.scale["v"][w.table[0, block]] = np.nan
        w.upload()
        assert torch.isnan(tg.tst_kv_attention(Qd, w.cache, pages, lens)).all(), block
        w.ref.scale["v"][w.table[0, block]] = 1.0
        w.upload()
        # the scale of a block changes what weights are relative to, and so how each is rounded, here and before: twice half a step of values of at most 127 * 1.5 / 64
        assert_within(tg.tst_kv_attention(Qd, w.cache, pages, lens), want, np.full(want.shape, 2 * WEIGHT[dtype] * 127 * 1.5 / 64), dtype, block)


@pytest.mark.parametrize("columns", [30, 1000])
def test_attention_over_the_cache_where_there_are_no_pages(columns):
    """Pages that are none of the cache's make the rows that see them NaN, and so do positions behind the table; rows of negative positions see nothing."""
    w = World([400, 70, 33, 20], 2, 64, 16, 38, columns=columns)
    w.table[0, 23], w.table[1, 0], w.table[2, 2] = w.ref.pages, -7, 2 ** 31 - 1
    new = [40, 2, 1, 24]
    at = starts(new)
    Qd = strided(queries(w, at[-1], 2, 64, 38), "f32")
    pages, lens = w.arrays()
    Y = tg.tst_kv_attention(Qd, w.cache, pages, lens, int32(at))
    # page 23 is positions 368 ..: rows 8 .. of the first sequence
    good = np.r_[np.arange(8), np.arange(at[3], at[4])]
    want, bound = reference_over_cache(w, f32(Qd), new, at, 0.125, "f32")
    assert_within(Y[good], want[good], bound[good], "f32")
    assert (Y[at[3]:at[3] + 4] == 0).all()
    assert torch.isnan(Y[8:at[3]]).all()
    lens[:] = torch.tensor([2 ** 31 - 1, 16 * columns + 1, -5, -2 ** 31], dtype=torch.int32)     # one more than the table holds
    w.table[:] = w.r.integers(0, w.ref.pages, w.table.shape)
    Y = tg.tst_kv_attention(Qd, w.cache, cuda(w.table), lens, int32(at))
    assert torch.isnan(Y[:40]).all() and torch.isnan(Y[41]).all() and torch.isfinite(Y[40]).all() and (Y[42:] == 0).all()
    for wrong in ([40, 0, 67, 10, 50], [-9, 5, 2 ** 31 - 1, 4, 67], [67, 60, 40, 20, 0], [0, 67, 0, 67, 0]):
        wide = torch.full((87, 2, 64), 7.0, device="cuda")
        tg.tst_kv_attention(Qd, w.cache, pages, lens, int32(wrong), Y=wide[10:77])
        assert (wide[:10] == 7).all() and (wide[77:] == 7).all()


def test_attention_over_the_cache_leaves_other_rows_as_they_are():
    w = World([300, 50], 1, 64, 16, 39, columns=1000)     # room for sequences that are cut, which needs a workspace
    Qd = strided(queries(w, 12, 2, 64, 39), "bf16")
    pages, lens = w.arrays()
    Y = torch.full((12, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(8 << 20, dtype=torch.uint8, device="cuda")
    out = tg.tst_kv_attention(Qd, w.cache, pages, lens, int32([3, 7, 9]), Y=Y, workspace=ws)
    assert out is Y and (Y[:3] == 7).all() and (Y[9:] == 7).all()
    assert torch.equal(tg.tst_kv_attention(Qd, w.cache, pages, lens, int32([3, 7, 9]))[3:9], Y[3:9])
    with pytest.raises(tg.TstgemmError) as e:
        tg.tst_kv_attention(Qd, w.cache, pages, lens, int32([3, 7, 9]), workspace=ws[:256])
    assert e.value.code == -8


def test_a_cache_of_more_than_4_gib():
    """Pages whose codes lie behind 2^31 and 2^32 bytes."""
    heads, size, page = 8, 128, 256
    pages = (1 << 32) // (heads * page * size) + 40
    cache = tg.tst_kv_cache(pages, page, heads, size)
    small = tg.tst_kv_cache(8, page, heads, size)
    lens = int32([700, 300])
    far = torch.tensor([[pages - 1, 3, pages // 2 + 7], [pages - 2, pages // 2, -1]], dtype=torch.int32, device="cuda")
    near = torch.tensor([[0, 1, 2], [5, 4, -1]], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(40)
    K, V = (torch.randn((1000, heads, size), generator=g, device="cuda").bfloat16() for _ in "kv")
    Q = torch.randn((2, 16, size), generator=g, device="cuda").bfloat16()
    offsets, out = int32([0, 700, 1000]), []
    for c, table in ((cache, far), (small, near)):
        tg.tst_kv_append(c, K, V, table, lens, offsets)
        out.append((*tg.tst_kv_read(c, table, lens, 1000, offsets), tg.tst_kv_attention(Q, c, table, lens)))
    for a, b in zip(*out):
        assert torch.equal(a, b)
    assert (out[0][0].float() - K.float()).abs().max() < 0.05


def test_sequences_of_2_30_tokens():
    """As long as a table can be, over pages that repeat: keys all alike, so that a result says how many tokens of either value were seen."""
    cache = tg.tst_kv_cache(2, 256, 1, 64)
    cache.v_codes[0], cache.v_codes[1] = 100, -30
    cache.v_scale.fill_(1.0)
    columns = (1 << 30) // 256
    page = torch.zeros((3, columns), dtype=torch.int32, device="cuda")
    page[0, columns // 2:], page[1, columns // 8:], page[2, columns - columns // 8:] = 1, 1, 1
    Y = tg.tst_kv_attention(torch.ones((3, 2, 64), device="cuda"), cache, page, int32([1 << 30, 1 << 30, (1 << 30) - 77]))
    # a quarter of a chunk (a 170th of a sequence) adds 2^16 products of 32 tokens at most, each rounded by 2^-24 of a sum whose magnitude is below 100 for each token: 2^-8 of 100,
    # and as much of the weights
    for y, want in zip(f32(Y), (35.0, -30 + 130 / 8, 100 - 130 / 8)):
        assert (np.abs(y - want) <= 2.0 ** -7 * 100).all()


def test_views_that_start_far_into_large_tensors():
    """Rows, heads and pages at offsets behind 2^31 entries."""
    big = torch.zeros((3, 1 << 30), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(41)
    x = torch.randn((3, 6, 64), generator=g, device="cuda").bfloat16()
    view = big[:, (1 << 30) - 384:].view(3, 6, 64)
    view.copy_(x)
    assert view.stride(0) == 1 << 30
    offsets = int32([0, 3])
    assert torch.equal(tg.tst_attention(view[:, :4], view[:, 4:5], view[:, 5:], offsets), tg.tst_attention(x[:, :4], x[:, 4:5], x[:, 5:], offsets))
    caches = [tg.tst_kv_cache(4, 16, 1, 64) for _ in range(2)]
    pages, lens = int32([[2]]), int32([3])
    for c, t in zip(caches, (view, x)):
        tg.tst_kv_append(c, t[:, 4:5], t[:, 5:], pages, lens, offsets)
    a, b = (tg.tst_kv_read(c, pages, lens, 3, offsets) for c in caches)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and a[0].any()
    assert torch.equal(tg.tst_kv_attention(view[:, :4], caches[0], pages, lens, offsets), tg.tst_kv_attention(x[:, :4], caches[1], pages, lens, offsets))


# ------------------------------------------------------------------------------------------------------------------------ together, streams, graphs
def sequence_of_calls(cache, x, q_heads, pages, lens, offsets, cos, sin, **kw):
    """Append and attend, the newest tokens by the cache and by themselves."""
    heads = cache.heads
    q, k = tg.tst_kv_append(cache, x[:, q_heads:q_heads + heads], x[:, q_heads + heads:], pages, lens, offsets, Q=x[:, :q_heads], cos=cos, sin=sin, keys=True, **kw)
    return q, k, tg.tst_kv_attention(q, cache, pages, lens, offsets, **kw), *tg.tst_kv_read(cache, pages, lens, x.shape[0], offsets, dtype=x.dtype, **kw)


def test_a_prompt_and_what_follows_it():
    """A prompt by itself and over the cache that it was appended to agree up to the codes; further tokens go by the cache.  Each against the definition."""
    heads, q_heads, size, page = 2, 6, 64, 32
    lens = [75, 20, 130]
    w = World(lens, heads, size, page, 42, spare=9)
    w.table = np.concatenate([w.table, np.full((3, 1), -1, np.int32)], 1)
    free = sorted(set(range(w.ref.pages)) - set(w.table[w.table >= 0].tolist()))
    for i, n in enumerate(lens):
        w.table[i, -(-n // page)] = free[i]
    r = rng(42, 5)
    cos, sin = angles(200, size // 2)
    cos_d, sin_d, at = cuda(cos), cuda(sin), starts(lens)
    x = r.standard_normal((at[-1], q_heads + 2 * heads, size)).astype(np.float32)
    xd, pages, lens_d, offsets = cuda(x), cuda(w.table), int32(lens), int32(at)
    q, k, over, k_back, v_back = sequence_of_calls(w.cache, xd, q_heads, pages, lens_d, offsets, cos_d, sin_d)
    alone = tg.tst_attention(q, k, xd[:, q_heads + heads:], offsets)
    position = np.concatenate([np.arange(n) for n in lens])
    K, Q = (ref.rotate(x[:, a:b], position, cos, sin, False) for a, b in ((q_heads, q_heads + heads), (0, q_heads)))
    for i, n in enumerate(lens):
        w.ref.append("k", K[at[i]:at[i + 1]], w.table, i, 0)
        w.ref.append("v", x[at[i]:at[i + 1], q_heads + heads:], w.table, i, 0)
    w.assert_cache()
    want, bound = prompt_reference(Q, K, x[:, q_heads + heads:], at, 0.125, "f32")
    assert_within(alone, want, bound, "f32")
    want, bound = reference_over_cache(w, Q, lens, at, 0.125, "f32")
    assert_within(over, want, bound, "f32")
    # what a code stands for is off by half a step, a largest entry of a block over 254: logits by 64 of them, results by as much of the values
    assert (over - alone).abs().max() < 0.1
    for step in range(20):
        lens = [n + 1 for n in lens]
        w.lens = lens
        x = r.standard_normal((3, q_heads + 2 * heads, size)).astype(np.float32) * 1.5
        q, k, over, *_ = sequence_of_calls(w.cache, cuda(x), q_heads, pages, int32(lens), None, cos_d, sin_d)
        K, Q = (ref.rotate(x[:, a:b], np.array(lens) - 1, cos, sin, False) for a, b in ((q_heads, q_heads + heads), (0, q_heads)))
        for i, n in enumerate(lens):
            w.ref.append("k", K[i:i + 1], w.table, i, n - 1)
            w.ref.append("v", x[i:i + 1, q_heads + heads:], w.table, i, n - 1)
        w.assert_cache(f"step {step}")
        want, bound = reference_over_cache(w, Q, [1] * 3, [0, 1, 2, 3], 0.125, "f32")
        assert_within(over, want, bound, "f32")


@pytest.mark.parametrize("columns", [40, 1000])
def test_from_a_graph_and_on_another_stream(columns):
    """Captured once, replayed as the sequences grow, with eager work between; the same on a stream that is given."""
    heads, q_heads, size, page = 2, 8, 128, 16
    start = [30, 500, 16]
    worlds = [World([n + 8 for n in start], heads, size, page, 43, columns=columns) for _ in range(3)]
    g = torch.Generator(device="cuda").manual_seed(43)
    cos, sin = (cuda(t) for t in angles(600, size // 2))
    x = torch.randn((3, q_heads + 2 * heads, size), generator=g, device="cuda").bfloat16()
    pages, lens = cuda(worlds[0].table), int32([n + 1 for n in start])
    offsets = int32([0, 3])
    side = torch.cuda.Stream()

    def eager(w, **kw):
        return (*sequence_of_calls(w.cache, x, q_heads, pages, lens, None, cos, sin, **kw),
                tg.tst_attention(x[:, :q_heads], x[:, q_heads:q_heads + heads], x[:, q_heads + heads:], offsets, **kw))

    eager(worlds[0])
    eager(worlds[1])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured = eager(worlds[1])
    for step in range(6):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        lens += 1
        want = eager(worlds[0])
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        other = eager(worlds[2], stream=side)
        torch.cuda.current_stream().wait_stream(side)
        for a, b, c in zip(want, captured, other):
            assert torch.equal(a, b) and (step == 0 or torch.equal(a, c))
        if step == 0:      # the third cache has not had the first token
            worlds[2].cache.k_codes.copy_(worlds[0].cache.k_codes)
            worlds[2].cache.v_codes.copy_(worlds[0].cache.v_codes)
            worlds[2].cache.k_scale.copy_(worlds[0].cache.k_scale)
            worlds[2].cache.v_scale.copy_(worlds[0].cache.v_scale)
        torch.randn((1000, 1000), device="cuda").sum().item()


def test_two_graphs_that_share_a_workspace():
    w = World([3000, 40], 1, 64, 64, 44)
    pages, lens = w.arrays()
    Q = [strided(queries(w, 2, 4, 64, s), "f16") for s in (44, 45)]
    want = [tg.tst_kv_attention(q, w.cache, pages, lens) for q in Q]
    ws, out, graphs = torch.empty(8 << 20, dtype=torch.uint8, device="cuda"), [torch.empty_like(q) for q in Q], []
    for q, y in zip(Q, out):
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            tg.tst_kv_attention(q, w.cache, pages, lens, Y=y, workspace=ws)
        graphs.append(graph)
    for _ in range(3):
        for y in out:
            y.zero_()
        ws.fill_(255)
        for graph in (*graphs, *graphs[::-1]):
            graph.replay()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_same_results_both_ways(dtype, monkeypatch):
    """Through the binding's native half and past it."""
    from paper_2510_06957_amd import attention
    heads, q_heads, size = 2, 4, 80
    worlds = [World([65, 300, 9], heads, size, 32, 46) for _ in range(2)]
    x = strided(rng(46, 2).standard_normal((6, q_heads + 2 * heads, size)), dtype)
    pages, lens, offsets = cuda(worlds[0].table), int32([65, 300, 9]), int32([0, 3, 5, 6])
    cos, sin = (cuda(t) for t in angles(300, 20))
    assert attention._native is not None
    a = sequence_of_calls(worlds[0].cache, x, q_heads, pages, lens, offsets, cos, sin)
    a += (tg.tst_attention(x[:, :4], x[:, 4:6], x[:, 6:], offsets), tg.tst_attention(x[:, :4], x[:, 4:6], x[:, 6:], offsets, scale=0.2))
    monkeypatch.setattr(attention, "_native", None)
    b = sequence_of_calls(worlds[1].cache, x, q_heads, pages, lens, offsets, cos, sin)
    b += (tg.tst_attention(x[:, :4], x[:, 4:6], x[:, 6:], offsets), tg.tst_attention(x[:, :4], x[:, 4:6], x[:, 6:], offsets, scale=0.2))
    for s, t in zip(a, b):
        assert torch.equal(s, t) and s.dtype == t.dtype
    for s, t in zip(worlds[0].cache._tensors, worlds[1].cache._tensors):
        assert torch.equal(s, t)


def test_what_does_not_fit_is_refused():
    w = World([40, 9], 2, 64, 16, 47)
    pages, lens = w.arrays()
    x = torch.zeros((2, 8, 64), device="cuda")
    K, Q = x[:, :2], x[:, :4]
    cos = torch.zeros((50, 32), device="cuda")
    two = int32([0, 1, 2])
    before = w.download()

    def refused(call, *args, **kw):
        with pytest.raises((ValueError, tg.TstgemmError)):
            call(*args, **kw)

    for bad in (K.cpu(), K.double(), K.to(torch.int8), x[:, :3], x[:1, :2], x[:, :2, :32], x[:, :2].transpose(1, 2), K[0], None):
        refused(tg.tst_kv_append, w.cache, bad, K, pages, lens)
        refused(tg.tst_kv_append, w.cache, K, bad, pages, lens)
    for bad in (pages.long(), pages[0], pages[:, :0], pages.cpu(), pages.float(), pages.t().contiguous().t(), pages[:1], None):
        refused(tg.tst_kv_append, w.cache, K, K, bad, lens)
        refused(tg.tst_kv_attention, Q, w.cache, bad, lens)
        refused(tg.tst_kv_read, w.cache, bad, lens, 2)
    for bad in (lens.long(), lens[:1], lens.cpu(), torch.zeros(4, dtype=torch.int32, device="cuda")[::2], None):
        refused(tg.tst_kv_append, w.cache, K, K, pages, bad)
        refused(tg.tst_kv_attention, Q, w.cache, pages, bad)
        refused(tg.tst_kv_read, w.cache, pages, bad, 2)
    for bad in (two.long(), two[:2], two.cpu(), int32([0, 1, 2, 2])):
        refused(tg.tst_kv_append, w.cache, K, K, pages, lens, bad)
        refused(tg.tst_kv_attention, Q, w.cache, pages, lens, bad)
        refused(tg.tst_kv_read, w.cache, pages, lens, 2, bad)
    refused(tg.tst_kv_append, w.cache, K[:1], K[:1], pages, lens)          # a token for each sequence
    refused(tg.tst_kv_append, None, K, K, pages, lens)
    refused(tg.tst_kv_append, w.cache, K, K.bfloat16(), pages, lens)
    for kw in (dict(Q=Q), dict(keys=True), dict(cos=cos), dict(sin=cos), dict(Q=Q, cos=cos, sin=cos[:, :31]), dict(Q=Q.half(), cos=cos, sin=cos), dict(Q=Q[:1], cos=cos, sin=cos),
               dict(Q=Q[:, :, :32], cos=cos, sin=cos), dict(cos=cos.half(), sin=cos), dict(cos=torch.zeros((50, 33), device="cuda"), sin=torch.zeros((50, 33), device="cuda")),
               dict(cos=cos[:, :0], sin=cos[:, :0]), dict(cos=cos[:0], sin=cos[:0]), dict(cos=cos[0], sin=cos[0])):
        refused(tg.tst_kv_append, w.cache, K, K, pages, lens, **kw)
    for bad in (x[:, :3], x[:, :4, :32], Q.double(), Q.cpu(), Q[:1], Q[0], None):
        refused(tg.tst_kv_attention, bad, w.cache, pages, lens)
    refused(tg.tst_kv_attention, Q, None, pages, lens)
    for scale in (float("nan"), float("inf"), -float("inf")):
        refused(tg.tst_kv_attention, Q, w.cache, pages, lens, scale=scale)
        refused(tg.tst_attention, Q, K, K, two, scale=scale)
    for Y in (Q.bfloat16(), Q[:1], torch.empty((4, 2, 64), device="cuda").transpose(0, 1), Q.cpu()):
        refused(tg.tst_kv_attention, Q, w.cache, pages, lens, Y=Y)
        refused(tg.tst_attention, Q, K, K, two, Y=Y)
    refused(tg.tst_kv_read, w.cache, pages, lens, -1, two)
    refused(tg.tst_kv_read, w.cache, pages, lens, 3)
    refused(tg.tst_kv_read, w.cache, pages, lens, 2, dtype=torch.float64)
    refused(tg.tst_kv_read, w.cache, pages, lens, (1 << 22) + 1, two)
    for q, k, v in ((Q, K, x[:, :1]), (x[:, :3], K, K), (Q, K.half(), K), (Q, K, K.half()), (Q, K[:1], K[:1]), (Q, K[:, :, :32], K[:, :, :32]), (Q.cpu(), K, K), (Q, K, None), (Q[0], K, K)):
        refused(tg.tst_attention, q, k, v, two)
    for bad in (two.long(), two.cpu(), two[:0], two[None], [0, 2], torch.zeros(6, dtype=torch.int32, device="cuda")[::2]):
        refused(tg.tst_attention, Q, K, K, bad)
    wide = torch.zeros((2, 4, 257), device="cuda")
    refused(tg.tst_attention, wide, wide, wide, two)
    neg = torch._neg_view(K)
    refused(tg.tst_kv_append, w.cache, neg, K, pages, lens)
    refused(tg.tst_attention, Q, neg, K, two)
    for bad in (dict(pages=0), dict(page=17), dict(page=8), dict(page=512), dict(heads=0), dict(heads=1025), dict(head_size=0), dict(head_size=257)):
        refused(tg.tst_kv_cache, **{**dict(pages=2, page=16, heads=1, head_size=8), **bad})
    c = w.cache
    for bad in ((c.k_codes[:1], c.v_codes, c.k_scale, c.v_scale), (c.k_codes, c.k_codes, c.k_scale, c.v_scale), (c.k_codes.float(), c.v_codes, c.k_scale, c.v_scale),
                (c.k_codes, c.v_codes, c.k_scale[:1], c.v_scale), (c.k_codes, c.v_codes, c.k_scale, c.v_scale.double()), (c.k_codes, c.v_codes, c.k_scale, None)):
        refused(tg.KvCache, 16, 64, *bad)
    refused(tg.KvCache, 32, 64, *c._tensors)
    refused(tg.KvCache, 16, 65, *c._tensors)
    torch.cuda.synchronize()
    after = w.download()
    for name in "kv":
        same(after[name][0], before[name][0])
        same(after[name][1], before[name][1])
