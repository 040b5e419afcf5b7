"""GPU tests of the cache and of attention where numbers are large or far apart: values near the largest there are, scales of blocks that differ, lengths and counts near
the ends of 32 bits, and a cache whose tensors are not what they were.  Against the definitions, as in test_gpu_attention.py."""
import math

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2510_06957_amd as tg
from test_gpu_attention import (PROMPT_CUT, PROMPT_WEIGHT, World, assert_within, cuda, f32, int32, prompt, prompt_reference, queries, reference_over_cache, rng, same, starts, strided)

pytestmark = pytest.mark.gpu

LARGEST = {"f32": float(np.finfo(np.float32).max), "bf16": float(torch.finfo(torch.bfloat16).max)}


def test_counts_beyond_32_bits_are_refused():
    """2^32 and a few: their low 32 bits would do for a call."""
    w = World([40, 9], 1, 1, 16, 60)
    pages, lens = w.arrays()
    before, offsets = w.download(), int32([0, 3, 5])
    for n in (2 ** 32 + 5, 2 ** 32):
        many = torch.ones((1, 1, 1), device="cuda").expand(n, 1, 1)
        for call in (lambda: tg.tst_kv_read(w.cache, pages, lens, n, offsets), lambda: tg.tst_kv_append(w.cache, many, many, pages, lens, offsets),
                     lambda: tg.tst_kv_attention(many, w.cache, pages, lens, offsets)):
            with pytest.raises(tg.TstgemmError) as e:
                call()
            assert e.value.code == -1
    after = w.download()
    for name in "kv":
        same(after[name][0], before[name][0])
        same(after[name][1], before[name][1])


def test_a_cache_keeps_its_tensors():
    """What a cache says of itself cannot be set, and one whose tensors have been given other memory is refused, both halves of the binding."""
    from paper_2510_06957_amd import attention
    w = World([40, 9], 2, 64, 16, 66)
    pages, lens = w.arrays()
    x = torch.ones((2, 8, 64), device="cuda")
    c = w.cache
    for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
        with pytest.raises(AttributeError):
            setattr(c, name, getattr(c, name).clone())
    for name in ("pages", "page", "heads", "head_size", "device_index"):
        with pytest.raises(AttributeError):
            setattr(c, name, getattr(c, name) + 1)
    c.v_scale *= 1.0       # what is there already
    calls = (lambda: tg.tst_kv_append(c, x[:, :2], x[:, :2], pages, lens), lambda: tg.tst_kv_read(c, pages, lens, 2), lambda: tg.tst_kv_attention(x[:, :4], c, pages, lens))
    for t in (c.k_codes, c.v_codes, c.k_scale, c.v_scale):
        saved, other = t.data, t.clone()
        t.data = other
        for call in calls:
            with pytest.raises(ValueError):
                call()
        assert attention._native.kv_read(c, pages, lens, 2, None, None) is None
        t.data = saved
        for call in calls:
            call()


def test_lengths_beyond_2_30_tokens():
    """Behind the largest table there is: positions from 2^30 on have no page, whatever the length says."""
    columns = (1 << 30) // 256
    r = rng(65)
    for k, there in ((4, 3), (1000, 0), (2 ** 30 - 1, 0)):
        cache = tg.tst_kv_cache(2, 256, 1, 64)
        pages = torch.zeros((1, columns), dtype=torch.int32, device="cuda")
        pages[0, -1] = 1
        K, V = (cuda(r.standard_normal((7, 1, 64)).astype(np.float32)) for _ in "kv")
        lens, offsets = int32([(1 << 30) + k]), int32([0, 7])
        tg.tst_kv_append(cache, K, V, pages, lens, offsets)
        assert not cache.k_codes[0].any() and not cache.v_codes[0].any() and not cache.k_scale[0].any() and not cache.v_scale[0].any()
        assert not cache.k_codes[1, :, :253].any() and not cache.k_scale[1, :, :15].any()
        assert cache.k_codes[1, 0, 253:].any(1).tolist() == [there > 0] * 3
        for x, got in zip((K, V), tg.tst_kv_read(cache, pages, lens, 7, offsets, dtype=torch.float32)):
            assert torch.isnan(got[there:]).all() and (not there or (got[:there] - x[:there]).abs().max() < 0.03)
        if k < 2 ** 29:
            Y = tg.tst_kv_attention(K, cache, pages, lens, offsets)
            assert torch.isfinite(Y[:there]).all() and torch.isnan(Y[there:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("columns", [100, 1000])
@pytest.mark.parametrize("new", [1, 20])
def test_attention_over_the_cache_scales_of_blocks_that_weigh_nothing(new, columns, dtype):
    """A block whose tokens weigh nothing, with a scale of values far above the others', leaves them their bits.  Weights keep theirs (11; 22 in fp32) relative to the largest
    product of a weight and a scale, and 2^-32 (2^-40) of it below: n terms of 127 of that."""
    w = World([1500], 1, 64, 16, 64, columns=columns)
    w.ref.codes["k"][:] = np.abs(w.ref.codes["k"])
    at = [0, new]
    Qd = strided(np.abs(queries(w, new, 2, 64, 64)) + 0.5, dtype)
    pages, lens = w.arrays()
    for block in (0, 3, 40, 61, 91):
        page = w.table[0, block]
        saved = {n: (w.ref.codes[n][page].copy(), w.ref.scale[n][page].copy()) for n in "kv"}
        w.ref.codes["k"][page] = -127
        w.ref.scale["k"][page] = 0.2           # logits 100 and more below the others'
        w.ref.scale["v"][page] = 0
        want, bound = reference_over_cache(w, f32(Qd), [new], at, 0.125, dtype)
        bound = bound + 1500 * 2.0 ** (-40 if dtype == "f32" else -32) * 127 * 1.5 / 64
        for large in (1e6, 1e12, 1e30):
            w.ref.scale["v"][page] = large
            w.upload()
            assert_within(tg.tst_kv_attention(Qd, w.cache, pages, lens, int32(at)), want, bound, dtype, f"block {block} scale {large}")
        for n in "kv":
            w.ref.codes[n][page], w.ref.scale[n][page] = saved[n]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("columns", [100, 1000])
@pytest.mark.parametrize("new", [[1, 1], [30, 4]])
@pytest.mark.parametrize("alike", [False, True])
def test_attention_over_the_cache_of_large_values(alike, new, columns, dtype):
    """A result lies between the values it is a mean of, of hundreds of tokens that weigh about the same and stand for the largest there are."""
    w = World([900, 77], 2, 64, 16, 63, columns=columns)
    scale = np.nextafter(np.float32(LARGEST[dtype] / 127), np.float32(0))
    if alike:
        w.ref.codes["v"][:, 0], w.ref.codes["v"][:, 1] = 127, -127
        w.ref.scale["v"][:] = scale
    else:
        w.ref.codes["v"][:] = np.abs(w.ref.codes["v"])
        w.ref.scale["v"][:] = scale * (0.5 + 0.5 * w.r.random(w.ref.scale["v"].shape))
    w.upload()
    at = starts(new)
    Qd = strided(queries(w, at[-1], 4, 64, 63, 0.01), dtype)
    pages, lens = w.arrays()
    want, bound = reference_over_cache(w, f32(Qd), new, at, 0.125, dtype)
    Y = tg.tst_kv_attention(Qd, w.cache, pages, lens, int32(at))
    assert torch.isfinite(Y).all()
    assert_within(Y, want, bound, dtype)


@pytest.mark.parametrize("columns", [100, 1000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_over_the_cache_queries_and_scales_far_from_one(dtype, columns):
    """Logits are ordinary numbers, or 0, where a query times the factor is beyond 32 bits, or below."""
    w = World([500, 30], 2, 64, 16, 68, columns=columns)
    pages, lens = w.arrays()
    for large, factor, keys in ((2.0 ** 60, 2.0 ** 127, 0.0), (2.0 ** 100, 2.0 ** 46, 2.0 ** -148), (2.0 ** -126, 2.0 ** -2, 2.0 ** 119), (2.0 ** -140, 2.0 ** 8, 2.0 ** 119), (2.0 ** 100, 2.0 ** -145, 2.0 ** 38)):
        w.ref.scale["k"][:] = keys
        w.upload()
        Qd = strided(queries(w, 2, 4, 64, 68, large), dtype)
        want, bound = reference_over_cache(w, f32(Qd), [1, 1], [0, 1, 2], factor, dtype)
        assert_within(tg.tst_kv_attention(Qd, w.cache, pages, lens, scale=factor), want, bound, dtype, f"{large} {factor} {keys}")


@pytest.mark.parametrize("scale", [0.0, 2.0 ** -140, -2.0 ** -133, 2.0 ** -126])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [[200, 33], [100] * 30])
def test_prompts_small_scales(lens, dtype, scale):
    """Products of queries and keys near 2^126, times next to nothing."""
    q, k, v = prompt(lens, 4, 2, 64, dtype, 67, large=2e18)
    at = starts(lens)
    want, bound = prompt_reference(f32(q), f32(k), f32(v), at, scale, dtype, None, np.arange(0, 200, 7))
    rows = np.concatenate([a + np.arange(0, b - a, 7) for a, b in zip(at, at[1:])])
    assert_within(f32_rows(tg.tst_attention(q, k, v, int32(at), scale=scale), rows), want[rows], bound[rows], dtype)


def f32_rows(Y, rows):
    return Y[torch.from_numpy(rows).cuda()]


def large_prompt(lens, q_heads, heads, size, dtype, most, gap):
    """Logits of 0 and now and then 7 powers of two more; values of up to `most`, of one sign in a channel."""
    T, r = sum(lens), rng(61, sum(lens), size)
    Q, K, V = (np.zeros((T, h, size)) for h in (q_heads, heads, heads))
    Q[..., 0] = 1
    K[..., 0] = np.where(r.random((T, heads)) < 0.02, 7 * math.log(2), 0)
    K[20:40, :, 0] = 0
    V[:] = (0.5 + 0.5 * r.random(V.shape)) * most
    V[20:45] = most
    V[..., 1::2] *= -1
    return [strided(np.clip(x, -LARGEST[dtype], LARGEST[dtype]), dtype, gap) for x in (Q, K, V)]


@pytest.mark.parametrize("lens,q_heads,heads,size,gap", [([300, 33], 4, 2, 64, 0), ([100, 33, 1], 4, 2, 96, 0), ([1217, 64], 64, 2, 64, 0), ([1217, 835], 64, 16, 128, 0),
                                                          ([130, 41], 4, 2, 200, 0), ([130, 41], 4, 2, 64, 3), ([700], 2, 1, 128, 0)])
@pytest.mark.parametrize("most", [1e37, None])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompts_of_large_values(dtype, most, lens, q_heads, heads, size, gap):
    """A result lies between the values it is a mean of, however many there are and however large."""
    q, k, v = large_prompt(lens, q_heads, heads, size, dtype, most or LARGEST[dtype], gap)
    at = starts(lens)
    few = sorted({0, q_heads // 2, q_heads - 1})
    rows = np.unique(np.r_[np.arange(0, 70), np.arange(120, 135), np.arange(250, 262), np.arange(1200, 1217)])
    seen = np.concatenate([a + rows[rows < b - a] for a, b in zip(at, at[1:])])
    Y = tg.tst_attention(q, k, v, int32(at), scale=1.0)
    want, bound = prompt_reference(f32(q), f32(k), f32(v), at, 1.0, dtype, few, rows)
    assert torch.isfinite(Y).all()
    assert_within(Y[torch.from_numpy(seen).cuda()][:, few], want[seen][:, few], bound[seen][:, few], dtype)
    assert torch.equal(tg.tst_attention(q, k, v, int32(at), scale=1.0), Y)


@pytest.mark.parametrize("lens,q_heads,size", [([90, 40], 4, 64), ([300, 77], 4, 64), ([1217, 64], 64, 64), ([130, 41], 4, 200)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompts_large_values_that_a_row_does_not_see_do_not_touch_it(dtype, lens, q_heads, size):
    """From a row on values are as large as there are, or none in a channel; rows before it, and the other sequence, keep their last bit."""
    q, k, v = (strided(x.cpu().float().numpy(), dtype) for x in prompt(lens, q_heads, 2, size, dtype, 62))
    at = starts(lens)
    clean = tg.tst_attention(q, k, v, int32(at))
    cut = lens[0] - 20
    v[cut:lens[0]] = LARGEST[dtype]
    v[cut + 5:lens[0], :, 3] = float("inf")
    v[cut + 9:lens[0], :, 5] = float("nan")
    Y = tg.tst_attention(q, k, v, int32(at))
    assert torch.equal(Y[:cut], clean[:cut]) and torch.equal(Y[lens[0]:], clean[lens[0]:])
    spoilt = torch.zeros(Y.shape, dtype=torch.bool, device="cuda")
    spoilt[cut + 5:lens[0], :, 3] = True
    spoilt[cut + 9:lens[0], :, 5] = True
    assert torch.equal(~torch.isfinite(Y), spoilt)
    few, rows = [0, q_heads - 1], np.arange(cut, lens[0])
    finite = np.where(np.isfinite(f32(v)), f32(v), 0)
    want, bound = prompt_reference(f32(q), f32(k), finite, at, 1 / math.sqrt(size), dtype, few, rows)
    got, keep = f32(Y)[rows][:, few], ~spoilt[cut:lens[0]].cpu().numpy()[:, few]
    assert_within(torch.from_numpy(np.where(keep, got, 0)), np.where(keep, want[rows][:, few], 0), np.where(keep, bound[rows][:, few], 0), dtype)


@pytest.mark.parametrize("q_heads,heads,size", [(64, 8, 64), (64, 8, 80), (64, 16, 128), (66, 2, 96)])
@pytest.mark.parametrize("lens", [[1217, 835], [1217, 0, 3, 64, 65, 400, 1]])
def test_prompts_in_whole_tiles_fp32(lens, q_heads, heads, size):
    """Enough rows for the kernel of large calls, over many tiles of keys; a few heads and rows of each sequence against the definition."""
    q, k, v = prompt(lens, q_heads, heads, size, "f32", 69)
    at = starts(lens)
    Y = tg.tst_attention(q, k, v, int32(at))
    few = [0, q_heads // 2 + 1, q_heads - 1]
    rows = np.unique(np.r_[np.arange(0, 70), np.arange(120, 135), np.arange(250, 262), np.arange(820, 835), np.arange(1200, 1217)])
    seen = np.concatenate([a + rows[rows < b - a] for a, b in zip(at, at[1:])])
    want, bound = prompt_reference(f32(q), f32(k), f32(v), at, 1 / math.sqrt(size), "f32", few, rows)
    assert_within(f32_rows(Y, seen)[:, few], want[seen][:, few], bound[seen][:, few], "f32")
    assert torch.equal(tg.tst_attention(q, k, v, int32(at)), Y)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lens,q_heads,size", [([90, 40], 4, 64), ([300, 77], 4, 80), ([1217, 64], 64, 64), ([130, 41], 4, 200)])
def test_prompts_keys_whose_logits_are_minus_infinity(lens, q_heads, size, dtype):
    """In 16 bits they weigh nothing; in fp32, whose three planes have none for an infinity, rows that see one are NaN."""
    q, k, v = prompt(lens, q_heads, 2, size, dtype, 70)
    at, j = starts(lens), 30
    q[..., 0] = q[..., 0].abs() + 0.5
    clean = tg.tst_attention(q, k, v, int32(at))
    k[j, :, 0] = -float("inf")
    Y = tg.tst_attention(q, k, v, int32(at))
    assert torch.equal(Y[:j], clean[:j]) and torch.equal(Y[lens[0]:], clean[lens[0]:])
    if dtype == "f32":
        assert torch.isnan(Y[j:lens[0]]).all()
        return
    rows = np.r_[j, j + 1, np.arange(40, lens[0], 37), lens[0] - 1]
    for h in (0, q_heads - 1):
        K, V = (np.delete(f32(t)[:lens[0], h // (q_heads // 2)].astype(np.float64), j, 0) for t in (k, v))
        want, bound = ref.attention(f32(q)[rows, h].astype(np.float64), K, V, rows, 1 / math.sqrt(size), PROMPT_WEIGHT[dtype], PROMPT_CUT[dtype])
        assert_within(Y[torch.from_numpy(rows).cuda(), h], want, bound, dtype)
