"""GPU tests of the cache and of attention where numbers are large or far apart: values near the largest there are, scales of blocks that differ, lengths and counts near
the ends of 32 bits, and a cache whose tensors are not what they were.  Against the definitions, as in test_gpu_attention.py."""
import math

import numpy as np
import pytest
import torch

import paper_2510_06957_amd as tg
from test_gpu_attention import (TYPES, World, assert_within, cuda, f32, int32, prompt, prompt_reference, queries, reference_over_cache, rng, same, starts, strided)

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
