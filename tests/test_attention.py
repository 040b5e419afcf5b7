"""Host-side checks of include/tst_attention.h (no GPU): symbols, sizes, refusals of the C entry points."""
import ctypes
import pathlib
import re
import subprocess

import pytest

import paper_2510_06957_amd as tg
from paper_2510_06957_amd import attention

ROOT = pathlib.Path(__file__).resolve().parent.parent
EINVAL, EWORKSPACE = -1, -8
a = 1 << 20     # an address that is not looked at


def cache(**change):
    f = dict(struct_size=ctypes.sizeof(attention._CacheStruct), pages=10, page_tokens=32, heads=2, head_size=64, k_codes=a, v_codes=a, k_scale=a, v_scale=a)
    f.update(change)
    return attention._CacheStruct(**f)


def sequences(**change):
    f = dict(struct_size=ctypes.sizeof(attention._SequencesStruct), sequences=3, tokens=5, offsets=a, lens=a, table=a, columns=4, table_stride=4)
    f.update(change)
    return attention._SequencesStruct(**f)


def heads(**change):
    f = dict(data=a, token_stride=512, head_stride=64)
    f.update(change)
    return attention._HeadsStruct(**f)


def rotation(**change):
    f = dict(struct_size=ctypes.sizeof(attention._RotationStruct), cos=a, sin=a, positions=100, pairs=32, interleaved=0)
    f.update(change)
    return attention._RotationStruct(**f)


BAD_CACHES = [dict(struct_size=8), dict(pages=0), dict(pages=-1), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=512), dict(heads=0), dict(heads=1025), dict(head_size=0),
              dict(head_size=257), dict(k_codes=None), dict(v_codes=a + 8), dict(k_scale=None), dict(v_scale=a + 2)]
BAD_SEQUENCES = [dict(struct_size=8), dict(sequences=-1), dict(sequences=(1 << 20) + 1), dict(tokens=-1), dict(tokens=(1 << 22) + 1), dict(offsets=None), dict(offsets=a + 2), dict(lens=None),
                 dict(table=None), dict(columns=0), dict(columns=1 << 26), dict(table_stride=3), dict(table_stride=1 << 62)]
BAD_HEADS = [dict(data=None), dict(data=a + 1), dict(token_stride=-1), dict(head_stride=-64), dict(token_stride=1 << 40)]


def test_every_declared_symbol_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "tst_attention.h").read_text(), flags=re.S)
    names = set(re.findall(r"\bint\s+(tst_\w+)\s*\(", text))
    assert names == set(attention._SIGNATURES) and len(names) == 7
    lib = ctypes.CDLL(str(tg.library_path()))
    for n in names:
        assert hasattr(lib, n)
    for n in ("KvCache", "tst_kv_cache", "tst_kv_append", "tst_kv_read", "tst_kv_attention", "tst_attention"):
        assert n in tg.__all__ and callable(getattr(tg, n))


def test_the_header_is_plain_c(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "tst_attention.h"\nint main(void) {\n    size_t codes = 0, scales = 0;\n    tst_kv_cache_t c = {sizeof(tst_kv_cache_t), 1, 16, 1, 8, 0, 0, 0, 0};\n'
                   "    return tst_kv_cache_bytes(3, 32, 2, 80, &codes, &scales) != TSTGEMM_OK || codes != 3 * 32 * 2 * 96 || scales != 12 ||\n"
                   "           tst_kv_row(1) != 64 || tst_kv_read(&c, 0, TST_F32, 0, 0, 0) != TSTGEMM_EINVAL;\n}\n")
    lib = tg.library_path()
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", f"-I{ROOT / 'include'}", str(src), "-o", str(tmp_path / "use"),
                    str(lib), f"-Wl,-rpath,{lib.parent}", "-Wl,-rpath,/opt/rocm/lib", "-L/opt/rocm/lib"], check=True)
    subprocess.run([str(tmp_path / "use")], check=True)


@pytest.mark.parametrize("size,row", [(-1, 0), (0, 0), (1, 64), (64, 64), (65, 96), (80, 96), (96, 96), (97, 128), (128, 128), (129, 192), (192, 192), (193, 256), (256, 256), (257, 0)])
def test_rows_of_codes(size, row):
    lib = attention._ops()
    assert lib.tst_kv_row(size) == row
    codes, scales = ctypes.c_size_t(), ctypes.c_size_t()
    rc = lib.tst_kv_cache_bytes(1 << 20, 256, 1024, size, ctypes.byref(codes), ctypes.byref(scales))
    assert rc == (0 if row else EINVAL) and (not row or (codes.value == 2 ** 38 * row and scales.value == 2 ** 34))


def test_refusals_of_the_cache():
    lib = attention._ops()
    k, s, r = heads(), sequences(), rotation()
    c, need = cache(), ctypes.c_size_t()
    ref = ctypes.byref
    for change in BAD_CACHES:
        bad = ref(cache(**change))
        assert lib.tst_kv_append(bad, ref(s), 0, ref(k), ref(k), None, 0, None, None, None, None) == EINVAL, change
        assert lib.tst_kv_read(bad, ref(s), 0, a, a, None) == EINVAL, change
        assert lib.tst_kv_attention_workspace_bytes(bad, ref(s), 4, ref(need)) == EINVAL, change
        assert lib.tst_kv_attention(ref(k), 0, 4, bad, ref(s), 1.0, a, a, 1 << 40, None) == EINVAL, change
    for change in BAD_SEQUENCES:
        bad = ref(sequences(**change))
        assert lib.tst_kv_append(ref(c), bad, 0, ref(k), ref(k), None, 0, None, None, None, None) == EINVAL, change
        assert lib.tst_kv_read(ref(c), bad, 0, a, a, None) == EINVAL, change
        assert lib.tst_kv_attention(ref(k), 0, 4, ref(c), bad, 1.0, a, a, 1 << 40, None) == EINVAL, change
    for change in BAD_HEADS:
        bad = ref(heads(**change))
        assert lib.tst_kv_append(ref(c), ref(s), 1, bad, ref(k), None, 0, None, None, None, None) == EINVAL, change
        assert lib.tst_kv_append(ref(c), ref(s), 1, ref(k), bad, None, 0, None, None, None, None) == EINVAL, change
        assert lib.tst_kv_append(ref(c), ref(s), 1, ref(k), ref(k), bad, 4, ref(r), a, None, None) == EINVAL, change
        assert lib.tst_kv_attention(bad, 1, 4, ref(c), ref(s), 1.0, a, a, 1 << 40, None) == EINVAL, change
        for i in range(3):
            assert lib.tst_attention(*(bad if i == j else ref(k) for j in range(3)), 1, 4, 2, 64, a, 1, 5, 1.0, a, None) == EINVAL, change
    for change in (dict(struct_size=8), dict(cos=None), dict(sin=None), dict(cos=a + 2), dict(positions=0), dict(pairs=0), dict(pairs=33)):
        assert lib.tst_kv_append(ref(c), ref(s), 1, ref(k), ref(k), ref(k), 4, ref(rotation(**change)), a, a, None) == EINVAL, change
    ok = [ref(c), ref(s), 1, ref(k), ref(k), ref(k), 4, ref(r), a, a, None]   # cache, sequences, type, K, V, Q, q_heads, rotation, q_out, k_out, stream
    for i, v in ((2, 3), (2, -1), (3, None), (4, None), (5, None), (6, 0), (6, 1025), (8, None), (8, a + 1), (9, a + 1)):
        assert lib.tst_kv_append(*ok[:i], v, *ok[i + 1:]) == EINVAL, i
    for i, v in ((2, 5), (3, None), (4, None), (3, a + 1)):
        args = [ref(c), ref(s), 1, a, a, None]
        assert lib.tst_kv_read(*args[:i], v, *args[i + 1:]) == EINVAL, i
    none = ref(sequences(sequences=0, tokens=0, offsets=None, lens=None, table=None))    # nothing to do
    assert lib.tst_kv_append(ref(c), none, 1, None, None, None, 0, None, None, None, None) == 0
    assert lib.tst_kv_read(ref(c), none, 1, None, None, None) == 0
    assert lib.tst_kv_attention(None, 1, 4, ref(c), none, 1.0, None, None, 0, None) == 0


def test_refusals_of_attention():
    lib, ref = attention._ops(), ctypes.byref
    c, s, q, need = cache(), sequences(), heads(), ctypes.c_size_t()
    assert lib.tst_kv_attention_workspace_bytes(ref(c), ref(s), 4, ref(need)) == 0
    assert need.value == 0                                              # 128 tokens at most: nothing is cut
    s = sequences(columns=400, table_stride=400)
    assert lib.tst_kv_attention_workspace_bytes(ref(c), ref(s), 4, ref(need)) == 0 and need.value > 0
    for heads_ in (0, 3, 1026, -2):
        assert lib.tst_kv_attention_workspace_bytes(ref(c), ref(s), heads_, ref(need)) == EINVAL
    assert lib.tst_kv_attention_workspace_bytes(ref(c), ref(s), 4, None) == EINVAL
    assert lib.tst_kv_attention_workspace_bytes(ref(c), ref(sequences(tokens=1 << 22)), 64, ref(need)) == EINVAL     # rows x heads
    n = need.value
    ok = [ref(q), 1, 4, ref(c), ref(s), 0.5, a, a, n, None]              # Q, type, q_heads, cache, sequences, scale, Y, workspace, bytes, stream
    for i, v, code in ((0, None, EINVAL), (1, 3, EINVAL), (2, 5, EINVAL), (5, float("nan"), EINVAL), (5, float("inf"), EINVAL), (5, 2.5e38, EINVAL), (6, None, EINVAL), (6, a + 1, EINVAL), (7, None, EWORKSPACE),
                       (8, n - 1, EWORKSPACE), (7, a + 128, EINVAL)):
        assert lib.tst_kv_attention(*ok[:i], v, *ok[i + 1:]) == code, i
    ok = [ref(q), ref(q), ref(q), 1, 4, 2, 64, a, 1, 5, 0.5, a, None]    # Q, K, V, type, q_heads, heads, size, offsets, sequences, tokens, scale, Y, stream
    for i, v in ((0, None), (1, None), (2, None), (3, 3), (4, 0), (4, 3), (4, 1026), (5, 0), (5, 3), (6, 0), (6, 257), (7, None), (7, a + 1), (8, -1), (8, (1 << 20) + 1), (9, -1), (9, (1 << 22) + 1),
                 (10, float("nan")), (10, float("-inf")), (10, -2.5e38), (11, None), (11, a + 1)):
        assert lib.tst_attention(*ok[:i], v, *ok[i + 1:]) == EINVAL, i
    assert lib.tst_attention(ref(q), ref(q), ref(q), 1, 64, 2, 64, a, 1, 1 << 22, 0.5, a, None) == EINVAL           # rows x heads
    assert lib.tst_attention(ref(q), ref(q), ref(q), 1, 1024, 1024, 64, a, 4097, 5, 0.5, a, None) == EINVAL         # sequences x heads
    for i in (8, 9):
        args = [None, None, None, 1, 4, 2, 64, None, 1, 5, 0.5, None, None]
        args[i] = 0
        assert lib.tst_attention(*args) == 0                             # nothing to do


def test_sizes_beyond_32_bits_are_refused():
    for args in ((2 ** 32 + 4, 32, 2, 64), (4, 32, 2 ** 32 + 2, 64)):
        codes, scales = ctypes.c_size_t(), ctypes.c_size_t()
        with pytest.raises(tg.TstgemmError):
            attention._call("tst_kv_cache_bytes", *args, ctypes.byref(codes), ctypes.byref(scales))


@pytest.mark.parametrize("kind,at", [("_CacheStruct", 1), ("_CacheStruct", 3), ("_SequencesStruct", 1), ("_SequencesStruct", 2), ("_SequencesStruct", 6), ("_RotationStruct", 3),
                                     ("_RotationStruct", 4)])
@pytest.mark.parametrize("value", [2 ** 32 + 5, 2 ** 32, 2 ** 31, -2 ** 31 - 1])
def test_counts_of_structs_beyond_32_bits_are_refused(kind, at, value):
    kind = getattr(attention, kind)
    fields = [1] * len(kind._fields_)
    assert getattr(attention._struct(kind, "call", *fields), kind._fields_[at][0]) == 1
    fields[at] = value
    with pytest.raises(tg.TstgemmError) as e:
        attention._struct(kind, "call", *fields)
    assert e.value.code == EINVAL


def test_the_binding_and_its_native_half_refuse_what_is_not_on_a_gpu():
    import torch
    x, i = torch.zeros((2, 2, 64)), torch.zeros((2, 1), dtype=torch.int32)
    with pytest.raises(ValueError):
        tg.tst_attention(x, x, x, torch.tensor([0, 2], dtype=torch.int32))
    with pytest.raises(ValueError):
        tg.KvCache(16, 64, torch.zeros((1, 1, 16, 64), dtype=torch.int8), torch.zeros((1, 1, 1, 64, 16), dtype=torch.int8), torch.zeros((1, 1, 1)), torch.zeros((1, 1, 1)))
    with pytest.raises(ValueError):
        tg.tst_kv_append(None, x, x, i, i[:, 0])
    attention._ops()
    native = attention._native
    assert native is not None
    assert native.attention(x, x, x, i, None) is None and native.kv_attention(x, None, i, i, None, None) is None
    assert native.kv_append(None, x, x, i, i, None, None, None, None, False, False) is None and native.kv_read(None, i, i, 2, None, None) is None
    for call in (native.attention, native.kv_attention, native.kv_append, native.kv_read):
        with pytest.raises(TypeError):
            call(x)


@pytest.mark.parametrize("prompts,steps", [([], 3), ([[1, 2], []], 3), ([[]], 3), ([[1], [2000]], 3), ([[1, -1]], 3), ([[1]], 0)])
def test_the_example_refuses_prompts_that_it_has_no_answer_to(prompts, steps):
    import types

    import torch
    from paper_2510_06957_amd.decode_step import answer
    with pytest.raises(ValueError):
        answer(types.SimpleNamespace(embedding=torch.zeros((2000, 1))), prompts, steps)
