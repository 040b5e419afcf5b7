"""Host-side checks of the operators in include/tst_ops.h (no GPU): symbols, sizes, refusals of the C entry points."""
import ctypes
import pathlib
import re
import subprocess

import pytest

import paper_2510_06957_amd as tg
from paper_2510_06957_amd import operators

ROOT = pathlib.Path(__file__).resolve().parent.parent
EINVAL, EWORKSPACE = -1, -8
P = ctypes.c_void_p


def test_every_declared_symbol_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "tst_ops.h").read_text(), flags=re.S)
    names = set(re.findall(r"\bint\s+(tst_\w+)\s*\(", text))
    assert names == set(operators._SIGNATURES) and len(names) == 10
    lib = ctypes.CDLL(str(tg.library_path()))
    for n in names:
        assert hasattr(lib, n)
    for n in ("tst_quantize", "tst_w8_pack", "tst_w8_gemm", "tst_w8_linear", "tst_moe_pack", "tst_moe", "tst_logprobs"):
        assert n in tg.__all__ and callable(getattr(tg, n))


def test_the_header_is_plain_c(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "tst_ops.h"\nint main(void) { size_t n = 0; return tst_w8_bytes(65, 17, &n) != TSTGEMM_OK || n != 4096; }\n')
    lib = tg.library_path()
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", f"-I{ROOT / 'include'}", str(src), "-o", str(tmp_path / "use"),
                    str(lib), f"-Wl,-rpath,{lib.parent}", "-Wl,-rpath,/opt/rocm/lib", "-L/opt/rocm/lib"], check=True)
    subprocess.run([str(tmp_path / "use")], check=True)


@pytest.mark.parametrize("K,N,want", [(1, 1, 1024), (64, 16, 1024), (65, 16, 2048), (64, 17, 2048), (4096, 11008, 4096 * 11008), (131071, 33, 131072 * 48)])
def test_w8_bytes(K, N, want):
    assert operators._bytes("tst_w8_bytes", K, N) == want


def test_the_gpu_tests_take_every_tile_of_the_8_bit_product(tmp_path):
    """The rule itself, compiled for the host: a change of it may not leave a kernel without a test."""
    from w8_tiles import FAR, TILES
    src = tmp_path / "choice.cpp"
    src.write_text('#include "w8_choice.h"\n#include <cstdio>\nint main()\n{\n'
                   '    for (const auto &t : tst::kGemmTiles) std::printf("%s %d %d\\n", t.rows ? "rows" : "tiles", t.mt, t.nt);\n'
                   '    int M, K, N;\n'
                   '    while (std::scanf("%d%d%d", &M, &K, &N) == 3) {\n'
                   '        const auto t = tst::choose_tile(M, K, N, 256);\n'
                   '        std::printf("%s %d %d\\n", t.rows ? "rows" : "tiles", t.mt, t.nt);\n    }\n}\n')
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", f"-I{ROOT / 'paper_2510_06957_amd' / 'csrc'}", str(src), "-o", str(tmp_path / "choice")], check=True)
    shapes = [(tile, s) for tile, all_ in TILES.items() for s in all_] + list(FAR.items())
    out = subprocess.run([str(tmp_path / "choice")], input="\n".join("%d %d %d" % s for _, s in shapes), text=True, capture_output=True, check=True).stdout
    tiles = [(k, int(m), int(n)) for k, m, n in (line.split() for line in out.splitlines())]
    there, chosen = tiles[:len(TILES)], tiles[len(TILES):]
    assert set(there) == set(TILES) and len(chosen) == len(shapes)
    for (tile, shape), got in zip(shapes, chosen):
        assert got == tile, shape


def moe_struct(**change):
    fields = dict(struct_size=ctypes.sizeof(operators._MoeStruct), type=1, experts=8, width=64, inner=64)
    fields.update({n: 4096 for n in ("router", "gate", "up", "down", "gate_scale", "up_scale", "down_scale")})
    fields.update(change)
    return operators._MoeStruct(**fields)


def test_refusals():
    """Nothing here reaches the GPU: the addresses are not looked at."""
    lib = operators._ops()
    a = 1 << 20
    n = ctypes.c_size_t()
    for args in ((0, 4), (4, 0), (131072, 4), (-1, 4)):
        assert lib.tst_w8_bytes(*args, ctypes.byref(n)) == EINVAL
    assert lib.tst_w8_bytes(4, 4, None) == EINVAL
    for args in ((None, 1, 4, 4, a), (a, 1, 4, 4, None), (a, 0, 4, 4, a), (a, 1, 0, 4, a), (a, 1, 131072, 4, a), (a, 1, 4, 4, a + 8)):
        assert lib.tst_w8_pack(*args, None) == EINVAL
    ok = [a, 0, 64, a, 64, a, 2, 64, None]     # X, type, stride, Q, stride, scale, M, K, stream
    for i, v in ((0, None), (0, a + 2), (1, 3), (1, -1), (2, 63), (3, None), (4, 63), (5, None), (6, -1), (7, 0), (7, 2 ** 30 + 1)):
        assert lib.tst_quantize(*ok[:i], v, *ok[i + 1:]) == EINVAL, i
    ok = [a, 64, a, a, a, None, a, 1, 2, 64, 32, None]   # Q, stride, scale, packed, w_scale, b, Y, type, M, K, N, stream
    for i, v in ((0, None), (0, a + 8), (1, 63), (1, 72), (2, None), (3, None), (3, a + 8), (4, None), (6, None), (6, a + 1), (7, 3), (8, -1),
                 (9, 0), (9, 131072), (10, 0)):
        assert lib.tst_w8_gemm(*ok[:i], v, *ok[i + 1:]) == EINVAL, i
    need = operators._bytes("tst_w8_linear_workspace_bytes", 2, 64)
    ok = [a, 1, 64, a, a, None, a, 2, 64, 32, a, need, None]
    for i, v, code in ((0, None, EINVAL), (0, a + 1, EINVAL), (1, 5, EINVAL), (2, 63, EINVAL), (6, None, EINVAL), (10, None, EWORKSPACE),
                       (11, need - 1, EWORKSPACE), (10, a + 128, EINVAL)):
        assert lib.tst_w8_linear(*ok[:i], v, *ok[i + 1:]) == code, i
    assert lib.tst_w8_linear_workspace_bytes(-1, 4, ctypes.byref(n)) == EINVAL


def test_sizes_that_no_grid_counts_are_refused():
    """A dimension of a grid has fewer than 2^32 threads."""
    lib = operators._ops()
    a = 1 << 20
    for K, N in ((64, 1 << 30), (131071, 1 << 19), (1, 2 ** 31 - 1)):
        assert lib.tst_w8_pack(a, 1, K, N, a, None) == -6
    for N in ((1 << 27) - 15, 1 << 27, 2 ** 31 - 100):
        assert lib.tst_w8_gemm(a, 64, a, a, a, None, a, 1, 2, 64, N, None) == EINVAL
        assert lib.tst_w8_linear(a, 1, 64, a, a, None, a, 2, 64, N, a, 1 << 30, None) == EINVAL
    assert lib.tst_w8_gemm(a, 64, a, a, a, None, a, 1, 0, 64, (1 << 27) - 16, None) == 0   # no rows: nothing to do


def test_bytes_of_as_many_columns_as_there_can_be():
    for K, N, want in ((1, 2 ** 31 - 1, 2 ** 37), (131071, 2 ** 31 - 1, 2 ** 48)):
        assert operators._bytes("tst_w8_bytes", K, N) == want


def test_workspace_of_as_many_rows_as_there_can_be():
    for R in (2 ** 31 - 1, 2 ** 31 - 600, 1 << 24):
        assert operators._bytes("tst_logprobs_workspace_bytes", R, 1 << 20, 20) == 0


def test_refusals_of_moe():
    lib = operators._ops()
    a, n = 1 << 20, ctypes.c_size_t()
    s = moe_struct()
    assert lib.tst_moe_workspace_bytes(ctypes.byref(s), 5, 2, ctypes.byref(n)) == 0 and n.value > 0
    need = n.value
    for change in (dict(struct_size=8), dict(type=3), dict(experts=0), dict(experts=513), dict(width=0), dict(inner=131072)):
        assert lib.tst_moe_workspace_bytes(ctypes.byref(moe_struct(**change)), 5, 2, ctypes.byref(n)) == EINVAL, change
    for T, k in ((-1, 2), (5, 0), (5, 9), (5, 17)):
        assert lib.tst_moe_workspace_bytes(ctypes.byref(s), T, k, ctypes.byref(n)) == EINVAL
    assert lib.tst_moe_workspace_bytes(None, 5, 2, ctypes.byref(n)) == EINVAL
    ok = [a, 64, ctypes.byref(s), 2, 1, a, a, a, 5, a, need, None]   # X, stride, moe, k, normalize, Y, ids, p, T, workspace, bytes, stream
    for i, v, code in ((0, None, EINVAL), (0, a + 1, EINVAL), (1, 63, EINVAL), (2, None, EINVAL), (3, 9, EINVAL), (5, None, EINVAL), (6, None, EINVAL),
                       (7, None, EINVAL), (8, -1, EINVAL), (9, None, EWORKSPACE), (10, need - 1, EWORKSPACE), (9, a + 16, EINVAL)):
        assert lib.tst_moe(*ok[:i], v, *ok[i + 1:]) == code, i
    for name in ("router", "gate", "up", "down", "gate_scale", "up_scale", "down_scale"):
        ok[2] = ctypes.byref(moe_struct(**{name: None}))
        assert lib.tst_moe(*ok) == EINVAL, name
    ok[8] = 0
    assert lib.tst_moe(*ok) == 0   # no tokens: nothing to do


def test_refusals_of_logprobs():
    lib = operators._ops()
    a, n = 1 << 20, ctypes.c_size_t()
    for args in ((-1, 50, 3), (2, 0, 0), (2, 2 ** 30 + 1, 3), (2, 50, -1), (2, 50, 51), (2, 500, 65)):
        assert lib.tst_logprobs_workspace_bytes(*args, ctypes.byref(n)) == EINVAL
    ok = [a, 1, 50, a, 8, 1, 3, a, a, a, a, 2, 50, a, 1 << 30, None]
    # logits, type, stride, tokens, bytes, C, top, of_token, entropy, top_ids, of_top, R, V, workspace, bytes, stream
    for i, v in ((0, None), (0, a + 1), (1, 3), (2, 49), (3, None), (4, 2), (5, -1), (5, 65), (6, 51), (7, None), (9, None), (10, None), (11, -1), (12, 0)):
        assert lib.tst_logprobs(*ok[:i], v, *ok[i + 1:]) == EINVAL, i
    ok[11] = 0
    assert lib.tst_logprobs(*ok) == 0


def test_the_binding_refuses_what_is_not_on_a_gpu():
    import torch
    x = torch.zeros((2, 64))
    with pytest.raises(ValueError):
        tg.tst_quantize(x)
    with pytest.raises(ValueError):
        tg.tst_w8_pack(x.to(torch.int8), torch.ones(64))
    with pytest.raises(ValueError):
        tg.tst_logprobs(x)


def test_the_native_half_hands_back_what_is_not_on_a_gpu():
    import torch
    operators._ops()
    native = operators._native
    assert native is not None
    x = torch.zeros((2, 64))
    w = tg.W8(64, 32, 1, torch.zeros(2048, dtype=torch.uint8), torch.ones(32))
    for wrong in ((64, 33, torch.ones(33)), (128, 32, torch.ones(32)), (64, 32, torch.ones(31))):
        with pytest.raises(ValueError):
            tg.W8(wrong[0], wrong[1], 1, torch.zeros(2048, dtype=torch.uint8), wrong[2])
    assert native.w8_linear(x, w, None) is None and native.w8_gemm(x.to(torch.int8), torch.ones(2), w, None, None) is None
    assert native.moe(x, None, 2, True) is None and native.logprobs(x, None, 1) is None
    for call in (lambda: native.w8_linear(x), lambda: native.w8_gemm(x), lambda: native.moe(x), lambda: native.logprobs(x)):
        with pytest.raises(TypeError):
            call()


def test_w8_takes_no_tensors_that_hold_less_than_the_kernels_read():
    import torch
    packed, scale = torch.zeros(2048, dtype=torch.uint8), torch.ones(32)
    w = tg.W8(64, 32, 1, packed, scale)
    for p, s in ((packed[:1].expand(2048), scale), (torch.zeros(4096, dtype=torch.uint8)[::2], scale), (packed, scale[:1].expand(32)),
                 (packed, scale.to(torch.float16)), (packed.to(torch.bool), scale), (packed, scale.to("meta")), (packed.numpy(), scale), (packed, [1.0] * 32)):
        with pytest.raises(ValueError):
            tg.W8(64, 32, 1, p, s)
    w.K = 65
    with pytest.raises(ValueError):
        w._check()


def test_sizes_beyond_32_bits_are_refused():
    """... where what is left of them in 32 bits would be a size of its own."""
    n = ctypes.c_size_t()
    s = moe_struct()
    a = 1 << 20
    for name, args in (("tst_logprobs_workspace_bytes", (2 ** 32 + 5, 100, 3)), ("tst_logprobs_workspace_bytes", (5, 2 ** 32 + 100, 3)),
                       ("tst_logprobs_workspace_bytes", (5, 100, 2 ** 32 + 3)), ("tst_moe_workspace_bytes", (ctypes.byref(s), 2 ** 32 + 5, 2)),
                       ("tst_moe_workspace_bytes", (ctypes.byref(s), 5, 2 ** 32 + 2)), ("tst_w8_bytes", (2 ** 32 + 64, 16)), ("tst_w8_bytes", (64, -2 ** 32 + 16))):
        with pytest.raises(tg.TstgemmError) as e:
            operators._bytes(name, *args)
        assert e.value.code == EINVAL
    with pytest.raises(tg.TstgemmError):
        operators._call("tst_quantize", a, 0, 2 ** 32 + 64, a, 2 ** 32 + 64, a, 2 ** 32, 64, None)   # 0 rows are left
    operators._call("tst_quantize", a, 0, 2 ** 40, a, 2 ** 40, a, 0, 64, None)                       # strides have 64 bits


@pytest.mark.parametrize("argv", [["--tokens", "2001"], ["--tokens", "0"], ["--tokens", "-1"], ["--steps", "0"]])
def test_the_example_refuses_tokens_and_steps_that_are_not_there(argv, capsys):
    from paper_2510_06957_amd import decode_step
    with pytest.raises(SystemExit) as e:
        decode_step.main(argv)
    assert e.value.code == 2 and "--tokens" in capsys.readouterr().err
