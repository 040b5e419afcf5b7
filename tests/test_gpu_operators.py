"""GPU tests of the operators around the ternary product (include/tst_ops.h), through the binding, against their definitions in 64
bits on the CPU.  Tolerances are bounds of the rounding errors: u = 2^-24 for each fp32 operation, half a unit in the last place for
the result's type."""
import math

import numpy as np
import pytest
import torch

import paper_2510_06957_amd as tg
from w8_tiles import FAR, TILES

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LAST = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}   # relative half unit in the last place: 24, 8, 11 significant bits
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


def f64(t):
    return t.detach().cpu().double().numpy()


def assert_within(got, want, bound, dtype="f32", what=""):
    got = f64(got)
    bound = bound + LAST[dtype] * (np.abs(want) + bound) + TINY[dtype]
    assert got.shape == want.shape
    bad = ~(np.abs(got - want) <= bound)
    if bad.any():
        i = np.unravel_index(np.argmax(bad), bad.shape)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} outside; first at {i}: {got[i]!r}, want {want[i]!r} +- {bound[i]!r}")


def rng(*seed):
    return np.random.default_rng(list(seed))


# ---------------------------------------------------------------------------------------------------------------- 8 bits
def tokens(M, K, dtype, seed, columns=None):
    """[M, K] of a type on the GPU, a few channels large; a view with `columns` entries from row to row."""
    r = rng(seed, M, K)
    x = r.standard_normal((M, K)) * np.where(r.random(K) < 0.02, 20, 1)
    full = torch.full((M, columns or K), float("nan"), dtype=TYPES[dtype])
    full[:, :K] = torch.from_numpy(x).to(TYPES[dtype])
    return full.cuda()[:, :K]


def quantised(X):
    """The definition, with the roundings to 32 bits that it names."""
    x = X.detach().cpu().float().numpy()
    a = np.abs(x).max(1, keepdims=True)
    with np.errstate(all="ignore"):
        r = np.minimum(np.float32(127) / a, np.finfo(np.float32).max)
        q = np.rint(x * r)
    ok = np.isfinite(a)
    return np.where(ok, q, 0).astype(np.int8), np.where(ok, a / np.float32(127), np.float32("nan"))[:, 0]


@pytest.mark.parametrize("M,K", [(1, 1), (1, 4096), (3, 17), (5, 64), (7, 1000), (2, 16383), (33, 2053), (260, 512), (3, 40000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_quantize(M, K, dtype):
    for columns in (None, K + 3, (K + 7) // 8 * 8 + 8):
        X = tokens(M, K, dtype, 1, columns)
        Q, s = tg.tst_quantize(X)
        q, scale = quantised(X)
        assert Q.stride(0) % 64 == 0 or M == 1
        assert np.array_equal(Q.cpu().numpy(), q)
        assert np.array_equal(s.cpu().numpy(), scale)
    rows = torch.full((M, K + 5), 77, dtype=torch.int8, device="cuda")   # into rows of the caller's, which keep what lies beside
    tg.tst_quantize(X, rows[:, 2:K + 2])
    rows = rows.cpu().numpy()
    assert np.array_equal(rows[:, 2:K + 2], q) and (rows[:, :2] == 77).all() and (rows[:, K + 2:] == 77).all()


def test_quantize_of_rows_that_are_special():
    X = torch.zeros(9, 300)
    X[1] = 1e-42                                  # all subnormal
    X[2, 7] = -3.4028234e38
    X[3] = torch.linspace(-1, 1, 300)
    X[3, 5] = float("inf")
    X[4, 299] = float("nan")
    X[5] = torch.arange(300) % 255 / 2 - 63.5     # every code's border
    X[5, 0] = 127
    X[6, 0] = -0.0
    X[7, 123] = -float("inf")
    X[8] = torch.tensor([0x7f800001], dtype=torch.int32).view(torch.float32)   # a NaN whose upper half alone is infinity
    Q, s = tg.tst_quantize(X.cuda())
    q, scale = quantised(X)
    assert np.array_equal(Q.cpu().numpy(), q) and np.array_equal(s.cpu().numpy(), scale, equal_nan=True)
    assert np.isnan(scale[[3, 4, 7, 8]]).all() and scale[0] == 0 and not q[[0, 3, 4, 6, 7, 8]].any()


def layer(K, N, seed, kind="int8"):
    r = rng(seed, K, N)
    W = r.integers(-128, 128, (K, N)) if kind == "int8" else r.integers(-1, 2, (K, N))
    t = ((0.5 + r.random(N)) / 128).astype(np.float32)
    b = r.standard_normal(N).astype(np.float32)
    return W.astype(np.int8), t, b, tg.tst_w8_pack(torch.from_numpy(W.astype(np.int8)).cuda(), torch.from_numpy(t).cuda())


def product(q, s, W, t, b):
    """(the result, the bound of its fp32 roundings)"""
    acc = (q.astype(np.float64) @ W.astype(np.float64)) * s.astype(np.float64)[:, None] * t.astype(np.float64)
    y = acc if b is None else acc + b.astype(np.float64)
    return y, 4 * U * (np.abs(acc) + (0 if b is None else np.abs(b)))


SHAPES = [(1, 1, 1), (1, 64, 16), (1, 4096, 1000), (2, 65, 17), (5, 2053, 531), (16, 512, 64), (17, 300, 40), (31, 127, 129),
          (64, 1024, 256), (65, 130, 48), (130, 500, 260), (256, 768, 512), (257, 64, 255), (300, 2049, 515), (520, 1100, 700)]


@pytest.mark.parametrize("M,K,N", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_w8_gemm(M, K, N, dtype):
    W, t, b, w = layer(K, N, 2)
    r = rng(3, M, K)
    Q = torch.full((M, (K + 15) // 16 * 16 + 16), 99, dtype=torch.int8)   # what lies behind K does not matter
    Q[:, :K] = torch.from_numpy(r.integers(-128, 128, (M, K)).astype(np.int8))
    s = (r.random(M) / 100).astype(np.float32)
    Qd, sd = Q.cuda()[:, :K], torch.from_numpy(s).cuda()
    for bias in (None, b):
        Y = tg.tst_w8_gemm(Qd, sd, w, None if bias is None else torch.from_numpy(bias).cuda(), dtype=TYPES[dtype])
        assert Y.dtype == TYPES[dtype]
        assert_within(Y, *product(Q[:, :K].numpy(), s, W, t, bias), dtype, f"{M}x{K}x{N}")
    again = tg.tst_w8_gemm(Qd, sd, w, torch.from_numpy(b).cuda(), dtype=TYPES[dtype])
    assert torch.equal(again, Y)


@pytest.mark.parametrize("tile,M,K,N", [("%s-%d-%d" % tile, *s) for tile, shapes in TILES.items() for s in shapes])
def test_w8_gemm_on_every_tile(tile, M, K, N):
    W, t, b, w = layer(K, N, 63)
    q = rng(64, M, K).integers(-128, 128, (M, K)).astype(np.int8)
    Q = torch.full((M, (K + 15) // 16 * 16 + 16), -77, dtype=torch.int8)
    Q[:, :K] = torch.from_numpy(q)
    s = (rng(65, M).random(M) / 100).astype(np.float32)
    Qd, sd, bd = Q.cuda()[:, :K], torch.from_numpy(s).cuda(), torch.from_numpy(b).cuda()
    want, bound = product(q, s, W, t, b)
    for dtype in TYPES:
        Y = tg.tst_w8_gemm(Qd, sd, w, bd, dtype=TYPES[dtype])
        assert_within(Y, want, bound, dtype, f"{tile} {M}x{K}x{N}")
        assert torch.equal(tg.tst_w8_gemm(Qd, sd, w, bd, dtype=TYPES[dtype]), Y)
    odd = torch.empty(M * N + 1, device="cuda")[1:].view(M, N)   # off the border of wider stores
    tg.tst_w8_gemm(Qd, sd, w, Y=odd)
    assert_within(odd, *product(q, s, W, t, None), "f32", f"{tile} {M}x{K}x{N}")


@pytest.mark.parametrize("M,K,N", FAR.values())
def test_w8_gemm_of_rows_far_apart_on_every_tile(M, K, N):
    """Rows 4 MiB apart, the most there may be: offsets in a tile of 128 rows come to 2^29."""
    W, t, b, w = layer(K, N, 66)
    near = torch.zeros((M, (K + 15) // 16 * 16), dtype=torch.int8, device="cuda")
    near[:, :K] = torch.from_numpy(rng(67, M, K).integers(-128, 128, (M, K)).astype(np.int8))
    far = torch.empty((M, 1 << 22), dtype=torch.int8, device="cuda")
    far[:, :K] = near[:, :K]
    s = torch.ones(M, device="cuda")
    Y = tg.tst_w8_gemm(far[:, :K], s, w)
    assert torch.equal(Y, tg.tst_w8_gemm(near[:, :K], s, w))
    assert_within(Y, *product(near[:, :K].cpu().numpy(), s.cpu().numpy(), W, t, None))


@pytest.mark.parametrize("M,K,N", [(1, 131071, 3), (20, 131071, 5), (70, 131071, 33), (300, 131071, 260)])
def test_w8_gemm_sums_do_not_overflow(M, K, N):
    """The largest sum there is, 131071 * 128 * 128 = 2^31 - 16384, and the lowest."""
    W = torch.full((K, N), -128, dtype=torch.int8)
    W[:, 0] = 127
    one = torch.ones(max(M, N), device="cuda")
    w = tg.tst_w8_pack(W.cuda(), one[:N].contiguous())
    Q = torch.full((M, 131072), -128, dtype=torch.int8, device="cuda")[:, :K]
    Y = tg.tst_w8_gemm(Q, one[:M].contiguous(), w).cpu().numpy()
    want = np.full((M, N), np.float32(K * 16384))
    want[:, 0] = np.float32(-K * 128 * 127)
    assert np.array_equal(Y, want)


@pytest.mark.parametrize("M,K,N", [(1, 515, 259), (40, 512, 96), (100, 700, 130), (300, 640, 512)])
def test_w8_gemm_with_a_ternary_matrix_is_the_ternary_product(M, K, N):
    r = rng(4, M, K, N)
    W = r.integers(-1, 2, (K, N)).astype(np.int8)
    q = r.integers(-127, 128, (M, K)).astype(np.int8)
    Q = torch.zeros((M, (K + 63) // 64 * 64), dtype=torch.int8)
    Q[:, :K] = torch.from_numpy(q)
    one = torch.ones(max(M, N), device="cuda")
    t = tg.tcsc_upload(tg.tcsc_build(W))
    w = tg.tst_w8_pack(torch.from_numpy(tg.tcsc_to_dense(t)).cuda(), one[:N].contiguous())
    b = torch.from_numpy(r.integers(-50, 50, N).astype(np.float32)).cuda()
    assert torch.equal(tg.tst_w8_gemm(Q.cuda()[:, :K], one[:M].contiguous(), w, b),
                       tg.tstgemm(torch.from_numpy(q.astype(np.float32)).cuda(), t, b))


@pytest.mark.parametrize("M,K,N", [(1, 100, 33), (1, 8192, 520), (3, 4096, 64), (8, 1531, 129), (40, 1000, 65), (129, 300, 130), (513, 1024, 256)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_w8_linear_is_quantize_and_gemm(M, K, N, dtype):
    W, t, b, w = layer(K, N, 5)
    X = tokens(M, K, dtype, 6, K + 8)
    bd = torch.from_numpy(b).cuda()
    Y = tg.tst_w8_linear(X, w, bd)
    q, s = quantised(X)
    assert_within(Y, *product(q, s, W, t, b), dtype)
    assert torch.equal(Y, tg.tst_w8_gemm(*tg.tst_quantize(X), w, bd, dtype=TYPES[dtype]))
    odd = tokens(M, K, dtype, 6, K + 1)   # rows off every border
    assert torch.equal(Y, tg.tst_w8_linear(odd, w, bd))


@pytest.mark.parametrize("M", [1, 9, 64, 300])
def test_w8_linear_keeps_what_is_not_finite_to_its_row(M):
    W, t, b, w = layer(200, 70, 7)
    X = tokens(M, 200, "bf16", 8)
    clean = tg.tst_w8_linear(X, w)
    bad = [0] if M == 1 else [2, M - 1]
    for i, v in zip(bad, (float("nan"), -float("inf"))):
        X[i, 199] = v
    X[0 if M == 1 else 1] = X[0 if M == 1 else 1] * 1
    Y = tg.tst_w8_linear(X, w)
    for m in range(M):
        assert torch.isnan(Y[m]).all() if m in bad else torch.equal(Y[m], clean[m])


# ------------------------------------------------------------------------------------------------------------------- moe
def experts(E, D, F, dtype, seed, router=None):
    r = rng(seed, E, D, F)
    w = dict(router=torch.from_numpy(r.standard_normal((E, D)) / math.sqrt(D) if router is None else router).to(TYPES[dtype]))
    for name, rows, cols in (("gate", D, F), ("up", D, F), ("down", F, D)):
        w[name] = torch.from_numpy(np.clip(np.rint(r.standard_normal((E, rows, cols)) * 40), -128, 127).astype(np.int8))
        w[name + "_scale"] = torch.from_numpy(((0.5 + r.random((E, cols))) / (40 * math.sqrt(rows))).astype(np.float32))
    return w


def packed(w):
    return tg.tst_moe_pack(*(w[n].cuda() for n in ("router", "gate", "gate_scale", "up", "up_scale", "down", "down_scale")))


def moe_logits(X, w):
    """(logits, the bound of their roundings for each token)"""
    x, r = f64(X), f64(w["router"])
    return x @ r.T, (x.shape[1] + 1) * U * (np.abs(x) @ np.abs(r).T).max(1)


def clear_choice(X, w, k):
    """Whether the logits that decide lie farther apart than their roundings reach."""
    logits, d_logit = moe_logits(X, w)
    order = -np.sort(-logits, axis=1)
    return logits.shape[1] == 1 or ((order[:, :-1] - order[:, 1:])[:, :k].min(1) > 2 * d_logit).all()


def moe_reference(X, w, k, normalize, dtype):
    """(Y, ids, p, bound of Y, bound of p)"""
    x, r = f64(X), f64(w["router"])
    T, D = x.shape
    logits, d_logit = moe_logits(X, w)
    ids = np.argsort(-logits, axis=1, kind="stable")[:, :k]
    e = np.exp(logits - logits.max(1, keepdims=True))
    p = np.take_along_axis(e, ids, 1)
    p = p / (p if normalize else e).sum(1, keepdims=True)
    d_p = p * (4 * d_logit[:, None] + (r.shape[0] + 30) * U)
    Y, bound = np.zeros_like(x), np.zeros_like(x)
    F = w["gate"].shape[2]
    keep = 2.0 ** -24 if dtype == "f32" else 2.0 ** -16
    for t in range(T):
        for j in range(k):
            i = ids[t, j]
            W = {n: f64(w[n][i]) for n in ("gate", "up", "down")}
            S = {n: f64(w[n + "_scale"][i]) for n in ("gate", "up", "down")}
            g, u = (x[t] @ W["gate"]) * S["gate"], (x[t] @ W["up"]) * S["up"]
            dg = (3 * D + 2) * U * (np.abs(x[t]) @ np.abs(W["gate"])) * S["gate"]
            du = (3 * D + 2) * U * (np.abs(x[t]) @ np.abs(W["up"])) * S["up"]
            silu = g / (1 + np.exp(-g))
            h = silu * u
            dh = 1.1 * dg * np.abs(u) + np.abs(silu) * du + 1.1 * dg * du + (12 * U + keep) * np.abs(h)
            Y[t] += p[t, j] * S["down"] * (h @ W["down"])
            bound[t] += S["down"] * ((p[t, j] * dh + d_p[t, j] * np.abs(h)) @ np.abs(W["down"]))
            bound[t] += p[t, j] * S["down"] * (3 * F + k + 10) * U * (np.abs(h) @ np.abs(W["down"]))
    return Y, ids, p, bound, d_p


MOE = [(1, 1, 1, 1, 1), (1, 2, 1, 64, 64), (1, 8, 2, 256, 512), (2, 5, 5, 70, 33), (5, 12, 3, 153, 129), (16, 16, 4, 128, 64),
       (17, 7, 2, 200, 100), (33, 70, 6, 96, 48), (64, 4, 1, 64, 130), (70, 130, 8, 65, 31), (3, 512, 16, 40, 20), (60, 512, 2, 33, 17), (2, 3, 2, 17000, 16), (1, 4, 2, 64, 5000)]


@pytest.mark.parametrize("T,E,k,D,F", MOE)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_moe(T, E, k, D, F, dtype):
    w = experts(E, D, F, dtype, 11)
    moe = packed(w)
    for seed in range(12, 112):   # tokens whose choice rounding cannot change
        X = tokens(T, D, dtype, seed, D + 5)
        if clear_choice(X, w, k):
            break
    for normalize in (True, False):
        assert clear_choice(X, w, k)
        want, ids, p, bound, d_p = moe_reference(X, w, k, normalize, dtype)
        Y, got_ids, got_p = tg.tst_moe(X, moe, k, normalize=normalize)
        assert Y.dtype == TYPES[dtype] and np.array_equal(got_ids.cpu().numpy(), ids)
        assert_within(got_p, p, d_p, what="p")
        assert_within(Y, want, bound, dtype, "Y")
    again = tg.tst_moe(X, moe, k, normalize=False)
    assert torch.equal(again[0], Y) and torch.equal(again[2], got_p)


@pytest.mark.parametrize("T,E,k,D,F,most", [(64, 1, 1, 70, 50, 64), (64, 4, 4, 530, 90, 64), (50, 4, 3, 130, 333, 33), (40, 2, 1, 65, 700, 17),
                                            (101, 3, 3, 100, 40, 64), (60, 9, 6, 201, 150, 33)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_moe_of_experts_with_many_members(T, E, k, D, F, most, dtype):
    """Experts whose tokens fill all four tiles of 16, some of them in part; `most`: members that some expert has at least in 64 tokens."""
    w = experts(E, D, F, dtype, 61)
    for seed in range(62, 162):
        X = tokens(T, D, dtype, seed, D + 5)
        if clear_choice(X, w, k):
            break
    assert clear_choice(X, w, k)
    want, ids, p, bound, d_p = moe_reference(X, w, k, True, dtype)
    assert np.bincount(ids[:64].ravel()).max() >= most
    moe = packed(w)
    Y, got_ids, got_p = tg.tst_moe(X, moe, k)
    assert np.array_equal(got_ids.cpu().numpy(), ids)
    assert_within(got_p, p, d_p, what="p")
    assert_within(Y, want, bound, dtype, "Y")
    assert torch.equal(tg.tst_moe(X, moe, k)[0], Y)


@pytest.mark.parametrize("T", [5, 20, 60])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_moe_keeps_the_bits_of_h(T, dtype):
    """Columns of the result that are the difference of two entries of h some 2^-13 apart.  Each token has one entry that is not zero, so that
    sums round only where they have to: g and u by 4 units (planes, scale), silu of a positive g turns them into at most 1.3 of that and adds 4 for
    the exponential, the sum and the division, the products with u, its error and p 6, the cut to 24 bits 1; the second product has six terms."""
    r = rng(74, T)
    D, F = 16, 32
    x = np.zeros((T, D))
    x[:, 0] = 1 + r.random(T)
    X = torch.from_numpy(x).to(TYPES[dtype]).cuda()
    w = dict(router=torch.ones((1, D), dtype=TYPES[dtype]), gate=torch.from_numpy(r.integers(-128, 128, (1, D, F)).astype(np.int8)),
             up=torch.from_numpy(r.integers(-128, 128, (1, D, F)).astype(np.int8)), down=torch.zeros((1, F, D), dtype=torch.int8), gate_scale=torch.full((1, F), 0.03), up_scale=torch.from_numpy((0.01 + 0.01 * r.random((1, F))).astype(np.float32)),
             down_scale=torch.from_numpy((0.5 + r.random((1, D))).astype(np.float32)))
    for c in range(D):
        w["gate"][0, 0, 2 * c] = w["gate"][0, 0, 2 * c + 1] = int(r.integers(20, 100))
        w["up"][0, 0, 2 * c] = w["up"][0, 0, 2 * c + 1] = int(r.integers(20, 128))
        w["up_scale"][0, 2 * c + 1] = w["up_scale"][0, 2 * c] * (1 - 2.0 ** -13 * (1 + r.random()))
        w["down"][0, 2 * c, c], w["down"][0, 2 * c + 1, c] = 64, -64
    g = (f64(X) @ f64(w["gate"][0])) * f64(w["gate_scale"][0])
    h = g / (1 + np.exp(-g)) * (f64(X) @ f64(w["up"][0])) * f64(w["up_scale"][0])
    want = (h @ f64(w["down"][0])) * f64(w["down_scale"][0])
    bound = (4 * 1.3 + 4 + 4 + 6 + 1 + 6 + 2) * U * (h @ np.abs(f64(w["down"][0]))) * f64(w["down_scale"][0])
    assert (bound < 0.05 * np.abs(want)).all()
    Y, ids, p = tg.tst_moe(X, packed(w), 1)
    assert (p == 1).all()
    assert_within(Y, want, bound, dtype, "Y")


def test_moe_ties_go_to_the_lowest_expert():
    r = rng(13)
    rows = r.standard_normal((3, 80))
    w = experts(9, 80, 48, "f32", 14, router=rows[[0, 1, 1, 0, 2, 1, 0, 2, 2]])
    X = tokens(6, 80, "f32", 15)
    _, ids, _ = tg.tst_moe(X, packed(w), 7)
    logits = f64(X) @ f64(w["router"]).T
    assert np.array_equal(ids.cpu().numpy(), np.argsort(-logits, axis=1, kind="stable")[:, :7])
    w = experts(80, 80, 16, "bf16", 16, router=np.zeros((80, 80)))   # no preference at all
    Y, ids, p = tg.tst_moe(tokens(2, 80, "bf16", 17), packed(w), 4)
    assert np.array_equal(ids.cpu().numpy(), [[0, 1, 2, 3]] * 2) and (p == 0.25).all() and torch.isfinite(Y).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [3, 20])
def test_moe_keeps_what_is_not_finite_to_its_token(T, dtype):
    w = experts(6, 96, 80, dtype, 18)
    moe, X = packed(w), tokens(T, 96, dtype, 19)
    clean = tg.tst_moe(X, moe, 2)
    X[1, 5] = float("nan")
    X[T - 1, 0] = float("inf")
    Y, ids, p = tg.tst_moe(X, moe, 2)
    assert ((ids >= 0) & (ids < 6)).all()
    for t in range(T):
        if t in (1, T - 1):
            assert torch.isnan(Y[t]).all() and torch.isnan(p[t]).all()
        else:
            assert torch.equal(ids[t], clean[1][t]) and torch.equal(p[t], clean[2][t])
            assert_within(Y[t], f64(clean[0][t]), np.abs(f64(clean[0][t])) * 2.0 ** -8 + 1e-5, dtype)


# -------------------------------------------------------------------------------------------------------------- logprobs
def logits(R, V, dtype, seed, columns=None):
    z = torch.full((R, columns or V), float("nan"), dtype=TYPES[dtype])
    z[:, :V] = torch.from_numpy(rng(seed, R, V).standard_normal((R, V)) * 4).to(TYPES[dtype])
    return z.cuda()[:, :V]


def check_logprobs(Z, token, top, rows=slice(None)):
    """rows: those looked at"""
    out = tg.tst_logprobs(Z, None if token is None else token.cuda(), top=top)
    of_token, entropy, ids, of_top = (o[rows] for o in out)
    token = None if token is None else token[rows]
    z = f64(Z[rows])
    R, V = z.shape
    with np.errstate(all="ignore"):
        d = z - z.max(1, keepdims=True)
        e = np.exp(d)
        log_sum = np.log(e.sum(1, keepdims=True))
        lp = d - log_sum
        spread = np.where(e > 0, e * -d, 0).sum(1) / e.sum(1)
    d_sum = (V / 256 + 40) * U
    assert_within(entropy, log_sum[:, 0] + spread, d_sum * (2 + log_sum[:, 0] + 3 * spread), what="entropy")
    order = np.argsort(-z, axis=1, kind="stable")[:, :top]
    assert np.array_equal(ids.cpu().numpy(), order)

    def close(got, want, what):
        low = want < -1e30
        assert (f64(got)[low] < -1e30).all()
        want = np.where(low, 0, want)
        assert_within(torch.where(torch.from_numpy(low), 0.0, got.cpu()), want, d_sum + 3 * U * (np.abs(want) + log_sum), what=what)

    close(of_top, np.take_along_axis(lp, order, 1), "of_top")
    if token is not None:
        t = token.numpy().reshape(R, -1)
        assert of_token.shape == token.shape
        close(of_token.reshape(R, -1), np.take_along_axis(lp, t.astype(np.int64), 1), "of_token")


LOGITS = [(1, 1, 1), (1, 2, 2), (3, 63, 5), (2, 64, 64), (2, 1000, 20), (5, 1023, 1), (1, 8193, 3), (7, 32003, 5), (1, 50001, 20),
          (1, 262144, 64), (70, 4099, 7), (300, 1500, 0), (520, 2048, 4)]


@pytest.mark.parametrize("R,V,top", LOGITS)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_logprobs(R, V, top, dtype):
    r = rng(21, R, V)
    check_logprobs(logits(R, V, dtype, 22), torch.from_numpy(r.integers(0, V, R)), top)
    for columns in (V + 1, (V + 15) // 8 * 8):
        check_logprobs(logits(R, V, dtype, 23, columns), torch.from_numpy(r.integers(0, V, (R, 3)).astype(np.int32)), top)
    check_logprobs(logits(R, V, dtype, 24), None, top)


@pytest.mark.parametrize("V", [40, 1000, 9001, 140000])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_logprobs_of_masked_rows_and_ties(V, dtype):
    low = torch.finfo(TYPES[dtype]).min
    Z = logits(8, V, dtype, 25)
    Z[0, 5:] = -float("inf")                 # fewer left than alternatives asked for
    Z[1, :V - 3] = low                       # masked with the type's lowest value
    Z[2] = 0.0                               # all alike
    Z[3] = low                               # all alike, all masked
    Z[4, 1:] = -float("inf")                 # one left: entropy 0
    Z[5] = torch.where(torch.arange(V, device="cuda") % 7 == 3, 50.0, -50.0).to(TYPES[dtype])
    Z[6, ::2] = 0.0
    Z[6, 1::2] = -0.0
    Z[7] = Z[7].abs() + 60000                # far from zero (and infinite differences nowhere)
    Z[7] = Z[7].clamp(max=65000)
    check_logprobs(Z, torch.tensor([1, V - 1, 3, 4, 0, 3, 1, 2]), 9)


@pytest.mark.parametrize("R", [10, 1030])   # rows in splits, and whole ones
@pytest.mark.parametrize("V,top", [(5000, 1), (40007, 20), (70000, 64)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logprobs_of_rows_in_many_chunks(R, V, top, dtype):
    """What a list of candidates can make of a row: values that rise, fall, tie everywhere, in runs, at the bound, only at the end."""
    Z = torch.zeros((R, V), dtype=TYPES[dtype], device="cuda")
    n = torch.arange(V, device="cuda")
    Z[:10] = logits(10, V, dtype, 28)
    Z[0] = (n / V * 20 - 10).to(TYPES[dtype])
    Z[1] = (10 - n / V * 20).to(TYPES[dtype])
    Z[2] = (n % 5).to(TYPES[dtype])
    Z[3] = (n // (V // 7)).to(TYPES[dtype])
    Z[4, :V - top - 3] = -float("inf")
    Z[5, : V // 2] = torch.finfo(TYPES[dtype]).min
    Z[6] = Z[6].round()
    Z[7, 16384:16384 + 300 if V > 17000 else V] = 30.0
    Z[8, ::64] = 25.0
    Z[9, V - 1] = 60.0
    check_logprobs(Z, torch.arange(R) % V, top, slice(0, 10))


@pytest.mark.parametrize("V", [33, 2000, 70001])
def test_logprobs_of_rows_without_a_distribution(V):
    Z = logits(6, V, "f32", 26)
    clean = tg.tst_logprobs(Z, top=4)
    Z[0] = -float("inf")
    Z[1, V - 1] = float("nan")
    Z[2, 3] = float("inf")
    Z[3, 11] = torch.tensor([-1], dtype=torch.int32).view(torch.float32).item()   # a NaN with its sign bit set
    Z[4, 2] = -float("nan")
    of_token, entropy, ids, of_top = tg.tst_logprobs(Z, torch.zeros(6, dtype=torch.int64, device="cuda"), top=4)
    for r in range(5):
        assert torch.isnan(entropy[r]) and torch.isnan(of_token[r]) and torch.isnan(of_top[r]).all()
    assert ids[0].tolist() == [0, 1, 2, 3] and ids[1, 0] == V - 1 and ids[2, 0] == 3 and ids[3, 0] == 11 and ids[4, 0] == 2
    assert torch.equal(ids[5], clean[2][5]) and torch.equal(entropy[5], clean[1][5]) and torch.equal(of_top[5], clean[3][5])


@pytest.mark.parametrize("R", [7, 1100])   # rows in splits where they are long, and whole ones
@pytest.mark.parametrize("V", [1, 2, 5, 33, 64, 3000, 70001])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_logprobs_alternatives_of_rows_with_nan(V, R, dtype):
    """A NaN counts as largest wherever it stands, ties go to the lowest token, and a row has as many alternatives as are asked for: all
    of them where top is V."""
    Z = torch.zeros((R, V), dtype=TYPES[dtype], device="cuda")
    Z[:7] = logits(7, V, dtype, 29)
    Z[0, 0] = float("nan")
    Z[1] = float("nan")
    Z[2, 0] = Z[2, V // 2] = Z[2, V - 1] = float("nan")
    Z[3, ::2] = float("nan")
    Z[4, 0], Z[4, V - 1] = float("nan"), float("inf")
    Z[5] = -float("inf")
    Z[5, 0] = float("nan")
    Z[6, V // 2] = -float("nan")
    z = f64(Z[:7])
    order = np.lexsort((np.broadcast_to(np.arange(V), z.shape), -np.nan_to_num(z, nan=0.0), ~np.isnan(z)))
    for top in {1, min(V, 5), min(V, 64)}:
        of_token, entropy, ids, of_top = (o[:7].cpu() for o in tg.tst_logprobs(Z, torch.zeros(R, dtype=torch.int64, device="cuda"), top=top))
        assert np.array_equal(ids.numpy(), order[:, :top])
        assert torch.isnan(of_token).all() and torch.isnan(entropy).all() and torch.isnan(of_top).all()


@pytest.mark.parametrize("low", [-1e4, -3e4, -1e9])
@pytest.mark.parametrize("R", [9, 1030])
@pytest.mark.parametrize("V,top", [(700, 20), (40007, 20), (70000, 64)])
def test_logprobs_of_rows_masked_with_finite_values(V, top, R, low):
    """Masks that are neither infinite nor the type's lowest value: entries like any other, that tie."""
    for dtype in ("f32", "bf16", "f16")[:2 if low == -1e9 else 3]:
        Z = torch.zeros((R, V), dtype=TYPES[dtype], device="cuda")
        Z[:9] = logits(9, V, dtype, 73)
        n = torch.arange(V, device="cuda")
        keep = [n % 1000 == 7, n < 3, n >= V - 2, n == V // 2, n % 64 == 0, n < 0, n % 2 == 0, (n > V // 3) & (n < V // 3 + 30), n >= 0]
        for r, k in enumerate(keep):
            Z[r, ~k] = low
        check_logprobs(Z, torch.arange(R) % V, top, slice(0, 9))


def test_logprobs_of_tokens_outside_the_vocabulary():
    Z = logits(3, 500, "bf16", 27)
    t = torch.tensor([[-1, 4], [500, 499], [2 ** 40, -2 ** 40]], device="cuda")
    got = tg.tst_logprobs(Z, t)[0]
    assert torch.isnan(got).tolist() == [[True, False], [True, False], [True, True]]


# ------------------------------------------------------------------------------------------------- streams, graphs, nothing
def cases():
    W, t, b, w = layer(700, 300, 31)
    moe = packed(experts(9, 128, 96, "bf16", 32))
    small, many, x, z = (tokens(3, 700, "bf16", 33), tokens(200, 700, "bf16", 34), tokens(5, 128, "bf16", 35), logits(3, 40000, "f32", 36))
    token = torch.tensor([5, 39999, 7], device="cuda")
    return [("linear, few", lambda **o: tg.tst_w8_linear(small, w, **o)), ("linear, many", lambda **o: tg.tst_w8_linear(many, w, **o)),
            ("moe", lambda **o: tg.tst_moe(x, moe, 3, **o)), ("logprobs", lambda **o: tg.tst_logprobs(z, token, top=6, **o))]


def as_list(out):
    return list(out) if isinstance(out, tuple) else [out]


def test_calls_on_another_stream():
    side = torch.cuda.Stream()
    for name, call in cases():
        want = as_list(call())
        torch.cuda.synchronize()
        got = [as_list(call(stream=side)) for _ in range(4)]   # results and workspaces of calls that follow one another
        side.synchronize()
        for g in got:
            assert all(torch.equal(a, b) for a, b in zip(g, want)), name


def test_calls_in_a_graph():
    for name, call in cases():
        want = [o.clone() for o in as_list(call())]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = as_list(call())
        for _ in range(3):
            for o in out:
                o.zero_()
            graph.replay()
            call()                      # eager work of the same kind between the replays
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)), name


def test_no_tokens():
    W, t, b, w = layer(70, 30, 37)
    moe = packed(experts(4, 128, 32, "bf16", 38))
    e = torch.empty
    Q, s = tg.tst_quantize(e((0, 70), device="cuda"))
    assert Q.shape == (0, 70) and s.shape == (0,)
    assert tg.tst_w8_linear(e((0, 70), device="cuda"), w).shape == (0, 30)
    assert tg.tst_w8_gemm(e((0, 70), dtype=torch.int8, device="cuda"), s, w).shape == (0, 30)
    Y, ids, p = tg.tst_moe(e((0, 128), dtype=torch.bfloat16, device="cuda"), moe, 2)
    assert Y.shape == (0, 128) and ids.shape == p.shape == (0, 2)
    out = tg.tst_logprobs(e((0, 50), device="cuda"), e((0, 2), dtype=torch.int64, device="cuda"), top=3)
    assert [tuple(o.shape) for o in out] == [(0, 2), (0,), (0, 3), (0, 3)]
    torch.cuda.synchronize()


def test_plain_calls_go_through_the_native_half():
    """... and give what the long way gives, which takes over whatever is not plain."""
    from paper_2510_06957_amd import operators
    W, t, b, w = layer(700, 300, 51)
    bd, X = torch.from_numpy(b).cuda(), tokens(6, 700, "f16", 52, 720)
    Q, s = tg.tst_quantize(X)
    moe, x = packed(experts(9, 128, 96, "bf16", 53)), tokens(5, 128, "bf16", 54, 131)
    z, token = logits(4, 3000, "f32", 55, 3004), torch.tensor([[5, 2999], [7, 1], [0, 0], [2, -1]], dtype=torch.int32, device="cuda")
    native = operators._native
    assert native is not None
    here = torch.cuda.current_stream()
    for fast, slow in ((native.w8_linear(X, w, bd), tg.tst_w8_linear(X, w, bd, stream=here)), (native.w8_linear(X, w, None), tg.tst_w8_linear(X, w, stream=here)),
                       (native.w8_gemm(Q, s, w, bd, torch.bfloat16), tg.tst_w8_gemm(Q, s, w, bd, dtype=torch.bfloat16, stream=here)),
                       (native.w8_gemm(Q, s, w, None, None), tg.tst_w8_gemm(Q, s, w, stream=here)),
                       (native.moe(x, moe, 3, True), tg.tst_moe(x, moe, 3, stream=here)), (native.moe(x, moe, 9, False), tg.tst_moe(x, moe, 9, False, stream=here)),
                       (native.logprobs(z, token, 7), tg.tst_logprobs(z, token, 7, stream=here)), (native.logprobs(z, None, 0), tg.tst_logprobs(z, stream=here)),
                       (native.logprobs(z, token[:, 0].contiguous().long(), 1), tg.tst_logprobs(z, token[:, 0].contiguous().long(), 1, stream=here))):
        assert fast is not None
        for a, c in zip(as_list(fast), as_list(slow)):
            assert a.dtype == c.dtype and a.shape == c.shape and torch.equal(torch.nan_to_num(a.float(), 77), torch.nan_to_num(c.float(), 77))
    for none in (native.w8_linear(X.double(), w, bd), native.w8_linear(X.t(), w, bd), native.w8_linear(X[:, :600], w, bd), native.w8_linear(X, moe, bd),
                 native.w8_linear(X, w, s), native.w8_linear(X.cpu(), w, bd), native.w8_linear(None, w, bd), native.w8_gemm(Q, s, w, bd, torch.int8),
                 native.w8_gemm(Q, s[:3], w, bd, None), native.w8_gemm(Q, s, w, bd, "f32"), native.w8_gemm(X, s, w, bd, None),
                 native.w8_gemm(Q.contiguous(), s, w, bd, None), native.moe(x.float(), moe, 3, True), native.moe(x, w, 3, True), native.moe(x, moe, 10, True),
                 native.moe(x, moe, 3.0, True), native.moe(x, moe, 3, 1), native.logprobs(z, token.float(), 7), native.logprobs(z, token[:3], 7),
                 native.logprobs(z, token, 65), native.logprobs(z, token.t(), 7), native.logprobs(z[0], None, 1)):
        assert none is None
    with pytest.raises(TypeError):
        native.moe(x, moe)
    with torch.utils._python_dispatch.TorchDispatchMode():
        assert native.w8_linear(X, w, bd) is None


def test_more_rows_than_a_launch_takes():
    """2^24 workgroups of 256 have more threads than a grid counts."""
    M = (1 << 24) + 3
    r = torch.Generator(device="cuda").manual_seed(60)
    x = torch.randn((M, 2), generator=r, device="cuda")
    Q, s = tg.tst_quantize(x)
    token = torch.randint(0, 2, (M,), generator=r, device="cuda")
    of_token, entropy, ids, of_top = tg.tst_logprobs(x, token, top=2)
    lp = x.double().log_softmax(1)
    assert torch.equal(s, x.abs().amax(1) / torch.full_like(s, 127))
    assert torch.equal(Q.abs().amax(1), torch.full((M,), 127, dtype=torch.int8, device="cuda"))
    assert ((Q.float() * s[:, None] - x).abs() <= 0.501 * s[:, None]).all()
    assert torch.equal(ids, torch.sort(x, dim=1, descending=True, stable=True).indices.int())
    for got, want in ((of_token, lp.gather(1, token[:, None])[:, 0]), (entropy, -(lp.exp() * lp).sum(1)), (of_top, lp.gather(1, ids.long()))):
        assert ((got - want).abs() <= 50 * U * (1 + want.abs())).all()


def test_weights_are_those_of_the_pack():
    """Objects that have the names of a W8 or a Moe, or whose sizes have been changed, are refused: the kernels read as much as K and N say."""
    import types

    from paper_2510_06957_amd import operators
    W, t, b, w = layer(128, 64, 68)
    X = tokens(3, 128, "bf16", 69)
    Q, s = tg.tst_quantize(X)
    native, moe, x = operators._native, packed(experts(4, 64, 32, "bf16", 70)), tokens(2, 64, "bf16", 71)
    same = types.SimpleNamespace(K=128, N=64, count=1, packed=w.packed, scale=w.scale)
    like = types.SimpleNamespace(_raw=moe._raw, device_index=moe.device_index, D=64, dtype=moe.dtype)
    assert native.w8_linear(X, same, None) is None and native.w8_gemm(Q, s, same, None, None) is None and native.moe(x, like, 2, True) is None
    for call in (lambda: tg.tst_w8_linear(X, same), lambda: tg.tst_w8_gemm(Q, s, same), lambda: tg.tst_moe(x, like, 2)):
        with pytest.raises(ValueError):
            call()
    want = tg.tst_w8_linear(X, w)
    for name, value in (("N", 32), ("K", 64), ("packed", w.packed[:4096]), ("scale", w.scale[:32]), ("scale", w.scale.cpu()), ("packed", w.packed.cpu())):
        kept = getattr(w, name)
        setattr(w, name, value)
        assert native.w8_linear(X, w, None) is None and native.w8_gemm(Q, s, w, None, None) is None
        for call in (lambda: tg.tst_w8_linear(X, w), lambda: tg.tst_w8_gemm(Q, s, w)):
            with pytest.raises(ValueError):
                call()
        setattr(w, name, kept)
    assert torch.equal(tg.tst_w8_linear(X, w), want)


def test_views_that_negate_are_refused():
    """The imaginary part of a conjugate is a view of memory that holds the values negated."""
    from paper_2510_06957_amd import operators
    W, t, b, w = layer(1, 5, 72)
    z = torch.randn((6, 1), dtype=torch.complex64, device="cuda")
    x = z.conj().imag
    assert x.is_neg()
    bias = torch.randn(5, device="cuda")
    for call in (lambda: tg.tst_quantize(x), lambda: tg.tst_w8_linear(x, w), lambda: tg.tst_logprobs(x),
                 lambda: tg.tst_w8_linear(x.resolve_neg(), w, torch._neg_view(bias))):
        with pytest.raises(ValueError):
            call()
    assert operators._native.w8_linear(x, w, None) is None and operators._native.logprobs(x, None, 1) is None
    assert torch.equal(tg.tst_w8_linear(x.resolve_neg(), w), tg.tst_w8_linear(-z.imag.contiguous(), w))


def test_large_strides():
    """Rows far apart, up to what the product takes; and offsets that pass 32 bits."""
    W, t, b, w = layer(96, 40, 56)
    far = torch.empty(700 * (1 << 22), dtype=torch.int8, device="cuda")          # 2.9 GB
    rows = far.view(700, 1 << 22)[:, :96]
    Q = torch.from_numpy(rng(57).integers(-128, 128, (700, 96)).astype(np.int8)).cuda()
    s = torch.ones(700, device="cuda")
    rows.copy_(Q)
    near = torch.zeros((700, 96), dtype=torch.int8, device="cuda").copy_(Q)
    for M in (1, 5, 40, 200, 700):
        assert torch.equal(tg.tst_w8_gemm(rows[:M], s[:M], w), tg.tst_w8_gemm(near[:M], s[:M], w))
    with pytest.raises(tg.TstgemmError):
        tg.tst_w8_gemm(far[:(1 << 23) + 32].view(2, (1 << 22) + 16)[:, :96], s[:2], w)
    x = far.view(torch.bfloat16).view(700, 1 << 21)[:, :96]
    x.copy_(Q.bfloat16())
    y = near.bfloat16()
    assert torch.equal(tg.tst_w8_linear(x, w), tg.tst_w8_linear(y, w))
    assert all(torch.equal(a, c) for a, c in zip(tg.tst_logprobs(x, top=3), tg.tst_logprobs(y, top=3)))
    moe = packed(experts(5, 96, 32, "bf16", 58))
    assert all(torch.equal(a, c) for a, c in zip(tg.tst_moe(x[632:], moe, 2), tg.tst_moe(y[632:], moe, 2)))


def test_given_results_and_workspaces():
    W, t, b, w = layer(300, 65, 39)
    X = tokens(4, 300, "f16", 40)
    Y = torch.empty((4, 65), dtype=torch.float16, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    assert tg.tst_w8_linear(X, w, Y=Y, workspace=ws) is Y
    assert torch.equal(Y, tg.tst_w8_linear(X, w))
    odd = torch.empty(4 * 65 + 1, dtype=torch.float16, device="cuda")[1:].view(4, 65)   # off the border of wider stores
    assert torch.equal(tg.tst_w8_gemm(*tg.tst_quantize(X), w, Y=odd), Y)
    with pytest.raises(tg.TstgemmError) as e:
        tg.tst_w8_linear(X, w, workspace=ws[:256])
    assert e.value.code == -8
    with pytest.raises(tg.TstgemmError) as e:
        tg.tst_w8_linear(X, w, workspace=ws[1:])
    assert e.value.code == -1


def test_refusals_on_the_gpu():
    W, t, b, w = layer(64, 32, 41)
    X = tokens(2, 64, "f32", 42)
    Q, s = tg.tst_quantize(X)
    off = torch.zeros((2, 80), dtype=torch.int8, device="cuda")
    moe = packed(experts(4, 64, 32, "bf16", 43))
    x = tokens(2, 64, "bf16", 44)
    for call in (lambda: tg.tst_w8_linear(X.double(), w), lambda: tg.tst_w8_linear(X[:, :60], w), lambda: tg.tst_w8_linear(X.t(), w),
                 lambda: tg.tst_w8_linear(X[:1].expand(2, 64), w), lambda: tg.tst_w8_linear(X, w, b=s),
                 lambda: tg.tst_w8_linear(X, w, Y=torch.empty((2, 32), dtype=torch.float16, device="cuda")),
                 lambda: tg.tst_w8_gemm(off[:, 1:65], s, w), lambda: tg.tst_w8_gemm(off.view(-1)[:2 * 72].view(2, 72)[:, :64], s, w),
                 lambda: tg.tst_w8_gemm(Q, s[:1], w), lambda: tg.tst_w8_gemm(Q.float(), s, w), lambda: tg.tst_w8_gemm(Q, s, w, dtype=torch.int32),
                 lambda: tg.tst_w8_pack(torch.zeros((4, 4), device="cuda"), s), lambda: tg.tst_quantize(X, Q[:1]),
                 lambda: tg.tst_w8_pack(np.zeros((4, 4), np.int8), s), lambda: tg.tst_w8_linear(X, moe), lambda: tg.tst_quantize(X, Q.cpu().numpy()),
                 lambda: tg.tst_w8_linear(X, w, workspace=4096), lambda: tg.tst_moe(x, w, 2), lambda: tg.tst_logprobs(X, [1, 2]),
                 lambda: tg.tst_moe_pack(np.zeros((2, 4)), *[None] * 6), lambda: tg.tst_moe_pack(x, *[np.zeros((2, 64, 4), np.int8), None] * 3),
                 lambda: tg.tst_moe(X, moe, 2), lambda: tg.tst_moe(x[:, :60], moe, 2), lambda: tg.tst_logprobs(X[0]),
                 lambda: tg.tst_logprobs(X, torch.zeros(3, dtype=torch.int64, device="cuda")),
                 lambda: tg.tst_logprobs(X, torch.zeros(2, dtype=torch.int16, device="cuda")), lambda: tg.tst_logprobs(X.cpu())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: tg.tst_moe(x, moe, 5), lambda: tg.tst_moe(x, moe, 0), lambda: tg.tst_logprobs(X, top=65), lambda: tg.tst_logprobs(X, top=-1)):
        with pytest.raises(tg.TstgemmError) as e:
            call()
        assert e.value.code == -1
