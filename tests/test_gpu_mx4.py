"""MX FP4 matrices and products on the GPU, through the C ABI, against the
float64 oracle (oracle/mx4.py).

Tolerances, derived from the arithmetic (u = 2^-24):
* quantized codes and scales, packed bytes and dequantized values: exact;
* a product's sum of K terms in float32, in any order and with truncating
  additions allowed: |err| <= 2 (K + 64) u sum |a w|; rounding to bf16 adds half
  an ulp, at most 2^-8 of the value;
* SwiGLU: with bounds dg, du on the two sums, |err| <= 1.1 |up| dg + |silu(gate)| du
  (silu's slope is below 1.1) + 16 u |value| for its own evaluation, + 1.1 dg du;
* SwiGLU in FP4: the block's scale byte is that of a magnitude within the bound of
  the block's largest, and each code is that of some value within the bound
  under that scale.
"""

import numpy as np
import pytest

from oracle import mx4 as X
from synth import bf16_bits_to_f32

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def env():
    import torch

    from paper_2609_00993_amd import moepd as M

    class Env:
        pass

    e = Env()
    e.M, e.torch, e.s = M, torch, torch.cuda.Stream()
    e.types = {"f32": (M.MOE_DTYPE_F32, torch.float32), "bf16": (M.MOE_DTYPE_BF16, torch.bfloat16)}

    def up(a):
        t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
        torch.cuda.synchronize()
        return t

    def done(st, what):
        M.check(st, what)
        torch.cuda.synchronize()

    def matrix(rows, cols, fill=0xA5):
        st, c, s = M.moe_mx4_size(rows, cols)
        M.check(st)
        t = [torch.full((max(n, 16),), fill, dtype=torch.uint8, device="cuda") for n in (c, s)]
        torch.cuda.synchronize()
        return t

    e.up, e.done, e.matrix = up, done, matrix
    return e


def _rows(rng, R, K, dtype):
    """Rows with exponents all over, blocks of zeros and of rounding ties; values of the given type."""
    v = rng.standard_normal((R, K)) * np.exp2(rng.integers(-30, 30, (R, 1)))
    v *= np.where(rng.random((R, K)) < 0.02, 16.0, 1.0)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.5, 4.0])
    pick = rng.random((R, K)) < 0.3
    v = np.where(pick, rng.choice(ties, (R, K)) * rng.choice([-1.0, 1.0], (R, K)), v)
    v[rng.random((R, K)) < 0.1] = 0.0
    if R > 2 and K > 40:
        v[1, 8:72] = 0.0
        v[2, :32] = np.exp2(-135.0) * np.arange(32)  # below the smallest block exponent
    v = v.astype(np.float32)
    if dtype == "bf16":
        v = (v.view(np.uint32) >> 16 << 16).view(np.float32)
    return v


def _device_rows(env, v, dtype, stride, offset):
    """v on the device, rows `stride` apart, the first `offset` elements into the allocation."""
    torch = env.torch
    R, K = v.shape
    buf = torch.full((offset + max(R, 1) * stride + 8,), float("nan"), dtype=env.types[dtype][1], device="cuda")
    view = buf[offset:offset + R * stride].view(R, stride)
    view[:, :K] = torch.from_numpy(v).cuda().to(buf.dtype)
    torch.cuda.synchronize()
    return buf[offset:]


def _blocks(v):
    K = v.shape[1]
    p = np.zeros((v.shape[0], -(-K // 32) * 32))
    p[:, :K] = v
    return p


def _check_quantized(held, want, R, K, what):
    c, s = X.release(held[0].cpu().numpy(), held[1].cpu().numpy(), R, K)
    n = want[0].shape[1]
    # a zero keeps either sign
    gc, wc = c[:, :n], want[0]
    same = (gc == wc) | ((gc & 7) + (wc & 7) == 0)
    assert same.all(), (what, np.argwhere(~same)[:5])
    assert np.array_equal(s[:, :n // 32], want[1]), what
    assert not (c[:, n:] & 7).any() and not s[:, n // 32:].any(), what


SHAPES = [(1, 1), (1, 256), (2, 33), (31, 64), (32, 255), (33, 257), (65, 7), (64, 512), (100, 801), (7, 2048)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,K", SHAPES)
def test_quantize_and_dequantize_are_exact(env, R, K, dtype):
    M = env.M
    rng = np.random.default_rng(R * 1000 + K)
    v = _rows(rng, R, K, dtype)
    want = X.quantize(_blocks(v))
    for stride, offset in ((K, 0), (K + 8 - K % 8, 0), (K + 5, 3)):
        x = _device_rows(env, v, dtype, stride, offset)
        held = env.matrix(R, K)
        env.done(M.moe_mx4_quantize(x, env.types[dtype][0], stride, R, K, None, None, *held, env.s), "quantize")
        _check_quantized(held, want, R, K, (R, K, dtype, stride, offset))
        for name, (code, t) in env.types.items():
            out = _device_rows(env, np.zeros((R, K), np.float32), name, stride, offset)
            env.done(M.moe_mx4_dequantize(*held, R, K, out, code, stride, env.s), "dequantize")
            got = out[:R * stride].view(R, stride).float().cpu().numpy()
            assert np.array_equal(got[:, :K], X.dequantize(*want)[:, :K].astype(np.float32)), (name, stride)
            assert np.isnan(got[:, K:]).all()  # nothing between the rows


def test_quantize_nan_and_infinity(env):
    M = env.M
    v = np.ones((3, 96), np.float32)
    v[0, 5], v[1, 40], v[1, 41], v[2, 95] = np.nan, np.inf, -1.0, -np.inf
    v[2, 0] = 3e38
    held = env.matrix(3, 96)
    x = _device_rows(env, v, "f32", 96, 0)
    env.done(M.moe_mx4_quantize(x, M.MOE_DTYPE_F32, 0, 3, 96, None, None, *held, env.s), "quantize")
    _check_quantized(held, X.quantize(v), 3, 96, "nan")
    out = env.torch.empty((3, 96), device="cuda")
    env.torch.cuda.synchronize()
    env.done(M.moe_mx4_dequantize(*held, 3, 96, out, M.MOE_DTYPE_F32, 0, env.s), "dequantize")
    got = out.cpu().numpy()
    assert np.isnan(got[0, :32]).all() and np.isnan(got[1, 32:64]).all() and np.isnan(got[2, 64:]).all()
    assert np.isfinite(got[0, 32:]).all() and np.isfinite(got[2, :64]).all()
    # a row with a NaN block gives NaN products, its neighbours do not
    wv = _rows(np.random.default_rng(1), 32, 96, "f32")
    wv = np.sign(wv) + 0.5
    w = env.matrix(32, 96)
    env.done(M.moe_mx4_quantize(env.up(wv.astype(np.float32)), M.MOE_DTYPE_F32, 0, 32, 96, None, None, *w, env.s), "w")
    v[1:] = 1.0
    env.done(M.moe_mx4_quantize(env.up(v), M.MOE_DTYPE_F32, 0, 3, 96, None, None, *held, env.s), "a")
    y = env.torch.zeros((3, 32), device="cuda")
    env.torch.cuda.synchronize()
    env.done(M.moe_mx4_gemm(*held, 3, *w, 1, None, 32, 96, y, M.MOE_DTYPE_F32, 0, env.s), "gemm")
    y = y.cpu().numpy()
    assert np.isnan(y[0]).all() and np.isfinite(y[1:]).all()


@pytest.mark.parametrize("K", [64, 300])
def test_quantize_gathers_and_counts_rows(env, K):
    M, torch = env.M, env.torch
    rng = np.random.default_rng(K)
    v = _rows(rng, 50, K, "bf16")
    index = rng.integers(-2, 50, 131).astype(np.int32)
    x = _device_rows(env, v, "bf16", K, 0)
    for count in (None, 131, 70, 64, 1, 0, -3, 500):
        held = env.matrix(131, K)
        n = None if count is None else env.up(np.array([count], np.int32))
        env.done(M.moe_mx4_quantize(x, M.MOE_DTYPE_BF16, 0, 131, K, env.up(index), n, *held, env.s), "quantize")
        used = 131 if count is None else min(max(count, 0), 131)
        g = np.where(index[:used, None] >= 0, v[np.maximum(index[:used], 0)], 0.0)
        filled = -(-used // 32) * 32
        g = np.concatenate([g, np.zeros((min(filled, 131) - used, K))]) if filled else g
        _check_quantized([held[0][:filled * -(-K // 256) * 128], held[1][:filled * -(-K // 256) * 8]],
                         X.quantize(_blocks(g)), g.shape[0], K, count)
        rest = held[0][filled * -(-K // 256) * 128:]
        assert (rest == 0xA5).all()  # blocks past the count are not touched


def test_pack_is_the_held_order(env):
    M = env.M
    rng = np.random.default_rng(8)
    for R, K in ((1, 32), (33, 96), (70, 512), (32, 288)):
        codes = rng.integers(0, 16, (R, K), dtype=np.uint8)
        scales = rng.integers(0, 256, (R, K // 32), dtype=np.uint8)
        held = env.matrix(R, K)
        env.done(M.moe_mx4_pack(env.up(codes[:, 0::2] | (codes[:, 1::2] << 4)), env.up(scales), R, K, *held, env.s), "pack")
        want = X.hold(codes, scales)
        assert np.array_equal(held[0].cpu().numpy(), want[0]) and np.array_equal(held[1].cpu().numpy(), want[1])


def _matrix(env, rng, R, K, spread=4):
    """(held device buffers, float64 values) of a random matrix, every code and a range of scales in use."""
    Kb = -(-K // 32) * 32
    codes = rng.integers(0, 16, (R, Kb), dtype=np.uint8)
    codes[:, K:] = 0
    scales = rng.integers(127 - spread, 128 + spread, (R, Kb // 32), dtype=np.uint8)
    held = X.hold(codes, scales)
    return [env.up(h) for h in held], X.dequantize(codes, scales)[:, :K]


def _sum_bound(mag, K):
    return 2.0 * (K + 64) * U * mag


def _run_product(env, rng, R, N, K, offsets, gated, out, stride, pad):
    M, torch = env.M, env.torch
    groups = 1 if offsets is None else len(offsets) - 1
    a, av = _matrix(env, rng, R, K)
    w, wv = _matrix(env, rng, groups * N * (2 if gated else 1), K)
    code, t = env.types[out]
    buf = torch.full((R * stride + pad + 8,), -777.0, dtype=t, device="cuda")
    dev = None if offsets is None else env.up(np.array(offsets, np.int32))
    torch.cuda.synchronize()
    if gated:
        st = M.moe_mx4_gemm_swiglu(*a, R, *w, groups, dev, N, K, buf[pad:], None, code, stride, env.s)
    else:
        st = M.moe_mx4_gemm(*a, R, *w, groups, dev, N, K, buf[pad:], code, stride, env.s)
    env.done(st, "product")
    got = buf.float().cpu().numpy().astype(np.float64)
    assert (got[:pad] == got[-1]).all() and (got[pad + R * stride:] == got[-1]).all()
    grid = got[pad:pad + R * stride].reshape(R, stride)
    assert (grid[:, N:] == got[-1]).all()  # nothing between the rows
    offs = [0, R] if offsets is None else np.clip(offsets, 0, R)
    y, mag = X.product(av, wv, offs, N * (2 if gated else 1))
    bound = _sum_bound(mag, K)
    if gated:
        y, bound = _gated(y, bound, N)
    if out == "bf16":
        bound = bound + 2.0 ** -8 * (np.abs(y) + bound)
    mine = ~np.isnan(y[:, 0])
    assert (grid[~mine, :N] == got[-1]).all()  # rows of no group
    err = np.abs(grid[mine, :N] - y[mine])
    assert (err <= bound[mine]).all(), (float((err / bound[mine]).max()), np.argwhere(err > bound[mine])[:4])


def _gated(y, bound, N):
    g, u, dg, du = y[:, :N], y[:, N:], bound[:, :N], bound[:, N:]
    h = X.swiglu(g, u)
    silu = X.swiglu(g, np.ones_like(g))
    return h, 1.1 * np.abs(u) * dg + np.abs(silu) * du + 1.1 * dg * du + 16 * U * np.abs(h)


DENSE = [(1, 1, 32), (1, 33, 256), (2, 64, 257), (31, 100, 512), (32, 32, 768), (33, 65, 1024), (64, 257, 100),
         (65, 31, 1280), (129, 128, 256), (300, 520, 1536), (513, 260, 768), (1, 700, 4096), (17, 1000, 2048),
         (300, 512, 4096), (40, 96, 4096)]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("R,N,K", DENSE)
def test_dense_products(env, R, N, K, gated, out):
    rng = np.random.default_rng(R * 7919 + N * 31 + K)
    _run_product(env, rng, R, N, K, None, gated, out, N, 0)


@pytest.mark.parametrize("out,stride,pad", [("f32", 104, 0), ("f32", 101, 0), ("f32", 104, 1), ("bf16", 108, 0),
                                            ("bf16", 103, 0), ("bf16", 104, 2)])
@pytest.mark.parametrize("gated", [False, True])
def test_strides_and_alignment_of_the_output(env, gated, out, stride, pad):
    for R in (5, 260):
        _run_product(env, np.random.default_rng(stride + pad), R, 100, 300, None, gated, out, stride, pad)


def _offsets(rng, kind, groups, rows):
    if kind == "even":
        return np.linspace(0, rows, groups + 1).astype(int)
    if kind == "one":  # all rows in one group, the others empty
        o = np.zeros(groups + 1, int)
        o[groups // 2 + 1:] = rows
        return o
    if kind == "gaps":  # rows before the first and from the last offset on belong to no group
        o = np.sort(rng.integers(3, rows - 5, groups + 1))
        return o
    if kind == "outside":  # offsets past the rows are clamped
        o = np.sort(rng.integers(0, rows + 40, groups + 1))
        o[-1] = rows + 1000
        return o
    return np.concatenate([[0], np.sort(rng.integers(0, rows + 1, groups - 1)), [rows]])


GROUPED = [("random", 3, 40, 65, 256), ("random", 8, 500, 96, 512), ("even", 5, 35, 128, 768), ("one", 6, 270, 64, 512),
           ("gaps", 7, 300, 40, 256), ("outside", 4, 200, 32, 256), ("random", 70, 150, 33, 256),
           ("random", 150, 900, 32, 64), ("even", 4, 1100, 260, 512), ("random", 300, 200, 17, 96),
           ("random", 6, 1500, 300, 1280), ("one", 3, 700, 513, 256), ("even", 2, 400, 64, 2816)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kind,groups,rows,N,K", GROUPED)
def test_grouped_products(env, kind, groups, rows, N, K, gated):
    rng = np.random.default_rng(groups * 101 + rows)
    _run_product(env, rng, rows, N, K, _offsets(rng, kind, groups, rows), gated, "f32", N, 0)


@pytest.mark.parametrize("rows_per_group", [1, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 160, 161, 192, 193, 224,
                                            255, 256, 257, 320, 511, 513])
def test_tile_edges(env, rows_per_group):
    """Groups of exactly so many rows, none starting at a multiple of a tile."""
    rng = np.random.default_rng(rows_per_group)
    offs = 5 + np.arange(4) * rows_per_group
    for gated in (False, True):
        _run_product(env, rng, int(offs[-1]) + 3, 288, 768, offs, gated, "f32", 288, 0)


@pytest.mark.parametrize("kind,groups,rows,N,K", [("random", 3, 40, 64, 256), ("even", 4, 9, 256, 512),
                                                  ("gaps", 5, 300, 96, 768), ("even", 3, 900, 320, 512),
                                                  ("one", 2, 333, 1024, 256), ("random", 40, 100, 32, 256)])
def test_swiglu_into_fp4(env, kind, groups, rows, N, K):
    M, torch = env.M, env.torch
    rng = np.random.default_rng(rows + N)
    offs = _offsets(rng, kind, groups, rows)
    a, av = _matrix(env, rng, rows, K, 2)
    w, wv = _matrix(env, rng, groups * 2 * N, K, 2)
    h = env.matrix(rows, N)
    env.done(M.moe_mx4_gemm_swiglu(*a, rows, *w, groups, env.up(offs.astype(np.int32)), N, K, *h, M.MOE_DTYPE_FP4, 0,
                                   env.s), "swiglu")
    y, mag = X.product(av, wv, offs, 2 * N)
    ref, bound = _gated(y, _sum_bound(mag, K), N)
    c, s = X.release(h[0].cpu().numpy(), h[1].cpu().numpy(), rows, N)
    mine = ~np.isnan(ref[:, 0])
    assert not (c[mine, N:] & 7).any() and not s[mine, N // 32:].any()  # the padding is zeros
    ref, bound, c, s = ref[mine], bound[mine], c[mine, :N], s[mine, :N // 32]

    def byte(v):
        return np.clip(np.floor(np.log2(np.maximum(v, 1e-300))) - 2 + 127, 0, 254)

    lo = np.maximum(np.abs(ref) - bound, 0).reshape(len(ref), -1, 32).max(axis=2)
    hi = (np.abs(ref) + bound).reshape(len(ref), -1, 32).max(axis=2)
    assert (s >= byte(lo)).all() and (s <= byte(hi)).all()
    scale = np.repeat(np.exp2(s.astype(np.float64) - 127), 32, axis=1)
    got = X.dequantize(c, s)
    assert (got >= X.e2m1_decode(X.e2m1_encode((ref - bound) / scale)) * scale).all()
    assert (got <= X.e2m1_decode(X.e2m1_encode((ref + bound) / scale)) * scale).all()


@pytest.mark.parametrize("R,N", [(3, 40), (300, 520), (700, 4100)])
def test_nan_rows_stay_nan_in_bf16(env, R, N):
    """Of a matrix's rows one has a NaN block, in every tile form: its products are NaN, no other's."""
    M, torch = env.M, env.torch
    rng = np.random.default_rng(R)
    K = 256
    codes = rng.integers(0, 16, (R, K), dtype=np.uint8)
    scales = np.full((R, K // 32), 127, np.uint8)
    scales[R // 2, 3] = 255
    a = [env.up(h) for h in X.hold(codes, scales)]
    w, _ = _matrix(env, rng, 2 * N, K, 1)
    for gated in (False, True):
        y = torch.zeros((R, N), dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        if gated:
            st = M.moe_mx4_gemm_swiglu(*a, R, *w, 1, None, N, K, y, None, M.MOE_DTYPE_BF16, 0, env.s)
        else:
            st = M.moe_mx4_gemm(*a, R, *w, 1, None, N, K, y, M.MOE_DTYPE_BF16, 0, env.s)
        env.done(st, "product")
        bad = torch.isnan(y).cpu().numpy()
        assert bad[R // 2].all() and not np.delete(bad, R // 2, axis=0).any()


@pytest.mark.parametrize("R,N", [(3, 64), (300, 512), (700, 4096)])
@pytest.mark.parametrize("infinite", [False, True])
def test_gates_past_float32(env, R, N, infinite):
    """Gates of 1.5 * 2^127 (times log2 e past the largest float) and of infinity are gates like
    any other: silu of one is itself, and u = 2^-12."""
    M, torch = env.M, env.torch
    K = 256
    codes = np.full((2 * N, K), 2, np.uint8)  # 1.0
    codes[:N] = 3  # 1.5
    a = [env.up(h) for h in X.hold(np.full((R, K), 2, np.uint8), np.full((R, K // 32), 127 + 60, np.uint8))]
    scale = np.full((2 * N, K // 32), 127 - 80, np.uint8)  # u = 2^(8 + 60 - 80)
    scale[:N] = 127 + 70 if infinite else 127 + 59
    w = [env.up(h) for h in X.hold(codes, scale)]
    y = torch.zeros((R, N), device="cuda")
    torch.cuda.synchronize()
    env.done(M.moe_mx4_gemm_swiglu(*a, R, *w, 1, None, N, K, y, None, M.MOE_DTYPE_F32, 0, env.s), "product")
    want = float("inf") if infinite else 1.5 * 2.0 ** (127 - 12)
    got = y.cpu().numpy().astype(np.float64)
    assert (got == want).all() if np.isinf(want) else (np.abs(got - want) <= 8 * 2.0 ** -24 * want).all()


def test_matrices_past_four_gigabytes(env):
    """Codes, weights and results whose byte offsets pass 32 bits: the last rows are those of a small call."""
    M, torch = env.M, env.torch
    torch.manual_seed(5)
    # 1,100,000 rows x 8192: 4.5 GB of codes, gathered from 64 rows
    R, K, N = 1_100_000, 8192, 32
    x = torch.randn((64, K), device="cuda", dtype=torch.bfloat16)
    index = torch.randint(0, 64, (R,), dtype=torch.int32, device="cuda")
    w, wv = _matrix(env, np.random.default_rng(1), N, K)
    q, one = env.matrix(R, K, 0), env.matrix(64, K)
    y, small = torch.empty((R, N), device="cuda"), torch.empty((64, N), device="cuda")
    torch.cuda.synchronize()
    assert q[0].numel() > 1 << 32
    M.check(M.moe_mx4_quantize(x, M.MOE_DTYPE_BF16, 0, R, K, index, None, *q, env.s))
    M.check(M.moe_mx4_gemm(*q, R, *w, 1, None, N, K, y, M.MOE_DTYPE_F32, 0, env.s))
    M.check(M.moe_mx4_quantize(x, M.MOE_DTYPE_BF16, 0, 64, K, None, None, *one, env.s))
    env.done(M.moe_mx4_gemm(*one, 64, *w, 1, None, N, K, small, M.MOE_DTYPE_F32, 0, env.s), "small")
    # the same products, added in another order by other tiles
    c, s = X.release(one[0].cpu().numpy(), one[1].cpu().numpy(), 64, K)
    _, mag = X.product(X.dequantize(c, s), wv, [0, 64], N)
    bound = torch.from_numpy(2 * _sum_bound(mag, K)).cuda()
    pick = index.long()
    for at in (slice(0, 1000), slice(R // 2, R // 2 + 1000), slice(R - 1000, R)):
        assert ((y[at].double() - small[pick[at]].double()).abs() <= bound[pick[at]]).all()
    del q, y
    # 700 groups of 3200 weight rows x 4096: 4.6 GB; each group's row is the same, the last weights are known
    G, N, K = 700, 3200, 4096
    st, cb, sb = M.moe_mx4_size(G * N, K)
    assert cb > 1 << 32
    wc = torch.randint(0, 256, (cb,), dtype=torch.uint8, device="cuda")
    ws = torch.randint(120, 130, (sb,), dtype=torch.uint8, device="cuda")
    a, _ = _matrix(env, np.random.default_rng(2), G, K)
    offs = torch.arange(G + 1, dtype=torch.int32, device="cuda")
    y, small = torch.empty((G, N), device="cuda"), torch.empty((G, N), device="cuda")
    torch.cuda.synchronize()
    M.check(M.moe_mx4_gemm(*a, G, wc, ws, G, offs, N, K, y, M.MOE_DTYPE_F32, 0, env.s))
    last = (cb // G * (G - 1), sb // G * (G - 1))
    env.done(M.moe_mx4_gemm(*a, G, wc[last[0]:], ws[last[1]:], 1, None, N, K, small, M.MOE_DTYPE_F32, 0, env.s), "last")
    scale = small[-1].abs().max()
    assert float(scale) > 0 and float((y[-1] - small[-1]).abs().max()) <= 1e-4 * float(scale)
    del wc, ws
    # 700,001 rows x 3201 bf16 results: 4.5 GB
    R, N, K = 700_001, 3201, 256
    a, w = env.matrix(R, K, 0x35), _matrix(env, np.random.default_rng(3), N, K)[0]
    a[1].fill_(127)
    y = torch.zeros((R, N), dtype=torch.bfloat16, device="cuda")
    small = torch.zeros((1, N), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    M.check(M.moe_mx4_gemm(*a, R, *w, 1, None, N, K, y, M.MOE_DTYPE_BF16, 0, env.s))
    env.done(M.moe_mx4_gemm(*a, 1, *w, 1, None, N, K, small, M.MOE_DTYPE_BF16, 0, env.s), "row")
    assert (y == small).all()  # every row is the same; one slice has one order


def test_products_are_deterministic_and_graph_safe(env):
    """A captured chain (quantize, gate/up, down) replays to the eager bits, with other work between."""
    M, torch = env.M, env.torch
    rng = np.random.default_rng(12)
    R, H, I, G = 333, 512, 256, 4
    offs = env.up(_offsets(rng, "random", G, R).astype(np.int32))
    x = env.up(rng.standard_normal((100, H)).astype(np.float32))
    index = env.up(rng.integers(0, 100, R).astype(np.int32))
    gu, _ = _matrix(env, rng, G * 2 * I, H)
    dn, _ = _matrix(env, rng, G * H, I)
    q, h = env.matrix(R, H), env.matrix(R, I)
    y = torch.zeros((R, H), device="cuda")
    torch.cuda.synchronize()

    def chain(s):
        M.check(M.moe_mx4_quantize(x, M.MOE_DTYPE_F32, 0, R, H, index, offs[G:], *q, s))
        M.check(M.moe_mx4_gemm_swiglu(*q, R, *gu, G, offs, I, H, *h, M.MOE_DTYPE_FP4, 0, s))
        M.check(M.moe_mx4_gemm(*h, R, *dn, G, offs, H, I, y, M.MOE_DTYPE_F32, 0, s))

    chain(env.s)
    torch.cuda.synchronize()
    want = y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=env.s):
        chain(env.s)
    for _ in range(3):
        y.fill_(-1.0)
        for b in (*q, *h):
            b.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        chain(env.s)
        torch.cuda.synchronize()
        assert torch.equal(y, want)
