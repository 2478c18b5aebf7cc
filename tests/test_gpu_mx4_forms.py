"""MX FP4 products on the GPU in each form of their tiles, and where sizes, gates and
scales are extreme.  Bounds are those of tests/test_gpu_mx4.py."""

from typing import NamedTuple, Optional

import numpy as np
import pytest

from oracle import mx4 as X
from tests.test_gpu_mx4 import _gated, _matrix, _need_gpu, _run_product, _sum_bound, env  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R", [3, 200])
def test_one_matrix_of_2_to_the_34_weights(env, R):
    """n x k past 2^33 in one group: its last columns against the oracle, in streaming and ring tiles."""
    M, torch = env.M, env.torch
    torch.manual_seed(R)
    N, K, last = 1 << 20, 1 << 14, 96
    st, code_bytes, scale_bytes = M.moe_mx4_size(N, K)
    M.check(st)
    w = [torch.randint(0, 256, (code_bytes,), dtype=torch.uint8, device="cuda"),
         torch.randint(120, 130, (scale_bytes,), dtype=torch.uint8, device="cuda")]
    a, av = _matrix(env, np.random.default_rng(R), R, K)
    y = torch.zeros((R, N), device="cuda")
    torch.cuda.synchronize()
    env.done(M.moe_mx4_gemm(*a, R, *w, 1, None, N, K, y, M.MOE_DTYPE_F32, 0, env.s), "gemm")
    ends = [t[t.numel() // N * (N - last):].cpu().numpy() for t in w]
    want, mag = X.product(av, X.dequantize(*(v[:, :n] for v, n in zip(X.release(*ends, last, K), (K, K // 32)))), [0, R], last)
    assert (np.abs(y[:, N - last:].cpu().numpy() - want) <= _sum_bound(mag, K)).all()
    assert bool((y[:, ::4099] != 0).any(dim=0).all())


def _gate_codes(value):
    """Codes of at most 32 magnitudes of E2M1 that add up to `value`, a multiple of 0.5."""
    codes, left = [], value
    for code, mag in ((7, 6.0), (6, 4.0), (5, 3.0), (4, 2.0), (3, 1.5), (2, 1.0), (1, 0.5)):
        while left >= mag:
            codes.append(code)
            left -= mag
    assert left == 0 and len(codes) <= 32
    return codes


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("R,N", [(3, 256), (40, 512), (700, 4096)])
def test_gates_far_below_zero(env, R, N, out):
    """silu(gate) * up where e^gate, then silu(gate) itself, pass below float32's normal numbers and
    up brings the product back: 16 u for its evaluation, and no more, down to gates of -110."""
    M, torch = env.M, env.torch
    K, up = 256, 2.0 ** 100
    gates = -0.5 * (np.arange(N) % 221)
    codes = np.zeros((2 * N, K), np.uint8)
    for c, g in enumerate(gates):
        q = _gate_codes(-g)
        codes[c, :len(q)] = np.array(q, np.uint8) | 8
    codes[N:, 64] = 2  # 1.0
    scales = np.full((2 * N, K // 32), 127, np.uint8)
    scales[N:, 2] = 127 + 100
    a = [env.up(h) for h in X.hold(np.full((R, K), 2, np.uint8), np.full((R, K // 32), 127, np.uint8))]
    w = [env.up(h) for h in X.hold(codes, scales)]
    code, dtype = env.types[out]
    y = torch.zeros((R, N), dtype=dtype, device="cuda")
    torch.cuda.synchronize()
    env.done(M.moe_mx4_gemm_swiglu(*a, R, *w, 1, None, N, K, y, None, code, 0, env.s), "product")
    want = X.swiglu(gates, np.full(N, up))
    bound = 16 * 2.0 ** -24 * np.abs(want) + 2.0 ** -140
    if out == "bf16":
        bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
    err = np.abs(y.float().cpu().numpy().astype(np.float64) - want)
    assert (err <= bound).all(), sorted(set(gates[np.argwhere(err > bound)[:, 1]]))


class Case(NamedTuple):
    """A product whose launch takes the form it is listed for (tests/test_mx4_form.py holds that
    without a GPU)."""

    name: str
    groups: Optional[tuple]  # rows of each group; None: one matrix of all rows
    rows: int
    N: int
    K: int
    gated: bool
    out: str
    before: int = 0  # rows of no group in front
    stride: int = 0  # 0: N
    pad: int = 0
    clamp: bool = False  # the last offset lies past the rows

    @property
    def offsets(self):
        if self.groups is None:
            return None
        o = self.before + np.concatenate([[0], np.cumsum(self.groups)])
        assert o[-1] <= self.rows
        if self.clamp:
            o[-1] = self.rows + 1000
        return o

    @property
    def group_rows(self):
        return (self.rows,) if self.groups is None else tuple(np.diff(np.clip(self.offsets, 0, self.rows)).tolist())


# rows of a group at the edges of 32-row blocks and of 128-row tiles, cut in one, two, three and four
EDGES = (1, 31, 32, 33, 0, 63, 64, 65, 96, 97, 127, 128, 129, 160, 200, 255, 256, 257, 320, 385)
KINDS = [(False, "f32"), (False, "bf16"), (True, "f32"), (True, "bf16"), (True, "fp4")]


def _cases():
    for gated, out in KINDS:
        tag = f"{'gated' if gated else 'plain'}-{out}"
        odd = out != "fp4"  # MX FP4 rows are whole blocks
        # ring tiles: one to seven slices, so the ring goes round, ends at either parity and in every slot
        n = (289 if odd else 288) if gated else 577
        for i, K in enumerate((200, 512, 700, 1000, 1270, 1700)):
            yield Case(f"ring-{tag}-K{K}", EDGES, sum(EDGES) + 9, n, K, gated, out, before=5,
                       stride=(0, n + 1, n + 6)[i % 3] * odd, pad=(0, 1, 3)[i // 2] * odd, clamp=i % 2 == 1)
        # groups found in the second and third run of 64
        many = tuple(20 + 25 * gated + (7 * g) % 11 for g in range(140))
        yield Case(f"ring-{tag}-140-groups", many, sum(many), 40 if odd else 64, 600, gated, out)
        # one group has all the rows; one matrix, its last column tile cut
        yield Case(f"ring-{tag}-one-group", (0, 2900, 0), 2950, (2 - gated) * 513 if odd else 544, 768, gated, out, before=20)
        yield Case(f"ring-{tag}-dense", None, 417, 3333 * (2 - gated) if odd else 3360, 760, gated, out)
        # streaming tiles: a tile's slices shared by one to eight waves, and dealt unevenly
        for rows in (7, 20, 32):
            yield Case(f"stream-{tag}-{rows}", None, rows, 1001 if odd else 992, (256, 700, 2300)[rows % 3], gated, out,
                       stride=1004 * odd, pad=odd)
        yield Case(f"stream-{tag}-few-groups", (3, 0, 9, 1, 32, 33, 40), 125, 201 if odd else 192, 1270, gated, out, before=4)
        yield Case(f"stream-{tag}-wide", tuple(1 + g % 15 for g in range(40)), 320, (161 if odd else 160) if gated else 481,
                   1270, gated, out, before=2, clamp=True)
        yield Case(f"stream-{tag}-tall", None, 70, 1001 if odd else 992, 2300, gated, out)
        yield Case(f"stream-{tag}-tall-wide", None, 1000 if not gated else 260, 1501 if odd else 1504, 1400, gated, out,
                   stride=1504 * odd, pad=odd)
        yield Case(f"stream-{tag}-tall-groups", (33, 70, 64, 0, 129, 65, 1), 370, 490 if odd else 480, 600, gated, out)
    for gated in (False, True):  # enough tiles for one wave each, several slices
        many = tuple((14 + 12 * gated) - g % 2 for g in range(200))
        yield Case(f"stream-{'gated' if gated else 'plain'}-one-wave", many, sum(many) + 30, 193 if gated else 520, 513, gated,
                   "f32", before=30)
        yield Case(f"stream-{'gated' if gated else 'plain'}-tall-one-wave", None, 70, 1001, 250, gated, "f32")


CASES = list(_cases())


@pytest.mark.parametrize("case", CASES, ids=[c.name for c in CASES])
def test_products_in_every_form(env, case):
    c = case
    rng = np.random.default_rng(CASES.index(c) + 1)
    if c.out != "fp4":
        _run_product(env, rng, c.rows, c.N, c.K, c.offsets, c.gated, c.out, c.stride or c.N, c.pad)
        return
    M = env.M
    offs = [0, c.rows] if c.groups is None else c.offsets
    a, av = _matrix(env, rng, c.rows, c.K, 2)
    w, wv = _matrix(env, rng, (len(offs) - 1) * 2 * c.N, c.K, 2)
    h = env.matrix(c.rows, c.N)
    dev = None if c.groups is None else env.up(np.array(offs, np.int32))
    env.done(M.moe_mx4_gemm_swiglu(*a, c.rows, *w, len(offs) - 1, dev, c.N, c.K, *h, M.MOE_DTYPE_FP4, 0, env.s), "swiglu")
    y, mag = X.product(av, wv, np.clip(offs, 0, c.rows), 2 * c.N)
    ref, bound = _gated(y, _sum_bound(mag, c.K), c.N)
    codes, scales = X.release(h[0].cpu().numpy(), h[1].cpu().numpy(), c.rows, c.N)
    mine = ~np.isnan(ref[:, 0])
    assert (codes[~mine] == [[5]]).sum() == codes[~mine][:, 0::2].size and (scales[~mine] == 0xA5).all()  # 0xA5 as it was
    assert not (codes[mine, c.N:] & 7).any() and not scales[mine, c.N // 32:].any()  # the padding is zeros
    ref, bound, codes, scales = ref[mine], bound[mine], codes[mine, :c.N], scales[mine, :c.N // 32]

    def byte(v):
        return np.clip(np.floor(np.log2(np.maximum(v, 1e-300))) - 2 + 127, 0, 254)

    lo = np.maximum(np.abs(ref) - bound, 0).reshape(len(ref), -1, 32).max(axis=2)
    hi = (np.abs(ref) + bound).reshape(len(ref), -1, 32).max(axis=2)
    assert (scales >= byte(lo)).all() and (scales <= byte(hi)).all()
    scale = np.repeat(np.exp2(scales.astype(np.float64) - 127), 32, axis=1)
    got = X.dequantize(codes, scales)
    assert (got >= X.e2m1_decode(X.e2m1_encode((ref - bound) / scale)) * scale).all()
    assert (got <= X.e2m1_decode(X.e2m1_encode((ref + bound) / scale)) * scale).all()


def _low_rows(dtype):
    """Blocks whose largest magnitudes run from 2^-149 (bf16: 2^-133) up past the smallest block
    exponents, each with every code, the ties between codes and their neighbours, and both signs."""
    least = -149 if dtype == "f32" else -133
    mults = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7], np.float64)
    rows = []
    for e in range(least, -113):
        v = np.concatenate([mults, -mults]) * 2.0 ** e  # largest 7 * 2^e: the block's exponent is e, or -127
        w = v.copy()
        w[np.abs(w) > 4 * 2.0 ** e] /= 4.0  # the same with a largest magnitude of 4 * 2^e
        f = np.float32 if dtype == "f32" else None
        for r in (v, w):
            r32 = r.astype(np.float32)  # rounds what float32 cannot hold
            if f is None:
                r32 = (r32.view(np.uint32) >> 16 << 16).view(np.float32)
            rows.append(r32)
    return np.stack(rows)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_smallest_block_exponents_are_exact(env, dtype):
    """Scale bytes 0, 1, 2 ... with every code, subnormal inputs and subnormal values: exact both ways."""
    M, torch = env.M, env.torch
    v = _low_rows(dtype)
    R, K = v.shape
    codes, scales = X.quantize(v)
    # byte 0 and its neighbours carry every code (of byte 0: all eight magnitudes, from subnormal inputs alone too)
    for byte in (0, 1, 2, 3):
        assert set((codes[scales[:, 0] == byte] & 7).ravel().tolist()) == set(range(8)), byte
    code, t = env.types[dtype]
    x = torch.from_numpy(v).cuda().to(t)
    held = env.matrix(R, K)
    torch.cuda.synchronize()
    assert np.array_equal(x.float().cpu().numpy(), v)
    env.done(M.moe_mx4_quantize(x, code, 0, R, K, None, None, *held, env.s), "quantize")
    c, s = X.release(held[0].cpu().numpy(), held[1].cpu().numpy(), R, K)
    assert np.array_equal(s[:, :1], scales)
    same = (c[:, :K] == codes) | ((c[:, :K] & 7) + (codes & 7) == 0)
    assert same.all(), np.argwhere(~same)[:5]
    want = X.dequantize(codes, scales)
    for name, (out_code, out_t) in env.types.items():
        out = torch.full((R, K), float("nan"), dtype=out_t, device="cuda")
        torch.cuda.synchronize()
        env.done(M.moe_mx4_dequantize(*held, R, K, out, out_code, 0, env.s), "dequantize")
        assert np.array_equal(out.float().cpu().numpy().astype(np.float64), want), name


@pytest.mark.parametrize("R,N", [(40, 70), (700, 4100)])
def test_products_of_the_smallest_and_largest_scales(env, R, N):
    """Rows of scale bytes 0 to 3 times weights of bytes 214 to 254: within the bound, not flushed."""
    M, torch = env.M, env.torch
    rng = np.random.default_rng(R)
    K = 512
    codes = rng.integers(0, 16, (R, K), dtype=np.uint8)
    scales = rng.integers(0, 4, (R, K // 32), dtype=np.uint8)
    wcodes = rng.integers(0, 16, (N, K), dtype=np.uint8)
    wscales = np.repeat(rng.integers(214, 251, (N, 1), dtype=np.uint8), K // 32, axis=1) + rng.integers(0, 5, (N, K // 32), dtype=np.uint8)
    y, mag = X.product(X.dequantize(codes, scales), X.dequantize(wcodes, wscales), [0, R], N)
    a, w = ([env.up(h) for h in X.hold(*m)] for m in ((codes, scales), (wcodes, wscales)))
    out = torch.zeros((R, N), device="cuda")
    torch.cuda.synchronize()
    env.done(M.moe_mx4_gemm(*a, R, *w, 1, None, N, K, out, M.MOE_DTYPE_F32, 0, env.s), "gemm")
    assert (np.abs(out.cpu().numpy() - y) <= _sum_bound(mag, K)).all()
    # and the other way about
    out.zero_()
    torch.cuda.synchronize()
    y, mag = X.product(X.dequantize(wcodes, wscales)[:R], X.dequantize(codes, scales)[:N], [0, min(R, N)], min(R, N))
    n = min(R, N)
    a, w = ([env.up(h) for h in X.hold(*m)] for m in ((wcodes[:n], wscales[:n]), (codes[:n], scales[:n])))
    out = torch.zeros((n, n), device="cuda")
    torch.cuda.synchronize()
    env.done(M.moe_mx4_gemm(*a, n, *w, 1, None, n, K, out, M.MOE_DTYPE_F32, 0, env.s), "gemm")
    assert (np.abs(out.cpu().numpy() - y[:n]) <= _sum_bound(mag[:n], K)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_whose_offsets_pass_32_bits(env, dtype):
    """Quantized from, and dequantized and multiplied into, rows 2^31 and more elements apart."""
    M, torch = env.M, env.torch
    rng = np.random.default_rng(13)
    R, K, stride = 3, 300, (1 << 31) + 5
    code, t = env.types[dtype]
    v = rng.standard_normal((R, K)).astype(np.float32)
    v = (v.view(np.uint32) >> 16 << 16).view(np.float32)
    buf = torch.empty((R - 1) * stride + K + 1, dtype=t, device="cuda")
    rows = torch.as_strided(buf, (R, K + 1), (stride, 1))
    rows[:, :K] = torch.from_numpy(v).cuda().to(t)
    rows[:, K] = float("nan")
    held = env.matrix(R, K)
    torch.cuda.synchronize()
    env.done(M.moe_mx4_quantize(buf, code, stride, R, K, None, None, *held, env.s), "quantize")
    padded = np.pad(v, ((0, 0), (0, -K % 32)))
    want = X.quantize(padded)
    c, s = X.release(held[0].cpu().numpy(), held[1].cpu().numpy(), R, K)
    n = padded.shape[1]
    assert ((c[:, :n] == want[0]) | ((c[:, :n] & 7) + (want[0] & 7) == 0)).all() and np.array_equal(s[:, :n // 32], want[1])
    rows.zero_()
    torch.cuda.synchronize()
    env.done(M.moe_mx4_dequantize(*held, R, K, buf, code, stride, env.s), "dequantize")
    values = X.dequantize(*want)[:, :K]
    assert np.array_equal(rows[:, :K].float().cpu().numpy(), values.astype(np.float32)) and not rows[:, K].any()
    w, wv = _matrix(env, rng, K, K)
    y, mag = X.product(values, wv, [0, R], K)
    bound = _sum_bound(mag, K) + (2.0 ** -8 * (np.abs(y) + _sum_bound(mag, K)) if dtype == "bf16" else 0.0)
    env.done(M.moe_mx4_gemm(*held, R, *w, 1, None, K, K, buf, code, stride, env.s), "gemm")
    assert (np.abs(rows[:, :K].float().cpu().numpy() - y) <= bound).all() and not rows[:, K].any()
