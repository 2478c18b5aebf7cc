"""The gated feed-forward block and its backward pass on the GPU, through the C ABI, against
the float64 oracle (oracle/ffn.py).

Tolerances, derived from the arithmetic (u = 2^-24; S the sum of the magnitudes of a sum's
K products):
* a sum of K products in float32, in any order, with products exact or rounded: e = (K + 8) 2 u S
  (twice u, for accumulators that cut off);
* h = silu(g) up: silu's slope is below 1.1, so 1.1 e_g |up| + (|silu(g)| + 1.1 e_g) e_up, and 16 u |h| for the
  function;
* dg = dh F, F = up s (1 + g (1 - s)), |s (1 + g (1 - s))| < 1.1: e_dh |F| + 64 u |dh up|; du = dh silu(g): e_dh |silu(g)|
  + 16 u |du|;
* a bf16 result adds half a step, 2^-8 of the value (float32: 2^-24);
* results below the normal range may be flushed: 1e-37 absolute.
"""

import numpy as np
import pytest

from oracle import ffn as F

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SENTINEL = 768.0  # of what must not be written


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _torch_type(dtype):
    import torch

    return torch.float32 if dtype == "f32" else torch.bfloat16


def _code(dtype):
    from paper_2609_00993_amd import moepd as M

    return M.MOE_DTYPE_F32 if dtype == "f32" else M.MOE_DTYPE_BF16


def _dev(a, dtype):
    import torch

    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.float32))).cuda().to(_torch_type(dtype))


def _strided(a, dtype, stride, fill=float("nan")):
    """Rows `stride` apart, NaN between them, on the device."""
    import torch

    t = torch.full((max(a.shape[0], 1), stride), fill, dtype=_torch_type(dtype), device="cuda")
    if a.shape[0]:
        t[:a.shape[0], :a.shape[1]] = _dev(a, dtype)
    return t


def _host(t):
    return t.float().cpu().numpy().astype(np.float64)


def _values(rng, shape, dtype, std=1.0):
    v = (rng.standard_normal(shape) * std).astype(np.float32)
    return _host(_dev(v, dtype))


def _step(dtype):
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24


def _close(got, want, tol, what):
    bad = ~(np.abs(got - want) <= tol + 1e-37)
    bad &= ~(np.isnan(got) & np.isnan(want))
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: " \
        f"{got[tuple(np.argwhere(bad)[0])]} for {want[tuple(np.argwhere(bad)[0])]}, tolerance {tol[tuple(np.argwhere(bad)[0])]}"


class Block:
    """Inputs of one block, and its calls on the device."""

    def __init__(self, rows, H, I, offsets=None, dtype="bf16", seed=0, pad=0):
        import torch

        self.rows, self.H, self.I, self.dtype, self.pad = rows, H, I, dtype, pad
        rng = np.random.default_rng(seed)
        self.rng = rng
        self.offsets = offsets
        self.spans = F.groups_of(offsets, rows)
        G = self.G = len(self.spans)
        self.x = _values(rng, (rows, H), dtype)
        self.dy = _values(rng, (rows, H), dtype)
        self.w_gu = _values(rng, (G, 2 * I, H), dtype, 1.5 / np.sqrt(H))
        self.w_dn = _values(rng, (G, H, I), dtype, 1.0 / np.sqrt(I))
        self.gu = _values(rng, (rows, 2 * I), dtype, 1.5)
        self.d_off = None if offsets is None else torch.tensor(list(offsets), dtype=torch.int32, device="cuda")
        self.stream = torch.cuda.Stream()
        # rows of no group hold NaN, which must reach nothing
        self.in_group = np.zeros(rows, bool)
        for lo, hi in self.spans:
            self.in_group[lo:hi] = True
        for a in (self.x, self.dy, self.gu):
            a[~self.in_group] = np.nan

    def empty(self, rows, cols, dtype=None, stride=None):
        import torch

        return torch.full((max(rows, 1), stride or cols), SENTINEL, dtype=_torch_type(dtype or self.dtype), device="cuda")

    def check_rows(self, got, want, tol, what):
        assert (got[~self.in_group] == SENTINEL).all(), f"{what}: rows of no group were written"
        live = self.in_group
        _close(got[live], want[live], tol[live], what)

    def gate_up(self, keep=True):
        import torch

        from paper_2609_00993_amd import moepd as M

        x = _strided(self.x, self.dtype, self.H + self.pad)
        w = _dev(self.w_gu, self.dtype)
        h, gu = self.empty(self.rows, self.I), self.empty(self.rows, 2 * self.I) if keep else None
        torch.cuda.synchronize()
        M.check(M.moe_ffn_gate_up(x, self.H + self.pad, self.rows, w, self.G, self.d_off, self.H, self.I, _code(self.dtype),
                                  gu, h, self.stream))
        torch.cuda.synchronize()
        want, S = F.rows_times(self.x, self.w_gu, self.spans)
        e = (self.H + 8) * 2 * U * S
        I, s = self.I, _step(self.dtype)
        if keep:
            self.check_rows(_host(gu)[:self.rows], want, e + s * np.abs(want), "gate_up")
        g, up, eg, eu = want[:, :I], want[:, I:], e[:, :I], e[:, I:]
        hw = F.swiglu(g, up)
        tol = 1.1 * eg * np.abs(up) + (np.abs(F.silu(g)) + 1.1 * eg) * eu + (16 * U + s) * np.abs(hw)
        self.check_rows(_host(h)[:self.rows], hw, tol * (1 + s), "h")
        return _host(h)[:self.rows]

    def down(self, out="bf16", pad=0):
        import torch

        from paper_2609_00993_amd import moepd as M

        a = _values(self.rng, (self.rows, self.I), self.dtype)
        a[~self.in_group] = np.nan
        y = self.empty(self.rows, self.H, out, self.H + pad)
        d_a, d_w = _strided(a, self.dtype, self.I), _dev(self.w_dn, self.dtype)
        torch.cuda.synchronize()
        M.check(M.moe_ffn_down(d_a, self.rows, d_w, self.G, self.d_off, self.H, self.I, _code(self.dtype), y, _code(out),
                               self.H + pad, self.stream))
        torch.cuda.synchronize()
        want, S = F.rows_times(a, self.w_dn, self.spans)
        got = _host(y)[:self.rows]
        assert (got[:, self.H:] == SENTINEL).all()
        self.check_rows(got[:, :self.H], want, (self.I + 8) * 2 * U * S + _step(out) * np.abs(want), "y")

    def down_backward(self, keep_h=True):
        import torch

        from paper_2609_00993_amd import moepd as M

        d_dy = _strided(self.dy, self.dtype, self.H + self.pad)
        d_gu, d_w = _strided(self.gu, self.dtype, 2 * self.I), _dev(self.w_dn, self.dtype)
        d, h = self.empty(self.rows, 2 * self.I), self.empty(self.rows, self.I) if keep_h else None
        torch.cuda.synchronize()
        M.check(M.moe_ffn_down_backward(d_dy, self.H + self.pad, self.rows, d_w, d_gu, self.G, self.d_off, self.H, self.I,
                                        _code(self.dtype), d, h, self.stream))
        torch.cuda.synchronize()
        dh, S = F.rows_times(self.dy, self.w_dn, self.spans, transposed=False)
        e = (self.H + 8) * 2 * U * S
        I, s = self.I, _step(self.dtype)
        g, up = self.gu[:, :I], self.gu[:, I:]
        dg, du = F.swiglu_gradient(g, up, dh)
        Fg, Fu = F.swiglu_gradient(g, up, np.ones_like(dh))
        tol = np.concatenate([e * np.abs(Fg) + 64 * U * np.abs(dh * up), e * np.abs(Fu) + 16 * U * np.abs(du)], axis=1)
        want = np.concatenate([dg, du], axis=1)
        self.check_rows(_host(d)[:self.rows], want, tol * (1 + s) + s * np.abs(want), "dgate_up")
        if keep_h:
            hw = F.swiglu(g, up)
            self.check_rows(_host(h)[:self.rows], hw, (16 * U + s) * (1 + s) * np.abs(hw), "h anew")

    def gate_up_backward(self, out="bf16", pad=0):
        import torch

        from paper_2609_00993_amd import moepd as M

        d_a, d_w = _strided(self.gu, self.dtype, 2 * self.I), _dev(self.w_gu, self.dtype)
        dx = self.empty(self.rows, self.H, out, self.H + pad)
        torch.cuda.synchronize()
        M.check(M.moe_ffn_gate_up_backward(d_a, self.rows, d_w, self.G, self.d_off, self.H, self.I, _code(self.dtype), dx,
                                           _code(out), self.H + pad, self.stream))
        torch.cuda.synchronize()
        want, S = F.rows_times(self.gu, self.w_gu, self.spans, transposed=False)
        got = _host(dx)[:self.rows]
        assert (got[:, self.H:] == SENTINEL).all()
        self.check_rows(got[:, :self.H], want, (2 * self.I + 8) * 2 * U * S + _step(out) * np.abs(want), "dx")

    def weight_grad(self, out="f32", accumulate=False):
        import torch

        from paper_2609_00993_amd import moepd as M

        m, n = 2 * self.I, self.H
        a, b = _strided(self.gu, self.dtype, m + self.pad), _strided(self.x, self.dtype, n + self.pad)
        old = _values(self.rng, (self.G, m, n), out) if accumulate else np.full((self.G, m, n), np.nan)
        dw = _dev(old, out)
        st, need = M.moe_ffn_weight_workspace(self.rows, self.G, m, n)
        M.check(st)
        assert 0 <= need <= 1 << 27
        ws = torch.full((need + 16,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN if read
        torch.cuda.synchronize()
        M.check(M.moe_ffn_weight_grad(a, m + self.pad, b, n + self.pad, self.rows, self.G, self.d_off, m, n,
                                      _code(self.dtype), dw, _code(out), accumulate, ws if need else None, need, self.stream))
        torch.cuda.synchronize()
        assert (ws[need:] == 0xFF).all()
        want, S = F.outer(self.gu, self.x, self.spans)
        K = max(hi - lo for lo, hi in self.spans)
        tol = (K + 8) * 2 * U * S
        if accumulate:
            want = want + old
            tol = tol + 2 * U * (np.abs(old) + S)
        _close(_host(dw), want, tol + _step(out) * np.abs(want), "dw")

    def everything(self):
        self.gate_up()
        self.down("bf16" if self.dtype == "bf16" else "f32")
        self.down_backward()
        self.gate_up_backward("bf16" if self.dtype == "bf16" else "f32")
        self.weight_grad()


SHAPES = [
    (1, 8, 8), (1, 512, 256), (2, 72, 40), (31, 64, 64), (33, 264, 136), (64, 200, 520), (97, 128, 128), (129, 320, 264),
    (160, 72, 256), (161, 136, 72), (300, 256, 128), (511, 1032, 8), (7, 8, 1032),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,H,I", SHAPES)
def test_one_group(rows, H, I, dtype):
    Block(rows, H, I, dtype=dtype, seed=rows + H + I).everything()


def _spread(rows, groups, seed, first=0):
    cuts = np.sort(np.random.default_rng(seed).integers(first, rows + 1, groups - 1))
    return [first, *cuts.tolist(), rows]


GROUPED = {
    "empty-first": (90, [0, 0, 40, 40, 90]),
    "none-at-the-ends": (120, [17, 50, 50, 101]),
    "all-empty": (40, [13, 13, 13]),
    "one-row-each": (70, list(range(71))),
    "many": (700, _spread(700, 150, 3)),
    "uneven": (900, [0, 1, 2, 800, 801, 866, 900]),
    "past-the-rows": (60, [-5, 20, 44, 99]),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(GROUPED))
def test_groups(name, dtype):
    rows, offsets = GROUPED[name]
    Block(rows, 136, 72, offsets, dtype=dtype, seed=len(name)).everything()


@pytest.mark.parametrize("pad", [8, 120])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(dtype, pad):
    b = Block(75, 88, 48, [3, 30, 75], dtype=dtype, pad=pad, seed=pad)
    b.gate_up()
    b.down("f32", pad)
    b.down_backward()
    b.gate_up_backward("f32", pad)
    b.weight_grad()


@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_outputs_and_options(out):
    b = Block(130, 264, 72, [0, 60, 60, 130], seed=4)
    b.gate_up(keep=False)
    b.down(out)
    b.down_backward(keep_h=False)
    b.gate_up_backward(out)
    b.weight_grad(out, accumulate=False)
    b.weight_grad(out, accumulate=True)


@pytest.mark.parametrize("rows,H,I,offsets", [
    (2000, 64, 40, None), (3000, 136, 72, [0, 1000, 1000, 3000]), (5001, 8, 8, None), (1300, 256, 264, [0, 1299, 1300]),
    (2600, 520, 128, [0, 700, 1300, 2600])])
def test_long_groups(rows, H, I, offsets):
    b = Block(rows, H, I, offsets, seed=rows)
    b.everything()
    b.weight_grad("bf16", accumulate=True)


def test_accumulate_float32():
    b = Block(50, 72, 40, [0, 0, 50], dtype="f32", seed=1)
    b.weight_grad("f32", accumulate=True)


def test_nan_stays_in_its_row_and_group():
    """A NaN in one row of x reaches that row's results and its group's weight gradient alone."""
    import torch

    from paper_2609_00993_amd import moepd as M

    b = Block(100, 72, 40, [0, 33, 66, 100], seed=9)
    b.x[40, 5] = np.nan
    x, w = _strided(b.x, "bf16", 72), _dev(b.w_gu, "bf16")
    h, gu = b.empty(100, 40), b.empty(100, 80)
    M.check(M.moe_ffn_gate_up(x, 0, 100, w, 3, b.d_off, 72, 40, M.MOE_DTYPE_BF16, gu, h, b.stream))
    dw = torch.zeros((3, 80, 72), device="cuda")
    a = _strided(b.gu, "bf16", 80)
    torch.cuda.synchronize()
    M.check(M.moe_ffn_weight_grad(a, 0, x, 0, 100, 3, b.d_off, 80, 72, M.MOE_DTYPE_BF16, dw, M.MOE_DTYPE_F32, False, None, 0,
                                  b.stream))
    torch.cuda.synchronize()
    bad = np.isnan(_host(h)).any(axis=1)
    assert bad[40] and bad.sum() == 1
    d = np.isnan(_host(dw))
    assert d[1, :, 5].all() and not d[0].any() and not d[2].any() and d.sum() == 80


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_gates(dtype):
    """Gates of large magnitude, infinite ones among them: no NaN from the activation or its slope."""
    import torch

    from paper_2609_00993_amd import moepd as M

    I = H = 8
    g = np.array([[0.0, -0.0, 20.0, -20.0, 87.0, -87.0, 300.0, -300.0], [1e30, -1e30, np.inf, 1.0, -1.28, -1.2, 3e38, -3e38]])
    rows = 2
    gu = np.concatenate([g, np.full((rows, I), 2.0)], axis=1)
    b = Block(rows, H, I, dtype=dtype)
    b.gu = _host(_dev(gu, dtype))
    b.w_dn = np.eye(8)[None]
    b.dy = np.full((rows, H), 0.5)
    d_dy, d_gu, w = _dev(b.dy, dtype), _dev(b.gu, dtype), _dev(b.w_dn, dtype)
    d, h = b.empty(rows, 2 * I), b.empty(rows, I)
    torch.cuda.synchronize()
    M.check(M.moe_ffn_down_backward(d_dy, 0, rows, w, d_gu, 1, None, H, I, _code(dtype), d, h, b.stream))
    torch.cuda.synchronize()
    g = b.gu[:, :I]
    with np.errstate(invalid="ignore"):
        s = F.sigmoid(g)
        rest = np.where(np.abs(g) > 256, 0.0, g * F.sigmoid(-g))
        want = np.concatenate([0.5 * 2.0 * s * (1 + rest), 0.5 * np.where(g < -256, 0.0, g * s)], axis=1)
        hw = np.where(g < -256, 0.0, g * s) * 2.0
    got = _host(d)
    fin = np.isfinite(want)
    assert (got[~fin] == want[~fin]).all()
    tol = (64 * U + _step(dtype)) * np.maximum(np.abs(want), 1e-30) + 64 * U
    assert (np.abs(got - np.where(fin, want, got)) <= tol)[fin].all()
    hh = _host(h)
    top = 3.3895e38 if dtype == "bf16" else 3.4028e38  # twice the largest gates pass the type's range
    inside = np.isfinite(hw) & (np.abs(hw) < top)
    assert (np.abs(hh - hw)[inside] <= ((16 * U + _step(dtype)) * np.abs(hw) + 1e-30)[inside]).all()
    assert np.isinf(hh[~inside]).all()


def test_same_bits_again_and_captured():
    """Two runs, and every replay of a captured run of the block and its gradients, give the same bits."""
    import torch

    from paper_2609_00993_amd import moepd as M

    rows, H, I, G = 700, 136, 72, 3
    b = Block(rows, H, I, [0, 300, 301, 700], seed=5)
    s = b.stream
    x, dy = _dev(b.x, "bf16"), _dev(b.dy, "bf16")
    w1, w2 = _dev(b.w_gu, "bf16"), _dev(b.w_dn, "bf16")
    gu, h, y, d, dx = (b.empty(rows, c) for c in (2 * I, I, H, 2 * I, H))
    dw1 = torch.zeros((G, 2 * I, H), device="cuda")
    dw2 = torch.zeros((1, H, I), device="cuda")
    st, need = M.moe_ffn_weight_workspace(rows, 1, H, I)
    M.check(st)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    bf, f32 = M.MOE_DTYPE_BF16, M.MOE_DTYPE_F32

    def go():
        M.check(M.moe_ffn_gate_up(x, 0, rows, w1, G, b.d_off, H, I, bf, gu, h, s))
        M.check(M.moe_ffn_down(h, rows, w2, G, b.d_off, H, I, bf, y, bf, 0, s))
        M.check(M.moe_ffn_down_backward(dy, 0, rows, w2, gu, G, b.d_off, H, I, bf, d, h, s))
        M.check(M.moe_ffn_gate_up_backward(d, rows, w1, G, b.d_off, H, I, bf, dx, bf, 0, s))
        M.check(M.moe_ffn_weight_grad(d, 0, x, 0, rows, G, b.d_off, 2 * I, H, bf, dw1, f32, False, ws, need, s))
        M.check(M.moe_ffn_weight_grad(dy, 0, h, 0, rows, 1, None, H, I, bf, dw2, f32, False, ws, need, s))

    outs = (gu, h, y, d, dx, dw1, dw2)
    go()
    torch.cuda.synchronize()
    first = [o.clone() for o in outs]
    go()
    torch.cuda.synchronize()
    same = lambda: all(torch.equal(a.view(torch.uint8), o.view(torch.uint8)) for a, o in zip(first, outs))  # noqa: E731
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        graph.capture_begin()
        go()
        graph.capture_end()
    for _ in range(3):
        for o in outs:
            o.fill_(0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same()


def test_rows_past_32_bit_offsets():
    """Rows whose bytes pass 4 GiB, in groups of which the last starts past them."""
    import torch

    from paper_2609_00993_amd import moepd as M

    rows, stride, H, I = 140_000, 1 << 14, 64, 32  # 4.6 GB of x
    offsets = [0, 70_000, 139_900, 140_000]
    x = torch.zeros((rows, stride), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x[:, :H] = torch.randn((rows, H), generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn((3, 2 * I, H), generator=g, device="cuda") / 8).to(torch.bfloat16)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    a = torch.randn((rows, 2 * I), generator=g, device="cuda").to(torch.bfloat16)
    h = torch.empty((rows, I), dtype=torch.bfloat16, device="cuda")
    gu = torch.empty((rows, 2 * I), dtype=torch.bfloat16, device="cuda")
    dw = torch.empty((3, 2 * I, H), device="cuda")
    st, need = M.moe_ffn_weight_workspace(rows, 3, 2 * I, H)
    M.check(st)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    M.check(M.moe_ffn_gate_up(x, stride, rows, w, 3, off, H, I, M.MOE_DTYPE_BF16, gu, h, s))
    M.check(M.moe_ffn_weight_grad(a, 0, x, stride, rows, 3, off, 2 * I, H, M.MOE_DTYPE_BF16, dw, M.MOE_DTYPE_F32, False, ws,
                                  need, s))
    torch.cuda.synchronize()
    for e, (lo, hi) in enumerate(zip(offsets[:-1], offsets[1:])):
        xs, ws_ = x[lo:hi, :H].double(), w[e].double()
        want = xs @ ws_.t()
        tol = (H + 8) * 2 * U * (xs.abs() @ ws_.abs().t()) + 2.0 ** -8 * want.abs()
        assert ((gu[lo:hi].double() - want).abs() <= tol).all(), e
        A = a[lo:hi].double()
        want = A.t() @ xs
        tol = (hi - lo + 8) * 2 * U * (A.abs().t() @ xs.abs()) + 2.0 ** -24 * want.abs()
        assert ((dw[e].double() - want).abs() <= tol).all(), e


def _activation(dtype, g, u, dh):
    """(dg, du, h anew) of moe_ffn_down_backward for gates, ups and dh (w_down is the identity), and those three as the type
    holds them; g, u, dh: [rows, 8]."""
    import torch

    from paper_2609_00993_amd import moepd as M

    rows, I = g.shape
    d_gu, d_dy = _dev(np.concatenate([g, u], axis=1), dtype), _dev(dh, dtype)
    w = _dev(np.eye(8)[None], dtype)
    d, h = (torch.full((rows, n), SENTINEL, dtype=_torch_type(dtype), device="cuda") for n in (2 * I, I))
    torch.cuda.synchronize()
    M.check(M.moe_ffn_down_backward(d_dy, 0, rows, w, d_gu, 1, None, 8, I, _code(dtype), d, h, torch.cuda.Stream()))
    torch.cuda.synchronize()
    d, gu = _host(d), _host(d_gu)
    return (d[:, :I], d[:, I:], _host(h)), (gu[:, :I], gu[:, I:], _host(d_dy))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slope_of_far_gates(dtype):
    """Gates whose e^-|g| is below the normal numbers, beside ups and dh that bring the results back, and ups and dh whose
    product alone passes the range: relative errors. q is within 4 u (2^x and its argument 2 u, a fused product 2 u), the reciprocal
    2 u, 1 + g (1 - s) 4 u (it does not cancel below -2), the products 3 u: 16 u, beside the type's rounding; results below the
    normal numbers 2^-126."""
    g, u, dh = np.meshgrid([-20.0, -44.0, -45.0, -49.0, -49.25, -60.0, -80.0, -87.0, -88.0, -92.0, -100.0, -104.0, -120.0, -130.0,
                            3.0, 50.0], [2.0, -1e10, 1e30, 3e-5], [0.5, -1e-5, 3e7, 1e-30])
    g, u, dh = (a.reshape(-1, 8) for a in (g, u, dh))
    (dg, du, h), (g, u, dh) = _activation(dtype, g, u, dh)
    want_g, want_u = F.swiglu_gradient(g, u, dh)
    for got, want in ((dg, want_g), (du, want_u), (h, F.swiglu(g, u))):
        assert (np.abs(want) < 1e38).all() and (np.abs(want) > 1e-30).sum() > want.size // 3
        assert (np.abs(got - want) <= (16 * U + _step(dtype)) * np.abs(want) + 2.0 ** -126).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slope_of_large_factors(dtype):
    """dh u past the range where the slope brings the result back, 0 among the slopes."""
    g = np.array([[-300.0, -1e30, -132.0, -100.0, -90.0, -60.0, -49.0, -30.0]])
    u, dh = np.full((1, 8), 1e25), np.full((1, 8), 2e20)
    (dg, du, _), (g, u, dh) = _activation(dtype, g, u, dh)
    want_g, want_u = F.swiglu_gradient(np.maximum(g, -256), u, dh)
    for got, want in ((dg, want_g), (du, want_u)):
        want = np.where(g < -131, 0.0, want)  # the slope is 0 there
        inside = np.abs(want) < 3e38
        assert inside.sum() >= 7 and (np.abs(got - want) <= (16 * U + _step(dtype)) * np.abs(want) + 2.0 ** -126)[inside].all()
        assert (np.abs(got[~inside]) >= 3e38).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_gates_take_the_limits(dtype):
    """In the forward pass (where a sum passes the range), anew, and in the gradients."""
    import torch

    from paper_2609_00993_amd import moepd as M

    inf = np.inf
    g = np.array([[-inf, inf, -inf, inf, -300.0, -3e38, 2.0, -inf]])
    u, dh = np.array([[3.0, 3.0, -1e30, -0.5, 7.0, -1.0, 4.0, 0.0]]), np.array([[1.0, 2.0, -1e5, 4.0, 1.0, 1e20, 0.5, 0.0]])
    (dg, du, h), _ = _activation(dtype, g, u, dh)
    gone = g[0] < -256
    for got in (dg, du, h):
        assert (got[0, gone] == 0).all()
    top = g[0] == inf
    assert (dg[0, top] == [6.0, -2.0]).all() and (du[0, top] == inf).all() and (h[0, top] == [inf, -inf]).all()
    assert not np.isnan(dg).any() and not np.isnan(du).any() and not np.isnan(h).any()

    x = np.array([[1e38, 2.0, 0, 0, 0, 0, 0, 0]])  # the gate's sum is 1e38 of the first column's weight, up 2
    w = np.zeros((1, 16, 8))
    w[0, :8, 0], w[0, 8:, 1] = [-100.0, 100.0, -1e38, 1.0, 0.0, -1e-38, -1.0, 1e38], 1.0
    out, gu = (torch.full((1, n), SENTINEL, dtype=_torch_type(dtype), device="cuda") for n in (8, 16))
    d_x, d_w = _dev(x, dtype), _dev(w, dtype)
    torch.cuda.synchronize()
    M.check(M.moe_ffn_gate_up(d_x, 0, 1, d_w, 1, None, 8, 8, _code(dtype), gu, out, torch.cuda.Stream()))
    torch.cuda.synchronize()
    gate, h = _host(gu)[0, :8], _host(out)[0]
    assert (gate[[0, 2]] == -inf).all() and (gate[[1, 7]] == inf).all() and (_host(gu)[0, 8:] == 2).all()
    assert (h[[0, 2, 4, 6]] == 0).all() and (h[[1, 7]] == inf).all() and not np.isnan(h).any()
