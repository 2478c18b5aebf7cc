"""The MX FP4 layer (MOE_DTYPE_FP4 contexts) through the C ABI against the float64
oracles: routing and layout exact, x_perm exact, h and y within the bounds of
tests/test_gpu_mx4.py (y on the GPU's own h), the combine on the GPU's own y;
empty batches, skewed routing, both phases at once, a captured decode layer."""

import numpy as np
import pytest

import oracle
from oracle import mx4 as X
from tests.gpu_util import read_dev
from tests.test_gpu_mx4 import U, _gated, _sum_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


class Layer:
    def __init__(self, E, e0, E_loc, k, H, I, T_P, T_D, seed, skew=0.0, d_priority_us=0):
        import torch

        from paper_2609_00993_amd import moepd as M

        self.M, self.torch, self.dims = M, torch, (E, e0, E_loc, k, H, I)
        rng = np.random.default_rng(seed)
        self.w, self.held = [], []
        for n, K in ((E_loc * 2 * I, H), (E_loc * H, I)):
            codes = rng.integers(0, 16, (n, K), dtype=np.uint8)
            base = 127 - int(round(np.log2(3.0 * np.sqrt(K))))
            scales = rng.integers(base - 1, base + 2, (n, K // 32), dtype=np.uint8)
            self.w.append(X.dequantize(codes, scales))
            self.held += [torch.from_numpy(b).cuda() for b in X.hold(codes, scales)]
        self.T = (T_P, T_D)
        bias = -skew * np.log(np.arange(1, E + 1))
        self.logits = [(rng.standard_normal((T, E)) + bias).astype(np.float32) for T in self.T]
        x = [rng.standard_normal((T, H)).astype(np.float32) for T in self.T]
        self.x = [(v.view(np.uint32) >> 16 << 16).view(np.float32) for v in x]
        self.dx = [torch.from_numpy(v).cuda().to(torch.bfloat16) for v in self.x]
        self.dl = [torch.from_numpy(v).cuda() for v in self.logits]
        self.out = [torch.zeros((T, H), device="cuda") for T in self.T]
        torch.cuda.synchronize()
        cfg = M.make_config(E, e0, E_loc, k, H, I, M.MOE_DTYPE_FP4, T_P + 3, T_D, d_priority_us=d_priority_us)
        st, self.ctx = M.moe_ctx_create(cfg, self.held[0], self.held[2], self.held[1], self.held[3])
        M.check(st, "create")
        self.s = [torch.cuda.Stream(), torch.cuda.Stream()]

    def run(self, ph):
        self.M.layer(self.ctx, ph, self.dl[ph], self.T[ph], self.dx[ph], self.out[ph], self.s[ph])

    def close(self):
        self.M.check(self.M.moe_ctx_destroy(self.ctx))

    def check(self, ph):
        M = self.M
        E, e0, E_loc, k, H, I = self.dims
        self.torch.cuda.synchronize()
        st, v = M.moe_phase_view(self.ctx, ph)
        M.check(st)
        T = self.T[ph]
        idx, w = oracle.route(self.logits[ph].astype(np.float64), k)
        counts, offsets, row_of_slot, token_of_row = oracle.layout(oracle.local_map(idx, e0, E_loc), E_loc)
        R = int(offsets[-1])
        assert np.array_equal(read_dev(v.topk_idx, (T, k), np.int32), idx)
        assert np.array_equal(read_dev(v.offsets, (E_loc + 1,), np.int32), offsets)
        assert np.array_equal(read_dev(v.token_of_row, (R,), np.int32), token_of_row)
        out = self.out[ph].cpu().numpy()
        if R == 0:
            assert not out.any()
            return

        def matrix(codes, scales, K):
            n = -(-R // 32) * 32
            return X.release(read_dev(codes, (n * K // 2,), np.uint8), read_dev(scales, (n * K // 32,), np.uint8), R, K)

        xc, xs = matrix(v.x_perm, v.x_perm_scales, H)
        wc, ws = X.quantize(self.x[ph][token_of_row])
        assert np.array_equal(xs, ws) and ((xc == wc) | ((xc & 7) + (wc & 7) == 0)).all()
        g, mag = X.product(X.dequantize(xc, xs), self.w[0], offsets, 2 * I)
        h, bound = _gated(g, _sum_bound(mag, H), I)
        hc, hs = matrix(v.h, v.h_scales, I)
        scale = np.repeat(np.exp2(hs.astype(np.float64) - 127), 32, axis=1)
        hq = X.dequantize(hc, hs)
        lo, hi = (X.e2m1_decode(X.e2m1_encode(b / scale)) * scale for b in (h - bound, h + bound))
        assert (hq >= lo).all() and (hq <= hi).all()
        # the block's exponent is that of its largest value, within the bound
        amax = np.abs(h).reshape(R, -1, 32).max(axis=2)
        top = (np.abs(h) + bound).reshape(R, -1, 32).max(axis=2)
        assert (np.exp2(hs.astype(np.float64) - 127) * 4 <= top * (1 + 1e-12)).all()
        assert (np.exp2(hs.astype(np.float64) - 127) * 8 >= amax * (1 - 1e-3) - 1e-30).all()
        y, ymag = X.product(hq, self.w[1], offsets, H)
        got = read_dev(v.y, (R, H), np.float32).astype(np.float64)
        assert (np.abs(got - y) <= _sum_bound(ymag, I) + 1e-37).all()
        want = oracle.combine(got, w, row_of_slot, T, H)
        each = oracle.combine(np.abs(got), w, row_of_slot, T, H)
        assert (np.abs(out - want) <= (2 * k + 40) * U * each + 1e-30).all()  # weights 2e-6, k float32 sums
        none = (row_of_slot < 0).all(axis=1)
        assert not out[none].any()


SHAPES = {
    "mid": dict(E=16, e0=0, E_loc=16, k=4, H=512, I=256, T_P=700, T_D=13),
    "share": dict(E=40, e0=8, E_loc=16, k=3, H=256, I=512, T_P=1501, T_D=5),
    "skewed": dict(E=24, e0=0, E_loc=6, k=2, H=768, I=256, T_P=900, T_D=40, skew=1.5),
    "one-token": dict(E=300, e0=100, E_loc=70, k=8, H=256, I=256, T_P=1, T_D=1),
    "empty": dict(E=8, e0=2, E_loc=4, k=1, H=256, I=256, T_P=0, T_D=0),
    "limits": dict(E=1024, e0=512, E_loc=256, k=16, H=256, I=256, T_P=3000, T_D=64),
}


@pytest.mark.parametrize("name", list(SHAPES))
def test_fp4_layer(name):
    g = Layer(**SHAPES[name], seed=len(name))
    try:
        for ph in (0, 1):
            g.run(ph)
            g.check(ph)
    finally:
        g.close()


def test_both_phases_at_once_give_their_own_bits():
    g = Layer(E=32, e0=0, E_loc=32, k=4, H=512, I=512, T_P=2048, T_D=64, seed=3, d_priority_us=500)
    try:
        alone = []
        for ph in (0, 1):
            g.run(ph)
            g.torch.cuda.synchronize()
            alone.append(g.out[ph].clone())
        for _ in range(3):
            for ph in (0, 1):
                g.out[ph].fill_(-1.0)
            g.torch.cuda.synchronize()
            g.run(0)
            g.run(1)
            g.torch.cuda.synchronize()
            assert all(g.torch.equal(g.out[ph], alone[ph]) for ph in (0, 1))
    finally:
        g.close()


def test_a_captured_decode_layer_replays():
    g = Layer(E=32, e0=0, E_loc=32, k=4, H=512, I=256, T_P=64, T_D=37, seed=4)
    torch = g.torch
    try:
        g.run(1)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=g.s[1]):
            g.run(1)
        rng = np.random.default_rng(9)
        for _ in range(3):
            g.logits[1] = rng.standard_normal(g.logits[1].shape).astype(np.float32)
            g.dl[1].copy_(torch.from_numpy(g.logits[1]))
            torch.cuda.synchronize()
            graph.replay()
            g.check(1)
    finally:
        g.close()


def test_create_checks_fp4_configs():
    from paper_2609_00993_amd import moepd as M

    def create(H=256, I=256, w=(0x1000, 0x2000, 0x3000, 0x4000)):
        st, ctx = M.moe_ctx_create(M.make_config(8, 0, 8, 2, H, I, M.MOE_DTYPE_FP4, 4, 4), *w)
        if ctx:
            M.moe_ctx_destroy(ctx)
        return st

    assert create(H=384) == M.MOE_ERR_INVALID_ARG and create(I=128) == M.MOE_ERR_INVALID_ARG
    assert create(w=(0x1000, 0x2000, None, 0x4000)) == M.MOE_ERR_INVALID_ARG
    assert create(w=(0x1008, 0x2000, 0x3000, 0x4000)) == M.MOE_ERR_INVALID_ARG
    assert create(w=(0x1000, 0x2000, 0x3000, 0x4004)) == M.MOE_ERR_INVALID_ARG
    assert create() == M.MOE_OK


def test_the_example_evens_its_router():
    from examples import fp4_router_training

    history = fp4_router_training.main(["--tokens", "512", "--steps", "5"])
    assert len(history) == 5 and history[0] > 2.0 and history[-1] < 1.3
