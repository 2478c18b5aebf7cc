"""MX FP4 products on the GPU in each form of their tiles, and where sizes, gates and
scales are extreme.  Bounds are those of tests/test_gpu_mx4.py."""

import numpy as np
import pytest

from oracle import mx4 as X
from tests.test_gpu_mx4 import _matrix, _need_gpu, _sum_bound, env  # noqa: F401

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
