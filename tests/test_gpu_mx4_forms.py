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
