"""The exact comparisons of tests/test_gpu_ffn_exact.py flag what the tests are there for: one term of a sum left out or
taken twice, at every length that they use (no GPU)."""

import pytest
import torch

from tests.exact_sums import product, whole


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", [8, 72, 2312, 7001, 32768, 65536, 70000])
def test_one_term_shows(K, dtype):
    g = torch.Generator().manual_seed(K)
    a, b = whole(g, 24, K), whole(g, 24, K)
    want = product(a, b, dtype)
    for at in {0, 7, K // 2, K - 8, K - 1}:
        for times in (0, 2):
            wrong = a.clone()
            wrong[:, at] *= times
            off = (product(wrong, b, dtype) != want).sum().item()
            assert off > 24 * 24 // 20, (at, times, off)


def test_sums_are_exact_in_any_order():
    g = torch.Generator().manual_seed(1)
    a, b = whole(g, 4, 70000).float(), whole(g, 4, 70000).float()
    want = (a.double() @ b.double().t())
    for order in (torch.arange(70000), torch.randperm(70000, generator=g)):
        s = torch.zeros(4, 4)
        for c in order.split(700):
            s += a[:, c] @ b[:, c].t()
        assert (s.double() == want).all()
