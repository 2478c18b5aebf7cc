"""Operands whose products sum exactly in float32, in any order: whole numbers from -2 to 2, so that K terms stay below
2^24 for K up to 2^22 and a float32 result is the sum itself, a bf16 result its nearest. One term too many or too few
moves the sum by 1 to 4, which shows in float32 always and in bf16 in many of a matrix's values (a sum of K terms is some 2
sqrt(K), its bf16 step 2^-7 of that: 4 at most for K up to 65536)."""

MOST = 2


def whole(generator, *shape):
    """A bf16 tensor on the generator's device."""
    import torch

    return torch.randint(-MOST, MOST + 1, shape, generator=generator, device=generator.device).to(torch.bfloat16)


def product(a, b, dtype):
    """a b^T, rounded once."""
    import torch

    want = a.to(torch.float64) @ b.to(torch.float64).t()
    assert want.numel() == 0 or want.abs().max() < 2 ** 24
    return want.to(torch.float32).to(dtype)
