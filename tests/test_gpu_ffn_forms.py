"""The feed-forward block's tiles in every form, against the float64 oracle with the tolerances of
tests/test_gpu_ffn.py. tests/test_ffn_form.py holds, without a GPU, that the cases reach the forms that
they name."""

import numpy as np
import pytest

from tests.test_gpu_ffn import Block

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _ragged(groups, most, seed):
    """Offsets of groups of 0 to `most` rows, every height in blocks of 32 among them."""
    n = np.random.default_rng(seed).integers(0, most + 1, groups)
    n[:8] = [0, 1, 32, 33, 64, 96, 128, most]
    return [0, *np.cumsum(n).tolist()]


# name: the tiles that at least one of the products takes; offsets (or rows of one group), H, I
CASES = {
    # up to eight rows: one to many blocks of K to a wave, shared evenly among the eight waves and not
    "few8-token": (1, 2120, 1096),
    "few8-one-block": (8, 64, 40),
    "few8-eight-blocks": (5, 512, 520),
    "few8-groups": ([0, 3, 3, 8], 1032, 136),
    # up to 32 rows a tile
    "few32-short": (33, 8, 8),
    "few32-long": (70, 2120, 1096),
    "few32-groups": ([0, 31, 31, 96, 97], 840, 392),
    # heights of one to five blocks, K of one to five slices with and without a rest
    "mid-1-2": (_ragged(100, 160, 1), 8, 72),
    "mid-3-1": (_ragged(100, 160, 2), 136, 8),
    "mid-4-5": (_ragged(100, 160, 3), 200, 264),
    "mid-5-4": (_ragged(100, 160, 4), 264, 256),
    "mid-many-groups": (_ragged(300, 40, 5), 72, 136),
    "mid-low": (_ragged(40, 128, 6), 520, 136),
    # 256 rows, one to six slices, groups of one row beside large ones
    "wide-1": (6000, 64, 2312),
    "wide-3": ([0, 2500, 2501, 6000], 136, 2312),
    "wide-halves": ([0, 2600, 5161, 5420, 6000], 136, 2312),  # rests of one and two blocks, shared with a full tile
    "wide-6": (6001, 328, 2312),
    "wide-2-3": (6000, 2312, 72),
    "wide-4-7": ([7, 3000, 5999], 2312, 200),
}


def rows_of(case):
    return case[0] if isinstance(case[0], int) else case[0][-1]


@pytest.mark.parametrize("name", list(CASES))
def test_every_form(name):
    where, H, I = CASES[name]
    offsets = None if isinstance(where, int) else where
    b = Block(rows_of(CASES[name]), H, I, offsets, seed=len(name) + H)
    b.everything()
    if not name.startswith("mid"):
        b.down("f32")
        b.gate_up_backward("f32")


WEIGHTS = {  # rows, groups, m, n of w_gate_up's gradient: one part and several
    "one-part": (300, 3, 272, 264),
    "parts": (9000, 1, 272, 264),
    "parts-groups": (6000, 2, 144, 520),
    "parts-uneven": (7001, 2, 16, 8),
}


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("name", list(WEIGHTS))
def test_weight_gradients(name, out, accumulate):
    rows, groups, m, n = WEIGHTS[name]
    cut = [0, 1, rows] if groups == 2 else np.linspace(0, rows, groups + 1).astype(int).tolist()
    Block(rows, n, m // 2, None if groups == 1 else cut, seed=rows).weight_grad(out, accumulate)


def test_accumulating_skips_groups_without_rows():
    """Their sums stay as they are, bit for bit."""
    import torch

    from paper_2609_00993_amd import moepd as M

    m, n = 48, 40
    dw = torch.full((3, m, n), float("nan"), device="cuda")
    dw[1] = 0
    a, b = torch.ones((5, m), device="cuda", dtype=torch.bfloat16), torch.ones((5, n), device="cuda", dtype=torch.bfloat16)
    off = torch.tensor([0, 0, 5, 5], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    M.check(M.moe_ffn_weight_grad(a, 0, b, 0, 5, 3, off, m, n, M.MOE_DTYPE_BF16, dw, M.MOE_DTYPE_F32, True, None, 0,
                                  torch.cuda.Stream()))
    torch.cuda.synchronize()
    assert torch.isnan(dw[0]).all() and torch.isnan(dw[2]).all() and (dw[1] == 5).all()
