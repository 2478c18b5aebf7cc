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


def test_weight_gradient_of_no_rows():
    import torch

    from paper_2609_00993_amd import moepd as M

    s = torch.cuda.Stream()
    for offsets, groups in ((None, 1), (torch.zeros(4, dtype=torch.int32, device="cuda"), 3)):
        for accumulate in (False, True):
            dw = torch.full((groups, 24, 16), 5.0, device="cuda")
            torch.cuda.synchronize()
            M.check(M.moe_ffn_weight_grad(None, 0, None, 0, 0, groups, offsets, 24, 16, M.MOE_DTYPE_BF16, dw, M.MOE_DTYPE_F32,
                                          accumulate, None, 0, s))
            torch.cuda.synchronize()
            assert (dw == (5.0 if accumulate else 0.0)).all()


@pytest.mark.parametrize("rows", [5, 300])
@pytest.mark.parametrize("H,I", [(32768, 8192), (8184, 32768), (32760, 8192)])
def test_widest_matrices(rows, H, I):
    """H I at its limit (weights of 1 GiB a group), with and without a rest of K, in the last columns."""
    import torch

    from paper_2609_00993_amd import moepd as M
    from tests.test_gpu_ffn import U

    g = torch.Generator(device="cuda")
    g.manual_seed(rows + H)
    mk = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)  # noqa: E731
    w1, w2, x, gu = mk(1, 2 * I, H), mk(1, H, I), mk(rows, H), mk(rows, 2 * I)
    y, h, d = (torch.empty((rows, n), dtype=torch.bfloat16, device="cuda") for n in (H, I, 2 * I))
    s, bf = torch.cuda.Stream(), M.MOE_DTYPE_BF16
    dx = torch.empty((rows, H), device="cuda")
    gu_out = torch.empty_like(gu)
    torch.cuda.synchronize()
    M.check(M.moe_ffn_gate_up(x, 0, rows, w1, 1, None, H, I, bf, gu_out, h, s))
    M.check(M.moe_ffn_down(gu[:, :I].contiguous(), rows, w2, 1, None, H, I, bf, y, bf, 0, s))
    M.check(M.moe_ffn_gate_up_backward(gu, rows, w1, 1, None, H, I, bf, dx, M.MOE_DTYPE_F32, 0, s))
    M.check(M.moe_ffn_down_backward(x, 0, rows, w2, gu, 1, None, H, I, bf, d, None, s))
    torch.cuda.synchronize()

    def close(got, a, b, K, step):
        a, b = a.double(), b.double()
        want = a @ b
        tol = (K + 8) * 2 * U * (a.abs() @ b.abs()) + step * want.abs()
        assert ((got.double() - want).abs() <= tol).all()

    close(gu_out[:, -16:], x, w1[0, -16:].t(), H, 2.0 ** -8)
    close(gu_out[:, I - 8:I + 8], x, w1[0, I - 8:I + 8].t(), H, 2.0 ** -8)
    close(y[:, -16:], gu[:, :I], w2[0, -16:].t(), I, 2.0 ** -8)
    close(dx[:, -16:], gu, w1[0, :, -16:], 2 * I, U)
    dh = x.double() @ w2[0, :, -8:].double()
    gate, up = gu[:, I - 8:I].double(), gu[:, -8:].double()
    silu = gate * torch.sigmoid(gate)
    tol = (H + 8) * 2 * U * (x.abs().double() @ w2[0, :, -8:].abs().double()) * silu.abs() + (2.0 ** -8 + 16 * U) * (dh * silu).abs()
    assert ((d[:, -8:].double() - dh * silu).abs() <= tol).all()


def test_two_streams_at_once():
    """Calls on different streams, with buffers of their own, do not disturb each other."""
    import torch

    from paper_2609_00993_amd import moepd as M

    rows, H, I, bf, f32 = 4000, 264, 136, M.MOE_DTYPE_BF16, M.MOE_DTYPE_F32
    sets = []
    for seed in (1, 2):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        mk = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)  # noqa: E731
        st, need = M.moe_ffn_weight_workspace(rows, 1, 2 * I, H)
        M.check(st)
        assert need > 0
        sets.append(dict(x=mk(rows, H), w=mk(1, 2 * I, H), gu=mk(rows, 2 * I), h=mk(rows, I), dw=torch.zeros((2 * I, H), device="cuda"),
                         ws=torch.empty(need, dtype=torch.uint8, device="cuda"), need=need, s=torch.cuda.Stream()))

    def go(c):
        M.check(M.moe_ffn_gate_up(c["x"], 0, rows, c["w"], 1, None, H, I, bf, c["gu"], c["h"], c["s"]))
        M.check(M.moe_ffn_weight_grad(c["gu"], 0, c["x"], 0, rows, 1, None, 2 * I, H, bf, c["dw"], f32, False, c["ws"], c["need"],
                                      c["s"]))

    alone = []
    for c in sets:
        torch.cuda.synchronize()
        go(c)
        torch.cuda.synchronize()
        alone.append([c[k].clone() for k in ("gu", "h", "dw")])
    for _ in range(5):
        for c in sets * 3:
            go(c)
    torch.cuda.synchronize()
    for c, want in zip(sets, alone):
        for k, w in zip(("gu", "h", "dw"), want):
            assert torch.equal(c[k], w)
