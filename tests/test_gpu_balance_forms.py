"""The balance loss and gradient on the GPU in each form of their kernels, by the bounds of
tests/test_gpu_balance.py."""

import numpy as np
import pytest

from tests.test_gpu_balance import Run, _check, _logits, _need_gpu, _topk  # noqa: F401

pytestmark = pytest.mark.gpu

# One launch does it all up to 256 tokens x 64 experts of one sequence: the last shape of
# each count of experts to a lane that takes it, and the first that does not.
EDGES = [(256, 64, 4), (257, 64, 4), (128, 128, 8), (129, 127, 8), (85, 192, 2), (86, 192, 2), (64, 253, 8), (65, 256, 8),
         (51, 300, 16), (52, 300, 16), (32, 512, 8), (33, 511, 8), (28, 570, 1), (29, 570, 1), (16, 1000, 3), (16, 1024, 16),
         (17, 1024, 16), (1, 513, 4), (1, 1024, 8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,E,k", EDGES)
def test_one_launch_and_its_edges(T, E, k, dtype):
    rng = np.random.default_rng(T * 1031 + E)
    logits = _logits(rng, T, E, dtype)
    idx = _topk(logits, k)
    _check(logits, idx, None, None, 1, 0.3, Run(logits, idx, dtype=dtype), dtype)
    # one sequence that leaves tokens out at both ends, some masked
    seq = np.array([T // 8, T - T // 5], np.int32)
    mask = (rng.random(T) < 0.7).astype(np.uint8)
    _check(logits, idx, mask, seq, 1, 0.3, Run(logits, idx, mask, seq, 1, dtype=dtype, stride=E + 5), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E", [129, 250, 300, 513, 1023])
def test_padded_rows_accumulate_and_in_place_at_four_experts_to_a_lane(E, dtype):
    rng = np.random.default_rng(E)
    T = 61
    logits = _logits(rng, T, E, dtype)
    idx = _topk(logits, 6)
    seq = np.array([1, 20, 20, 55], np.int32)
    mask = (rng.random(T) < 0.8).astype(np.uint8)
    base = _logits(rng, T, E, dtype, 1e-3)
    grad = np.array([-2.5], np.float32)
    for stride in (E, E + 1, E + 4 - E % 4, E + 6):
        for kw in (dict(grad=grad), dict(grad=grad, base=base), dict(grad=grad, inplace=True)):
            _check(logits, idx, mask, seq, 3, 0.3, Run(logits, idx, mask, seq, 3, stride=stride, dtype=dtype, **kw), dtype, -2.5,
                   kw.get("base"))


@pytest.mark.parametrize("T,E,S,long", [(3000, 100, 100, 1), (2600, 256, 60, 1), (5000, 64, 1100, 1), (4000, 200, 1500, 2),
                                        (700, 33, 5000, 1)])
def test_long_sequences_among_single_tokens(T, E, S, long):
    """`long` sequences hold nearly all the tokens, between runs of sequences of one token and of none."""
    rng = np.random.default_rng(S)
    logits = _logits(rng, T, E)
    idx = _topk(logits, 3)
    sizes = rng.integers(0, 2, S)
    at = rng.choice(S, long, replace=False)
    sizes[at] = (T - sizes.sum() + sizes[at].sum()) // long if sizes.sum() < T else 0
    ends = np.minimum(np.cumsum(sizes), T)
    seq = np.concatenate([[0], ends]).astype(np.int32)
    _check(logits, idx, None, seq, S, 0.3, Run(logits, idx, None, seq, S))


@pytest.mark.parametrize("T,E,S", [(40, 60, 1), (3000, 130, 1), (3000, 130, 9), (900, 200, 1200)])
def test_a_captured_loss_and_gradient_replay(T, E, S):
    """The one-launch form, the join that ends with a ticket and the join of its own for many sequences,
    captured once: replays on new logits, with eager calls between, give the eager bits."""
    import torch

    from paper_2609_00993_amd import moepd as M

    rng = np.random.default_rng(T + S)
    k, s = 4, torch.cuda.Stream()
    seq = None
    if S > 1:
        seq = torch.from_numpy(np.concatenate([[0], np.sort(rng.integers(0, T + 1, S - 1)), [T]]).astype(np.int32)).cuda()
    x, idx = torch.zeros((T, E), device="cuda"), torch.zeros((T, k), dtype=torch.int32, device="cuda")
    st, n = M.moe_balance_workspace(T, E, S)
    M.check(st)

    def outputs():
        return [torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(1, device="cuda"),
                torch.zeros((S, E), dtype=torch.int32, device="cuda"), torch.zeros(S + 1, dtype=torch.int32, device="cuda"),
                torch.zeros((T, E), device="cuda")]

    def call(ws, loss, counts, live, d):
        M.check(M.moe_balance_loss(x, M.MOE_DTYPE_F32, 0, idx, None, seq, S, T, E, k, 0.3, loss, counts, live, ws, n, s))
        M.check(M.moe_balance_loss_backward(x, M.MOE_DTYPE_F32, 0, None, seq, S, T, E, k, 0.3, counts, live, None, d, 0, False, s))

    mine, eager = outputs(), outputs()
    torch.cuda.synchronize()
    call(*eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(*mine)
    for _ in range(4):
        logits = _logits(rng, T, E)
        x.copy_(torch.from_numpy(logits))
        idx.copy_(torch.from_numpy(_topk(logits, k)))
        for t in mine:
            t.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        call(*eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(mine[1:], eager[1:]))
        assert float(mine[1]) > 0 and int(mine[3][S]) > 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_whose_offsets_pass_32_bits(dtype):
    """Logits and gradients 2^20 elements and more a row: the last rows lie past 2^32 elements."""
    import torch

    from paper_2609_00993_amd import moepd as M

    rng = np.random.default_rng(12)
    T, E, k, stride = 4200, 130, 4, (1 << 20) + 3
    logits = _logits(rng, T, E, dtype)
    idx = _topk(logits, k)
    s, t = torch.cuda.Stream(), torch.float32 if dtype == "f32" else torch.bfloat16
    code = M.MOE_DTYPE_F32 if dtype == "f32" else M.MOE_DTYPE_BF16
    assert (T - 1) * stride > 1 << 32
    x, d = (torch.empty(T * stride, dtype=t, device="cuda").view(T, stride) for _ in range(2))
    x[:, :E] = torch.from_numpy(logits).cuda().to(t)
    x[:, E], d[:, E] = float("nan"), float("nan")
    i = torch.from_numpy(idx).cuda()
    st, n = M.moe_balance_workspace(T, E, 1)
    M.check(st)
    ws, loss = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(1, device="cuda")
    counts, live = torch.zeros((1, E), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    M.check(M.moe_balance_loss(x, code, stride, i, None, None, 1, T, E, k, 0.3, loss, counts, live, ws, n, s))
    M.check(M.moe_balance_loss_backward(x, code, stride, None, None, 1, T, E, k, 0.3, counts, live, None, d, stride, False, s))
    torch.cuda.synchronize()

    class Got:
        pass

    got = Got()
    got.loss, got.counts, got.live = float(loss), counts.cpu().numpy(), live.cpu().numpy()
    got.d = d[:, :E].float().cpu().numpy().astype(np.float64)
    assert bool(torch.isnan(d[:, E]).all())
    _check(logits, idx, None, None, 1, 0.3, got, dtype)
