"""The operators of a training step together, as a program uses them (examples/expert_training.py): routing
and layout from a context, tokens into expert order, the experts' blocks, the combine, and every gradient
back to the gate and the experts, then AdamW.

The reference is the same layer in float64 on the bf16 weights, differentiated by torch's own autograd, with
the routing's picks as given. A gradient passes at most eight roundings to bf16 on its way (gate_up, h, y; dy,
dgate_up; drows, dx; the router's logits are float32), each at most 2^-8 of what is rounded, and the activation's slope
carries gate_up's into dgate_up with a factor of about one: 8 x 2^-8 of the gradient's 2-norm bounds their sum."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _from_device(address, shape, dtype):
    """A view's buffer as a tensor of its own."""
    import torch

    class Held:
        __cuda_array_interface__ = dict(shape=shape, typestr=dtype, data=(address, False), version=3)

    return torch.as_tensor(Held(), device="cuda").clone()


@pytest.mark.parametrize("T,E,k,H,I", [(300, 8, 2, 128, 64), (1, 8, 3, 64, 128), (777, 16, 4, 192, 320)])
def test_gradients_of_a_step(T, E, k, H, I):
    import torch

    from examples.expert_training import ExpertLayer

    s = torch.cuda.Stream()
    layer = ExpertLayer(T, E, k, H, I, s, seed=T)
    x = torch.randn((T, H), device="cuda").to(torch.bfloat16)
    c = torch.randn((T, H), device="cuda")
    torch.cuda.synchronize()
    out = layer.forward(x)
    layer.dout.copy_(c)  # the loss is sum(c out), and the balance loss
    torch.cuda.synchronize()
    layer.backward(x, balance=0.5)
    s.synchronize()
    idx = _from_device(layer.view.topk_idx, (T, k), "<i4").long()
    gate, w1, w2 = (w.double().requires_grad_() for w in layer.weights)
    xd = x.double()
    logits = xd @ gate.t()
    assert (logits.gather(1, idx).min(dim=1).values >= logits.topk(k, dim=1).values[:, -1] - 1e-3).all()
    w = torch.softmax(logits.gather(1, idx), dim=1)
    xe = xd.clone().requires_grad_()  # dx is that through the experts
    want = torch.zeros((T, H), dtype=torch.float64, device="cuda")
    for e in range(E):
        t, j = torch.nonzero(idx == e, as_tuple=True)
        g, u = (xe[t] @ w1[e].t()).split(I, dim=1)
        y = (torch.nn.functional.silu(g) * u) @ w2[e].t()
        want = want.index_add(0, t, w[t, j][:, None] * y)
    counts = torch.bincount(idx.reshape(-1), minlength=E).double()
    p = torch.softmax(logits, dim=1)
    balance = 0.5 * (E / (k * T) * counts * p.mean(dim=0)).sum()
    grads = torch.autograd.grad((want * c.double()).sum() + balance, [gate, w1, w2, xe])
    bound = 8 * 2.0 ** -8
    assert (out.double() - want).norm() <= bound * want.norm()
    for name, got, ref in zip(("gate", "gate_up", "down", "dx"), (*layer.grads, layer.dx), grads):
        assert (got.double() - ref).norm() <= bound * ref.norm(), name
    assert abs(layer.loss.item() - balance.item()) <= 1e-4 * balance.item()
    layer.end_batch()
    layer.close()


@pytest.mark.parametrize("bits", [8, 32])
def test_example_runs(bits):
    from examples import expert_training

    losses = expert_training.main(["--tokens", "256", "--steps", "3", "--state-bits", str(bits)])
    assert len(losses) == 3 and np.isfinite(losses).all()


def test_captured_way_back_beside_eager_work():
    """The experts' way there and back, captured and replayed between eager runs, gives the eager run's bits."""
    import torch

    from examples.expert_training import BF16, F32, ExpertLayer, M

    T, E, k, H, I = 200, 8, 2, 128, 64
    s = torch.cuda.Stream()
    layer = ExpertLayer(T, E, k, H, I, s, seed=4)
    x = torch.randn((T, H), device="cuda").to(torch.bfloat16)
    layer.dout.normal_()
    torch.cuda.synchronize()
    layer.forward(x)
    layer.backward(x)
    s.synchronize()
    first = [g.clone() for g in (*layer.grads[1:], layer.dx, layer.dlogits)]
    v, R = layer.view, T * k

    def back():
        M.check(M.moe_rows_combine_backward(layer.dout, F32, 0, layer.y, BF16, 0, R, v.topk_w, v.row_of_slot, T, k, H, layer.dy,
                                            BF16, 0, layer.dw, s))
        M.check(M.moe_gate_backward(v.topk_idx, v.topk_w, layer.dw, T, E, k, layer.dlogits, F32, 0, False, s))
        M.check(M.moe_ffn_down_backward(layer.dy, 0, R, layer.down, layer.gu, E, v.offsets, H, I, BF16, layer.dgu, None, s))
        M.check(M.moe_ffn_gate_up_backward(layer.dgu, R, layer.gate_up, E, v.offsets, H, I, BF16, layer.drows, BF16, 0, s))
        M.check(M.moe_rows_combine(layer.drows, BF16, 0, R, None, v.row_of_slot, T, k, H, layer.dx, BF16, 0, s))
        for a, b, dw in ((layer.dgu, layer.rows, layer.grads[1]), (layer.dy, layer.h, layer.grads[2])):
            M.check(M.moe_ffn_weight_grad(a, 0, b, 0, R, E, v.offsets, a.shape[1], b.shape[1], BF16, dw, F32, False, layer.work,
                                          layer.work_bytes, s))

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        graph.capture_begin()
        back()
        graph.capture_end()
    for i in range(4):
        for g in (*layer.grads[1:], layer.dx, layer.dlogits, layer.dy, layer.dgu):
            g.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay() if i % 2 else back()
        torch.cuda.synchronize()
        for want, got in zip(first, (*layer.grads[1:], layer.dx, layer.dlogits)):
            assert torch.equal(want, got)
    del graph
    layer.end_batch()
    layer.close()
