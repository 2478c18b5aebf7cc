"""A few steps of training an expert layer: router and experts, forward and back.

    python examples/expert_training.py [--tokens 4096] [--steps 10] [--state-bits 8]

A context routes a batch from its hidden states and lays it out; the tokens go into
expert order, through the experts' gated blocks and, weighted, back. The way back gives
the gradients of the experts' weights and, with the balance loss's, of the gate; one
AdamW step, with states in 8 bits or in 32, updates them all. The target is what another
layer of the same shape gives.
"""

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_00993_amd import moepd as M  # noqa: E402

P, BF16, F32 = M.MOE_PHASE_P, M.MOE_DTYPE_BF16, M.MOE_DTYPE_F32


class ExpertLayer:
    """The weights of a layer, its buffers for batches of T tokens, and its passes on one stream."""

    def __init__(self, T, E, k, H, I, stream, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.T, self.E, self.k, self.H, self.I, self.stream = T, E, k, H, I, stream
        randn = lambda std, *shape: torch.randn(shape, generator=g, device="cuda") * std  # noqa: E731
        self.masters = [randn(1 / math.sqrt(H), E, H), randn(1 / math.sqrt(H), E, 2 * I, H), randn(1 / math.sqrt(I), E, H, I)]
        self.gate, self.gate_up, self.down = self.weights = [w.to(torch.bfloat16) for w in self.masters]
        R = T * k  # every expert is resident: each slot has a row
        bf16 = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        f32 = lambda *shape: torch.empty(shape, device="cuda")  # noqa: E731
        self.rows, self.gu, self.h, self.y = bf16(R, H), bf16(R, 2 * I), bf16(R, I), bf16(R, H)
        self.out, self.dout = f32(T, H), f32(T, H)
        self.dy, self.dgu, self.drows, self.dx = bf16(R, H), bf16(R, 2 * I), bf16(R, H), bf16(T, H)
        self.dw, self.dlogits, self.dlogits16 = f32(T, k), f32(T, E), bf16(T, E)
        self.grads = [f32(E, H), f32(E, 2 * I, H), f32(E, H, I)]
        self.loss, self.counts = f32(1), torch.empty((1, E), dtype=torch.int32, device="cuda")
        self.live = torch.empty(2, dtype=torch.int32, device="cuda")
        sizes = [M.moe_balance_workspace(T, E, 1)] + [M.moe_ffn_weight_workspace(R, n, a, b) for n, a, b in
                                                      ((1, E, H), (E, 2 * I, H), (E, H, I))]
        for st, _ in sizes:
            M.check(st, "workspace")
        self.work_bytes = max(n for _, n in sizes)
        self.work = torch.empty(max(self.work_bytes, 256), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        cfg = M.make_config(E, 0, E, k, H, I, M.MOE_DTYPE_BF16, T, 0)
        st, self.ctx = M.moe_ctx_create(cfg, self.gate_up, self.down)
        M.check(st, "moe_ctx_create")
        st, self.view = M.moe_phase_view(self.ctx, P)
        M.check(st, "moe_phase_view")

    def close(self):
        M.check(M.moe_ctx_destroy(self.ctx), "moe_ctx_destroy")

    def forward(self, x):
        """out [T, H] float32 of x [T, H] bf16; keeps what the way back needs."""
        T, E, k, H, I, v, s = self.T, self.E, self.k, self.H, self.I, self.view, self.stream
        R = T * k
        M.check(M.moe_route_from_hidden(self.ctx, P, x, self.gate, None, T, s), "moe_route_from_hidden")
        M.check(M.moe_dispatch_layout(self.ctx, P, s), "moe_dispatch_layout")
        M.check(M.moe_rows_gather(x, BF16, 0, T, v.token_of_row, v.offsets + 4 * E, R, H, self.rows, 0, s), "moe_rows_gather")
        M.check(M.moe_ffn_gate_up(self.rows, 0, R, self.gate_up, E, v.offsets, H, I, BF16, self.gu, self.h, s), "moe_ffn_gate_up")
        M.check(M.moe_ffn_down(self.h, R, self.down, E, v.offsets, H, I, BF16, self.y, BF16, 0, s), "moe_ffn_down")
        M.check(M.moe_rows_combine(self.y, BF16, 0, R, v.topk_w, v.row_of_slot, T, k, H, self.out, F32, 0, s), "moe_rows_combine")
        return self.out

    def backward(self, x, balance=0.0):
        """From dout (the loss's gradient in out) to the weights' gradients, the balance loss's with them, and dx through
        the experts."""
        T, E, k, H, I, v, s = self.T, self.E, self.k, self.H, self.I, self.view, self.stream
        R = T * k
        M.check(M.moe_rows_combine_backward(self.dout, F32, 0, self.y, BF16, 0, R, v.topk_w, v.row_of_slot, T, k, H, self.dy,
                                            BF16, 0, self.dw, s), "moe_rows_combine_backward")
        M.check(M.moe_gate_backward(v.topk_idx, v.topk_w, self.dw, T, E, k, self.dlogits, F32, 0, False, s), "moe_gate_backward")
        if balance:
            M.check(M.moe_balance_loss(v.logits, F32, 0, v.topk_idx, None, None, 1, T, E, k, balance, self.loss, self.counts,
                                       self.live, self.work, self.work_bytes, s), "moe_balance_loss")
            M.check(M.moe_balance_loss_backward(v.logits, F32, 0, None, None, 1, T, E, k, balance, self.counts, self.live, None,
                                                self.dlogits, 0, True, s), "moe_balance_loss_backward")
        with torch.cuda.stream(s):
            self.dlogits16.copy_(self.dlogits)
        M.check(M.moe_ffn_down_backward(self.dy, 0, R, self.down, self.gu, E, v.offsets, H, I, BF16, self.dgu, None, s),
                "moe_ffn_down_backward")
        M.check(M.moe_ffn_gate_up_backward(self.dgu, R, self.gate_up, E, v.offsets, H, I, BF16, self.drows, BF16, 0, s),
                "moe_ffn_gate_up_backward")
        M.check(M.moe_rows_combine(self.drows, BF16, 0, R, None, v.row_of_slot, T, k, H, self.dx, BF16, 0, s), "moe_rows_combine")
        for a, b, rows, n, off, dw in ((self.dlogits16, x, T, 1, None, self.grads[0]),
                                       (self.dgu, self.rows, R, E, v.offsets, self.grads[1]),
                                       (self.dy, self.h, R, E, v.offsets, self.grads[2])):
            M.check(M.moe_ffn_weight_grad(a, 0, b, 0, rows, n, off, a.shape[1], b.shape[1], BF16, dw, F32, False, self.work,
                                          self.work_bytes, s), "moe_ffn_weight_grad")

    def end_batch(self):
        """The phase back to idle, once the batch's work is done."""
        self.stream.synchronize()
        M.check(M.moe_phase_reset(self.ctx, P), "moe_phase_reset")


class AdamW:
    """The table of a layer's weights, with states of `bits`."""

    def __init__(self, layer, bits, decay=0.0):
        self.states = []
        for w in layer.masters:
            n = w.numel()
            z = lambda count, t: torch.zeros(count, dtype=t, device="cuda")  # noqa: E731
            t = torch.float32 if bits == 32 else torch.uint8
            scales = (None, None) if bits == 32 else (z(-(-n // 32), t), z(-(-n // 32), t))
            self.states.append((z(n, t), z(n, t), *scales))
        table = [M.adamw_tensor(p, BF16, w, g, F32, m, v, ms, vs, w.numel(), decay) for p, w, g, (m, v, ms, vs) in
                 zip(layer.weights, layer.masters, layer.grads, self.states)]
        st, self.table = M.moe_adamw_create(table, bits)
        M.check(st, "moe_adamw_create")
        self.lr, self.t = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()

    def step(self, lr, stream):
        with torch.cuda.stream(stream):
            self.lr.fill_(lr)
            self.t += 1
        M.check(M.moe_adamw_step(self.table, 0.9, 0.95, 1e-8, self.lr, self.t, None, 1234, stream), "moe_adamw_step")

    def close(self):
        M.check(M.moe_adamw_destroy(self.table), "moe_adamw_destroy")


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args(argv)
    T, shape = a.tokens, dict(E=16, k=2, H=1024, I=512)
    stream = torch.cuda.Stream()
    layer, teacher = (ExpertLayer(T, **shape, stream=stream, seed=s) for s in (0, 1))
    opt = AdamW(layer, a.state_bits)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    losses = []
    try:
        for step in range(a.steps):
            x = torch.randn((T, shape["H"]), generator=g, device="cuda").to(torch.bfloat16)
            torch.cuda.synchronize()
            target = teacher.forward(x)
            out = layer.forward(x)
            with torch.cuda.stream(stream):
                torch.sub(out, target, out=layer.dout)
                loss = layer.dout.square().sum() / T
                layer.dout *= 2.0 / T
            layer.backward(x, balance=0.01)
            opt.step(1e-3, stream)
            for end in (layer, teacher):
                end.end_batch()
            losses.append(loss.item())
            print(f"step {step}: loss {losses[-1]:.4f}, balance {layer.loss.item():.5f}, fullest expert "
                  f"{layer.counts.max().item()} of {T * shape['k']} slots", flush=True)
    finally:
        opt.close()
        layer.close()
        teacher.close()
    return losses


if __name__ == "__main__":
    main()
