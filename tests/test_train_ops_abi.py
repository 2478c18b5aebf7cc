"""The feed-forward block's, the token rows' and AdamW's calls refuse bad arguments on the host, before
anything touches a GPU (fake pointers)."""

import pytest

from paper_2609_00993_amd import moepd as M

P = 0x1000
BAD = M.MOE_ERR_INVALID_ARG
BF16, F32, FP8 = M.MOE_DTYPE_BF16, M.MOE_DTYPE_F32, M.MOE_DTYPE_FP8


def _call(f, base, **kw):
    return f(**{**base, **kw})


SHAPE = [dict(stream=None), dict(rows=-1), dict(rows=(1 << 31) - 511), dict(groups=0), dict(groups=1025, offsets=P),
         dict(groups=2), dict(offsets=P + 2), dict(hidden=0), dict(hidden=12), dict(hidden=32776), dict(inter=4),
         dict(inter=32776), dict(hidden=32768, inter=16384), dict(dtype=FP8), dict(dtype=7)]

GATE_UP = dict(x=P, x_stride=0, rows=4, w_gate_up=P, groups=1, offsets=None, hidden=64, inter=32, dtype=BF16, gate_up=P, h=P,
               stream=P)


@pytest.mark.parametrize("kw", SHAPE + [dict(x=None), dict(w_gate_up=None), dict(h=None), dict(x=P + 8), dict(h=P + 4),
                                        dict(gate_up=P + 2), dict(w_gate_up=P + 8), dict(x_stride=56), dict(x_stride=68),
                                        dict(x_stride=(1 << 20) + 8), dict(x_stride=-64)])
def test_gate_up_refuses(kw):
    assert _call(M.moe_ffn_gate_up, GATE_UP, **kw) == BAD


DOWN = dict(h=P, rows=4, w_down=P, groups=1, offsets=None, hidden=64, inter=32, dtype=BF16, y=P, y_dtype=BF16, y_stride=0,
            stream=P)


@pytest.mark.parametrize("kw", SHAPE + [dict(h=None), dict(w_down=None), dict(y=None), dict(y=P + 8), dict(h=P + 2),
                                        dict(y_stride=56), dict(y_stride=66), dict(y_dtype=FP8), dict(y_dtype=BF16, dtype=F32)])
def test_down_refuses(kw):
    assert _call(M.moe_ffn_down, DOWN, **kw) == BAD


DOWN_BACK = dict(dy=P, dy_stride=0, rows=4, w_down=P, gate_up=P, groups=1, offsets=None, hidden=64, inter=32, dtype=BF16,
                 dgate_up=P, h=None, stream=P)


@pytest.mark.parametrize("kw", SHAPE + [dict(dy=None), dict(w_down=None), dict(gate_up=None), dict(dgate_up=None), dict(h=P + 8),
                                        dict(dy=P + 8), dict(gate_up=P + 8), dict(dgate_up=P + 4), dict(dy_stride=56)])
def test_down_backward_refuses(kw):
    assert _call(M.moe_ffn_down_backward, DOWN_BACK, **kw) == BAD


UP_BACK = dict(dgate_up=P, rows=4, w_gate_up=P, groups=1, offsets=None, hidden=64, inter=32, dtype=BF16, dx=P, dx_dtype=F32,
               dx_stride=0, stream=P)


@pytest.mark.parametrize("kw", SHAPE + [dict(dgate_up=None), dict(w_gate_up=None), dict(dx=None), dict(dx=P + 8),
                                        dict(dgate_up=P + 8), dict(dx_stride=56), dict(dx_dtype=M.MOE_DTYPE_FP4),
                                        dict(dtype=F32, dx_dtype=BF16)])
def test_gate_up_backward_refuses(kw):
    assert _call(M.moe_ffn_gate_up_backward, UP_BACK, **kw) == BAD


WEIGHT = dict(a=P, a_stride=0, b=P, b_stride=0, rows=4, groups=1, offsets=None, m=64, n=32, dtype=BF16, dw=P, dw_dtype=F32,
              accumulate=False, workspace=None, workspace_bytes=0, stream=P)


@pytest.mark.parametrize("kw", [
    dict(stream=None), dict(a=None), dict(b=None), dict(dw=None), dict(rows=-1), dict(rows=1 << 31), dict(groups=0), dict(groups=2),
    dict(groups=1025, offsets=P), dict(offsets=P + 1), dict(m=0), dict(m=12), dict(n=4), dict(m=65544), dict(m=65536, n=65536),
    dict(a_stride=56), dict(b_stride=36), dict(a=P + 8), dict(b=P + 2), dict(dw=P + 4), dict(dtype=FP8), dict(dw_dtype=FP8),
    dict(dtype=F32, dw_dtype=BF16), dict(workspace=P + 128)])
def test_weight_gradient_refuses(kw):
    assert _call(M.moe_ffn_weight_grad, WEIGHT, **kw) == BAD


def test_weight_workspace():
    st, need = M.moe_ffn_weight_workspace(9000, 1, 272, 264)
    assert st == M.MOE_OK and need > 0
    big = dict(WEIGHT, rows=9000, m=272, n=264)
    assert _call(M.moe_ffn_weight_grad, big) == BAD  # none given
    assert _call(M.moe_ffn_weight_grad, big, workspace=P, workspace_bytes=need - 1) == M.MOE_ERR_CAPACITY
    for a in ((-1, 1, 8, 8), (1 << 31, 1, 8, 8), (1, 0, 8, 8), (1, 1025, 8, 8), (1, 1, 0, 8), (1, 1, 8, 12), (1, 1, 65536, 65536)):
        assert M.moe_ffn_weight_workspace(*a)[0] == BAD


GATHER = dict(x=P, dtype=BF16, x_stride=0, T=4, token_of_row=P, row_count=None, rows=8, hidden=33, out=P, out_stride=0, stream=P)


@pytest.mark.parametrize("kw", [
    dict(stream=None), dict(x=None), dict(token_of_row=None), dict(out=None), dict(T=-1), dict(T=(1 << 24) + 1), dict(rows=-1),
    dict(rows=1 << 31), dict(hidden=0), dict(hidden=(1 << 20) + 1), dict(x_stride=32), dict(out_stride=-33), dict(dtype=FP8),
    dict(x=P + 1), dict(out=P + 2, dtype=F32), dict(token_of_row=P + 2), dict(row_count=P + 1)])
def test_gather_refuses(kw):
    assert _call(M.moe_rows_gather, GATHER, **kw) == BAD


COMBINE = dict(y=P, y_dtype=BF16, y_stride=0, rows=8, w=P, row_of_slot=P, T=4, k=2, hidden=33, out=P, out_dtype=F32,
               out_stride=0, stream=P)
SLOTS = [dict(stream=None), dict(row_of_slot=None), dict(T=-1), dict(T=1 << 25), dict(k=0), dict(k=17), dict(rows=-1),
         dict(hidden=0), dict(y_stride=32), dict(y_dtype=FP8), dict(y=P + 1), dict(w=P + 2), dict(row_of_slot=P + 2)]


@pytest.mark.parametrize("kw", SLOTS + [dict(y=None), dict(out=None), dict(out=P + 2), dict(out_dtype=9), dict(out_stride=31)])
def test_combine_refuses(kw):
    assert _call(M.moe_rows_combine, COMBINE, **kw) == BAD


COMBINE_BACK = dict(dout=P, dout_dtype=F32, dout_stride=0, y=P, y_dtype=BF16, y_stride=0, rows=8, w=P, row_of_slot=P, T=4, k=2,
                    hidden=33, dy=P, dy_dtype=BF16, dy_stride=0, dw=P, stream=P)


@pytest.mark.parametrize("kw", SLOTS + [dict(y=None), dict(dout=None), dict(dy=None), dict(dout=P + 2), dict(dout_dtype=FP8),
                                        dict(dy_dtype=FP8), dict(dy=P + 1), dict(dw=P + 2), dict(dy_stride=32),
                                        dict(dout_stride=1)])
def test_combine_backward_refuses(kw):
    assert _call(M.moe_rows_combine_backward, COMBINE_BACK, **kw) == BAD


GATE = dict(topk_idx=P, topk_w=P, dw=P, T=4, E=8, k=2, dlogits=P, dlogits_dtype=F32, dlogits_stride=0, accumulate=False, stream=P)


@pytest.mark.parametrize("kw", [
    dict(stream=None), dict(topk_idx=None), dict(topk_w=None), dict(dw=None), dict(dlogits=None), dict(T=-1), dict(E=0),
    dict(E=1025), dict(k=0), dict(k=9), dict(k=17, E=64), dict(dlogits_dtype=FP8), dict(dlogits_stride=7), dict(dlogits=P + 2),
    dict(topk_idx=P + 2), dict(topk_w=P + 1), dict(dw=P + 2)])
def test_gate_refuses(kw):
    assert _call(M.moe_gate_backward, GATE, **kw) == BAD


def test_nothing_to_do_is_legal():
    none = dict(rows=0)
    assert _call(M.moe_ffn_gate_up, GATE_UP, x=None, h=None, **none) == M.MOE_OK
    assert _call(M.moe_ffn_down, DOWN, h=None, y=None, **none) == M.MOE_OK
    assert _call(M.moe_ffn_down_backward, DOWN_BACK, dy=None, dgate_up=None, **none) == M.MOE_OK
    assert _call(M.moe_ffn_gate_up_backward, UP_BACK, dgate_up=None, dx=None, **none) == M.MOE_OK
    assert _call(M.moe_rows_gather, GATHER, x=None, out=None, **none) == M.MOE_OK
    assert _call(M.moe_rows_combine, COMBINE, T=0, y=None, out=None) == M.MOE_OK
    assert _call(M.moe_rows_combine_backward, COMBINE_BACK, T=0, dout=None, dy=None) == M.MOE_OK
    assert _call(M.moe_gate_backward, GATE, T=0, dlogits=None) == M.MOE_OK


def _tensor(**kw):
    a = dict(param=P, param_dtype=BF16, master=P, grad=P, grad_dtype=BF16, m=P, v=P, m_scales=None, v_scales=None, n=40)
    return M.adamw_tensor(**{**a, **kw})


@pytest.mark.parametrize("bits,kw", [
    (32, dict(param=None)), (32, dict(grad=None)), (32, dict(m=None)), (32, dict(v=None)), (32, dict(n=-1)),
    (32, dict(n=(1 << 40) + 1)), (32, dict(param_dtype=FP8)), (32, dict(grad_dtype=5)), (32, dict(param=P + 1)),
    (32, dict(master=P + 2)), (32, dict(grad=P + 2, grad_dtype=F32)), (32, dict(m=P + 2)), (32, dict(v=P + 1)),
    (32, dict(m_scales=P)), (32, dict(v_scales=P)), (32, dict(weight_decay=float("nan"))), (32, dict(weight_decay=float("inf"))),
    (8, {}), (8, dict(m_scales=P)), (8, dict(v_scales=P)), (16, {})])
def test_adamw_create_refuses(bits, kw):
    assert M.moe_adamw_create([_tensor(), _tensor(**kw)] if bits == 32 else [_tensor(**kw)], bits) == (BAD, None)


def test_adamw_counts_and_null():
    assert M.moe_adamw_create(None, 32) == (BAD, None)
    assert M.moe_adamw_create([], 32) == (BAD, None)
    assert M.moe_adamw_destroy(None) == M.MOE_OK
    assert M.moe_adamw_step(None, 0.9, 0.99, 1e-8, P, P, None, 0, P) == BAD
    assert M.moe_adamw_read(None, 0, P, P, F32, P) == BAD
