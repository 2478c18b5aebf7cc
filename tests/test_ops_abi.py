"""The MX FP4 and balance-loss calls refuse bad arguments on the host, before
anything touches a GPU (fake pointers)."""

import pytest

from paper_2609_00993_amd import moepd as M

P = 0x1000
BAD = M.MOE_ERR_INVALID_ARG


def test_mx4_size():
    assert M.moe_mx4_size(33, 257, ) == (M.MOE_OK, 64 * 512 // 2, 64 * 512 // 32)
    assert M.moe_mx4_size(0, 1) == (M.MOE_OK, 0, 0)
    for rows, cols in ((-1, 32), (1, 0), (1, (1 << 20) + 1), (1 << 31, 32)):
        assert M.moe_mx4_size(rows, cols)[0] == BAD


def _call(f, base, **kw):
    a = dict(base)
    a.update(kw)
    return f(**a)


QUANT = dict(x=P, x_dtype=M.MOE_DTYPE_BF16, x_stride=0, rows=4, cols=64, row_index=None, row_count=None, codes=P,
             scales=P, stream=P)


@pytest.mark.parametrize("kw", [
    dict(stream=None), dict(x=None), dict(codes=None), dict(scales=None), dict(rows=-1), dict(cols=0), dict(x_stride=63),
    dict(x_dtype=M.MOE_DTYPE_FP8), dict(x_dtype=M.MOE_DTYPE_FP4), dict(codes=P + 8), dict(scales=P + 4), dict(x=P + 1),
    dict(x=P + 2, x_dtype=M.MOE_DTYPE_F32), dict(row_index=P + 2), dict(row_count=P + 1), dict(rows=1 << 31)])
def test_quantize_refuses(kw):
    assert _call(M.moe_mx4_quantize, QUANT, **kw) == BAD


DEQUANT = dict(codes=P, scales=P, rows=4, cols=64, out=P, out_dtype=M.MOE_DTYPE_F32, out_stride=0, stream=P)


@pytest.mark.parametrize("kw", [dict(stream=None), dict(out=None), dict(codes=None), dict(scales=None), dict(rows=-1),
                                dict(cols=0), dict(out_stride=63), dict(out_dtype=M.MOE_DTYPE_FP4), dict(out=P + 2),
                                dict(codes=P + 4), dict(scales=P + 8)])
def test_dequantize_refuses(kw):
    assert _call(M.moe_mx4_dequantize, DEQUANT, **kw) == BAD


PACK = dict(in_codes=P, in_scales=P, rows=4, cols=64, codes=P, scales=P, stream=P)


@pytest.mark.parametrize("kw", [dict(stream=None), dict(in_codes=None), dict(in_scales=None), dict(codes=None),
                                dict(scales=None), dict(rows=-1), dict(cols=48), dict(cols=0), dict(in_codes=P + 8),
                                dict(codes=P + 1)])
def test_pack_refuses(kw):
    assert _call(M.moe_mx4_pack, PACK, **kw) == BAD


GEMM = dict(a=P, a_scales=P, rows=4, w=P, w_scales=P, groups=1, offsets=None, n=8, k=64, out=P,
            out_dtype=M.MOE_DTYPE_F32, out_stride=0, stream=P)


@pytest.mark.parametrize("kw", [
    dict(stream=None), dict(a=None), dict(a_scales=None), dict(w=None), dict(w_scales=None), dict(out=None),
    dict(rows=-1), dict(rows=1 << 31), dict(n=0), dict(k=0), dict(n=(1 << 20) + 1), dict(k=(1 << 20) + 1),
    dict(groups=0), dict(groups=1025, offsets=P), dict(groups=2), dict(out_stride=7), dict(out=P + 2),
    dict(out_dtype=M.MOE_DTYPE_FP8), dict(a=P + 8), dict(a_scales=P + 4), dict(w=P + 8), dict(w_scales=P + 4),
    dict(offsets=P + 2)])
def test_products_refuse(kw):
    assert _call(M.moe_mx4_gemm, GEMM, **kw) == BAD
    assert _call(M.moe_mx4_gemm_swiglu, dict(GEMM, out_scales=None), **kw) == BAD


def test_fp4_output_is_the_gated_products_alone():
    assert _call(M.moe_mx4_gemm, GEMM, out_dtype=M.MOE_DTYPE_FP4) == BAD
    gated = dict(GEMM, out_dtype=M.MOE_DTYPE_FP4, out_scales=P, n=32)
    for kw in (dict(out_scales=None), dict(n=40), dict(out_stride=32), dict(out=P + 8), dict(out_scales=P + 4)):
        assert _call(M.moe_mx4_gemm_swiglu, gated, **kw) == BAD
    assert _call(M.moe_mx4_gemm_swiglu, gated, out_dtype=M.MOE_DTYPE_BF16) == BAD  # scales without FP4


def test_no_rows_is_legal():
    none = dict(rows=0, stream=P)
    assert _call(M.moe_mx4_quantize, QUANT, x=None, codes=None, scales=None, **none) == M.MOE_OK
    assert _call(M.moe_mx4_dequantize, DEQUANT, out=None, codes=None, scales=None, **none) == M.MOE_OK
    assert _call(M.moe_mx4_pack, PACK, in_codes=None, in_scales=None, **none) == M.MOE_OK
    assert _call(M.moe_mx4_gemm, GEMM, a=None, out=None, **none) == M.MOE_OK


W = 0x2000  # 256-byte aligned
LOSS = dict(logits=P, logits_dtype=M.MOE_DTYPE_F32, logits_stride=0, topk_idx=P, token_mask=None, seq_offsets=None, S=1,
            T=4, E=8, k=2, coef=0.1, loss=P, counts=P, live=P, workspace=W, workspace_bytes=1 << 30, stream=P)


@pytest.mark.parametrize("kw", [
    dict(stream=None), dict(logits=None), dict(topk_idx=None), dict(loss=None), dict(counts=None), dict(live=None),
    dict(workspace=None), dict(workspace=W + 64), dict(S=0), dict(S=2), dict(S=65537, seq_offsets=P), dict(T=-1),
    dict(T=(1 << 24) + 1), dict(E=0), dict(E=1025), dict(k=0), dict(k=9), dict(k=17, E=32), dict(logits_stride=7),
    dict(logits_dtype=M.MOE_DTYPE_FP8), dict(logits=P + 2), dict(topk_idx=P + 2), dict(seq_offsets=P + 1), dict(loss=P + 2)])
def test_balance_loss_refuses(kw):
    assert _call(M.moe_balance_loss, LOSS, **kw) == BAD


def test_balance_workspace():
    st, n = M.moe_balance_workspace(4, 8, 1)
    assert st == M.MOE_OK and n > 0
    assert _call(M.moe_balance_loss, LOSS, workspace_bytes=n - 1) == M.MOE_ERR_CAPACITY
    for a in ((-1, 8, 1), ((1 << 24) + 1, 8, 1), (4, 0, 1), (4, 1025, 1), (4, 8, 0), (4, 8, 65537)):
        assert M.moe_balance_workspace(*a)[0] == BAD


BACK = dict(logits=P, logits_dtype=M.MOE_DTYPE_F32, logits_stride=0, token_mask=None, seq_offsets=None, S=1, T=4, E=8,
            k=2, coef=0.1, counts=P, live=P, grad=None, dlogits=W, dlogits_stride=0, accumulate=False, stream=P)


@pytest.mark.parametrize("kw", [
    dict(stream=None), dict(logits=None), dict(counts=None), dict(live=None), dict(dlogits=None), dict(S=0), dict(S=2),
    dict(T=-1), dict(E=0), dict(E=1025), dict(k=0), dict(k=9), dict(logits_stride=7), dict(dlogits_stride=7),
    dict(logits_dtype=7), dict(dlogits=W + 2), dict(grad=P + 2), dict(dlogits=P, accumulate=True),
    dict(dlogits=P, dlogits_stride=9)])
def test_balance_backward_refuses(kw):
    assert _call(M.moe_balance_loss_backward, BACK, **kw) == BAD


def test_balance_backward_without_tokens_is_legal():
    assert _call(M.moe_balance_loss_backward, BACK, T=0, logits=None, dlogits=None) == M.MOE_OK


@pytest.mark.parametrize("n", [1 << 20, (1 << 20) - 5, 700_001])
@pytest.mark.parametrize("groups,offsets", [(1, None), (1024, P)])
def test_products_refuse_more_workgroups_than_a_launch_holds(n, groups, offsets):
    """Tiles whose number passes 32 bits, multiples of 2^32 among them, are refused, not wrapped."""
    most = dict(rows=(1 << 31) - 32, n=n, groups=groups, offsets=offsets)
    for out_dtype in (M.MOE_DTYPE_F32, M.MOE_DTYPE_BF16):
        assert _call(M.moe_mx4_gemm, GEMM, out_dtype=out_dtype, **most) == BAD
        assert _call(M.moe_mx4_gemm_swiglu, dict(GEMM, out_scales=None), out_dtype=out_dtype, **most) == BAD
