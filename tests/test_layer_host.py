"""Argument checks of the block operators: refusals come before any device work, and sizes need no device."""
import pytest

import paper_2409_03864_b200 as tdx
from paper_2409_03864_b200 import build as tdx_build

P = 1 << 20        # an aligned address that is never used
INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = tdx.TDX_ERR_INVALID_ARG, tdx.TDX_ERR_UNSUPPORTED, tdx.TDX_ERR_ALIGNMENT, tdx.TDX_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def built():
    tdx_build.build()


def norm(**change):
    a = dict(rows=4, channels=8, group=4, dtype=tdx.TDX_BF16, norm_in=1, eps=1e-5, weight_in=P, scale=P, weight_out=P, dweight_in=P, dscale=P, dweight_out=P)
    for n in ("x", "gate", "residual", "sum", "y", "dsum", "dy", "dx", "dgate", "dresidual"):
        a.update({n: P, "ld_" + n: 8})
    return tdx.tdx_norm_args(**{**a, **change})


NORM_BAD = [
    (dict(rows=-1), INVALID), (dict(channels=-1), INVALID), (dict(group=-4), INVALID), (dict(group=3), INVALID), (dict(dtype=2), INVALID),
    (dict(norm_in=2), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(x=None), INVALID), (dict(ld_x=7), INVALID),
    (dict(ld_gate=7), INVALID), (dict(ld_residual=7), INVALID), (dict(x=P + 1), ALIGNMENT), (dict(gate=P + 1), ALIGNMENT), (dict(scale=P + 2), ALIGNMENT),
    (dict(weight_in=P + 2), ALIGNMENT), (dict(weight_out=P + 1), ALIGNMENT), (dict(channels=(1 << 20) + 1, group=0), UNSUPPORTED),
    (dict(channels=10000, group=2), UNSUPPORTED), (dict(ld_x=(1 << 24) + 1), UNSUPPORTED),
]


@pytest.mark.parametrize("change,status", NORM_BAD + [(dict(sum=None, y=None), INVALID), (dict(ld_sum=7), INVALID), (dict(ld_y=7), INVALID), (dict(y=P + 1), ALIGNMENT)])
def test_block_norm_refusals(change, status):
    assert tdx.tdx_block_norm(norm(**change)) == status, tdx.tdx_last_error()
    assert tdx.tdx_last_error()


@pytest.mark.parametrize("change,status", NORM_BAD + [
    (dict(dsum=None, dy=None), INVALID), (dict(dx=None), INVALID), (dict(dgate=None), INVALID), (dict(dresidual=None), INVALID), (dict(ld_dx=7), INVALID),
    (dict(ld_dy=7), INVALID), (dict(norm_in=0), INVALID), (dict(dweight_in=P + 2), ALIGNMENT), (dict(dscale=P + 1), ALIGNMENT)])
def test_block_norm_bwd_refusals(change, status):
    assert tdx.tdx_block_norm_bwd(norm(**change)) == status, tdx.tdx_last_error()


def test_block_norm_sizes_and_empty_calls():
    status, size = tdx.tdx_block_norm_workspace_size(norm())
    assert status == 0 and size > 0
    assert tdx.tdx_block_norm(norm(rows=0, x=None, sum=None, y=None)) == 0
    assert tdx.tdx_block_norm(norm(channels=0, group=0)) == 0
    assert tdx.lib().tdx_block_norm(None, None) == INVALID and tdx.lib().tdx_block_norm_bwd(None, None) == INVALID


def grouped(**change):
    a = dict(rows=6, experts=2, N=8, K=16, dtype=tdx.TDX_BF16, offsets=P, x=P, ld_x=16, weight=P, y=P, ld_y=8, dy=P, ld_dy=8, dx=P, ld_dx=16, dweight=P,
             workspace=P, workspace_bytes=1 << 40)
    return tdx.tdx_grouped_args(**{**a, **change})


GROUPED_BAD = [(dict(rows=-1), INVALID), (dict(experts=-1), INVALID), (dict(N=-1), INVALID), (dict(K=-1), INVALID), (dict(dtype=5), INVALID),
               (dict(offsets=None), INVALID), (dict(offsets=P + 2), ALIGNMENT), (dict(rows=1 << 31), UNSUPPORTED), (dict(experts=1 << 21), UNSUPPORTED),
               (dict(N=1 << 25, ld_y=1 << 25, ld_dy=1 << 25), UNSUPPORTED)]


@pytest.mark.parametrize("call,change,status", [
    ("", dict(x=None), INVALID), ("", dict(weight=None), INVALID), ("", dict(y=None), INVALID), ("", dict(ld_x=15), INVALID), ("", dict(ld_y=7), INVALID),
    ("", dict(x=P + 1), ALIGNMENT), ("", dict(weight=P + 1), ALIGNMENT), ("_dx", dict(dy=None), INVALID), ("_dx", dict(dx=None), INVALID),
    ("_dx", dict(weight=None), INVALID), ("_dx", dict(ld_dx=15), INVALID), ("_dw", dict(dy=None), INVALID), ("_dw", dict(x=None), INVALID),
    ("_dw", dict(dweight=None), INVALID), ("_dw", dict(ld_dy=7), INVALID), ("_dw", dict(dweight=P + 1), ALIGNMENT),
    *[(c, *bad) for c in ("", "_dx", "_dw") for bad in GROUPED_BAD]])
def test_grouped_refusals(call, change, status):
    assert getattr(tdx, "tdx_gemm_grouped" + call)(grouped(**change)) == status, tdx.tdx_last_error()
    assert tdx.tdx_last_error()


def test_grouped_sizes_and_empty_calls():
    status, size = tdx.tdx_gemm_grouped_workspace_size(grouped())
    assert status == 0 and size >= 0
    assert tdx.tdx_gemm_grouped(grouped(rows=0, x=None, y=None)) == 0
    assert tdx.tdx_gemm_grouped(grouped(experts=0, offsets=None)) == 0
    assert tdx.tdx_gemm_grouped_dx(grouped(K=0, dx=None)) == 0 and tdx.tdx_gemm_grouped_dw(grouped(N=0, dweight=None)) == 0
    assert tdx.lib().tdx_gemm_grouped(None, None) == INVALID


def attention(**change):
    a = dict(batch=2, max_len=5, rows=10, heads=4, q_heads=4, k_heads=2, v_heads=2, dim_k=8, dim_v=16, dtype=tdx.TDX_BF16, scale=0.5, log_decay=P, q=P, ld_q=32,
             k=P, ld_k=16, v=P, ld_v=32, out=P, ld_out=64, state_in=P, state_out=P, n_slots=2, dout=P, ld_dout=64, dq=P, ld_dq=32, dk=P, ld_dk=16, dv=P, ld_dv=32,
             dstate_out=P, dstate_in=P, workspace=P, workspace_bytes=1 << 40)
    return tdx.tdx_attention_args(**{**a, **change})


ATTENTION_BAD = [
    (dict(batch=-1), INVALID), (dict(heads=-1), INVALID), (dict(rows=9), INVALID), (dict(dtype=3), INVALID), (dict(q_heads=3), INVALID), (dict(k_heads=-2), INVALID),
    (dict(v_heads=8), INVALID), (dict(dim_k=0), INVALID), (dict(dim_v=-1), INVALID), (dict(dim_k=129, ld_q=1000, ld_k=1000), UNSUPPORTED),
    (dict(dim_v=200, ld_v=1000, ld_out=1000, ld_dout=1000), UNSUPPORTED), (dict(scale=float("inf")), INVALID), (dict(log_decay=None), INVALID), (dict(q=None), INVALID),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(ld_q=31), INVALID), (dict(ld_k=15), INVALID), (dict(ld_v=31), INVALID), (dict(n_slots=1), INVALID),
    (dict(state_stride=100), INVALID), (dict(q=P + 1), ALIGNMENT), (dict(log_decay=P + 2), ALIGNMENT), (dict(slots=P + 2), ALIGNMENT), (dict(seq_offsets=P + 1), ALIGNMENT),
    (dict(state_in=P + 2), ALIGNMENT), (dict(max_len=1 << 31, rows=1 << 32), UNSUPPORTED)]
ROWLESS = ("rows", "max_len", "seq_offsets")


@pytest.mark.parametrize("call,change,status", [
    ("", dict(out=None), INVALID), ("", dict(ld_out=63), INVALID), ("", dict(state_out=P + 2), ALIGNMENT), ("_bwd", dict(dout=None), INVALID), ("_bwd", dict(dq=None), INVALID),
    ("_bwd", dict(dk=None), INVALID), ("_bwd", dict(dv=None), INVALID), ("_bwd", dict(ld_dout=63), INVALID), ("_bwd", dict(ld_dk=15), INVALID),
    ("_bwd", dict(dstate_in=P + 1), ALIGNMENT), ("_step", dict(state_in=None), INVALID), ("_step", dict(state_out=None), INVALID), ("_step", dict(out=None), INVALID),
    *[(c, *bad) for c in ("", "_bwd") for bad in ATTENTION_BAD], *[("_step", *bad) for bad in ATTENTION_BAD if not any(n in bad[0] for n in ROWLESS)]])
def test_attention_refusals(call, change, status):
    assert getattr(tdx, "tdx_decay_attention" + call)(attention(**change)) == status, tdx.tdx_last_error()
    assert tdx.tdx_last_error()


def test_attention_sizes_and_empty_calls():
    status, small = tdx.tdx_decay_attention_workspace_size(attention(dout=None))
    assert status == 0 and small == 0                            # short sequences run whole
    status, cut = tdx.tdx_decay_attention_workspace_size(attention(batch=1, max_len=4096, rows=4096, dout=None))
    assert status == 0 and cut > 0
    status, back = tdx.tdx_decay_attention_workspace_size(attention())
    assert status == 0 and back >= 10 * 4 * 16 * 4               # one gradient a head before heads that share are summed
    assert tdx.tdx_decay_attention_workspace_size(attention(dim_k=0))[0] == INVALID
    assert tdx.tdx_decay_attention(attention(batch=0, rows=0)) == 0 and tdx.tdx_decay_attention_step(attention(batch=0)) == 0
    assert tdx.tdx_decay_attention_bwd(attention(heads=0, q_heads=0, k_heads=0, v_heads=0)) == 0
    assert tdx.lib().tdx_decay_attention(None, None) == INVALID and tdx.lib().tdx_decay_attention_step(None, None) == INVALID


@pytest.mark.parametrize("dtype", [tdx.TDX_BF16, tdx.TDX_F32])
def test_attention_workspace_goes_by_what_is_cut_and_not_by_the_batch(dtype):
    many = dict(heads=32, q_heads=32, k_heads=32, v_heads=32, dim_k=128, dim_v=128, dtype=dtype, max_len=8192, seq_offsets=P, n_slots=1 << 20,
                **{"ld_" + n: 4096 for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")})
    for dout in (None, P):
        status, one = tdx.tdx_decay_attention_workspace_size(attention(**many, batch=1, rows=8192, dout=dout))
        assert status == 0 and one > 0
        for short in (255, 4095):                                # sequences of one row beside the long one
            status, size = tdx.tdx_decay_attention_workspace_size(attention(**many, batch=1 + short, rows=8192 + short, dout=dout))
            assert status == 0 and size <= 2 * one * (8192 + short) / 8192, (short, one, size)
