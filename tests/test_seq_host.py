"""Argument checks of the sequence operators: refusals come before any device work, and sizes need no device."""
import ctypes

import pytest

import paper_2409_03864_b200 as tdx
from paper_2409_03864_b200 import build as tdx_build

P = 1 << 20        # an aligned address that is never used


@pytest.fixture(scope="module", autouse=True)
def built():
    tdx_build.build()


def conv(**change):
    a = dict(batch=2, max_len=5, rows=10, channels=8, width=4, dtype=tdx.TDX_BF16, silu=1, x=P, ld_x=8, weight=P, y=P, ld_y=8, state_in=P, state_out=P,
             n_slots=2, dy=P, ld_dy=8, dx=P, ld_dx=8, dweight=P, dbias=P, dstate_in=P, dstate_out=P)
    return tdx.tdx_conv1d_args(**{**a, **change})


def scan(**change):
    a = dict(batch=2, max_len=5, rows=10, channels=8, states=16, groups=2, dtype=tdx.TDX_F32, dt_softplus=1, x=P, ld_x=8, dt=P, ld_dt=8, A=P, B=P, ld_B=32,
             C=P, ld_C=32, D=P, z=P, ld_z=8, dt_bias=P, out=P, ld_out=8, state_in=P, state_out=P, n_slots=2, dout=P, ld_dout=8, dx=P, ld_dx=8, ddt=P,
             ld_ddt=8, dB=P, ld_dB=32, dC=P, ld_dC=32, dz=P, ld_dz=8, dA=P, dD=P, ddt_bias=P, saved=P, saved_bytes=1 << 30)
    return tdx.tdx_scan_args(**{**a, **change})


def w4(**change):
    a = dict(M=2, N=8, K=64, group_size=32, dtype=tdx.TDX_BF16, x=P, ld_x=64, weight=P, scales=P, zeros=P, y=P, ld_y=8)
    return tdx.tdx_w4_args(**{**a, **change})


INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = tdx.TDX_ERR_INVALID_ARG, tdx.TDX_ERR_UNSUPPORTED, tdx.TDX_ERR_ALIGNMENT, tdx.TDX_ERR_WORKSPACE

CONV_BAD = [
    (dict(batch=-1), INVALID), (dict(channels=-8), INVALID), (dict(rows=9), INVALID), (dict(max_len=-5, rows=-10), INVALID), (dict(dtype=2), INVALID),
    (dict(width=0), INVALID), (dict(width=9), INVALID), (dict(silu=2), INVALID), (dict(x=None), INVALID), (dict(weight=None), INVALID),
    (dict(y=None), INVALID), (dict(ld_x=7), INVALID), (dict(ld_y=7), INVALID), (dict(n_slots=1), INVALID), (dict(state_stride=23), INVALID),
    (dict(x=P + 1), ALIGNMENT), (dict(weight=P + 2), ALIGNMENT), (dict(state_in=P + 1), ALIGNMENT), (dict(slots=P + 2), ALIGNMENT),
    (dict(seq_offsets=P + 2), ALIGNMENT), (dict(max_len=1 << 31, rows=1 << 32), UNSUPPORTED), (dict(seq_offsets=P, rows=1 << 31), UNSUPPORTED),
]


@pytest.mark.parametrize("change,status", CONV_BAD)
def test_conv1d_refusals(change, status):
    assert tdx.tdx_causal_conv1d(conv(**change)) == status, tdx.tdx_last_error()
    assert tdx.tdx_last_error()


@pytest.mark.parametrize("change,status", [(dict(dy=None), INVALID), (dict(dx=None), INVALID), (dict(ld_dx=3), INVALID), (dict(ld_dy=3), INVALID),
                                           (dict(dweight=P + 1), ALIGNMENT), (dict(), WORKSPACE), (dict(workspace=P, workspace_bytes=8), WORKSPACE),
                                           (dict(workspace=P + 16, workspace_bytes=1 << 30), ALIGNMENT)])
def test_conv1d_bwd_refusals(change, status):
    assert tdx.tdx_causal_conv1d_bwd(conv(**change)) == status, tdx.tdx_last_error()


@pytest.mark.parametrize("change,status", [(dict(state_in=None), INVALID), (dict(state_out=None), INVALID), (dict(x=None), INVALID), (dict(batch=-1), INVALID),
                                           (dict(n_slots=1), INVALID), (dict(ld_y=1), INVALID)])
def test_conv1d_step_refusals(change, status):
    assert tdx.tdx_causal_conv1d_step(conv(**change)) == status, tdx.tdx_last_error()


SCAN_BAD = [
    (dict(batch=-1), INVALID), (dict(rows=11), INVALID), (dict(dtype=-1), INVALID), (dict(states=0), INVALID), (dict(states=129), UNSUPPORTED),
    (dict(groups=0), INVALID), (dict(groups=3), INVALID), (dict(dt_softplus=3), INVALID), (dict(x=None), INVALID), (dict(dt=None), INVALID),
    (dict(A=None), INVALID), (dict(B=None), INVALID), (dict(C=None), INVALID), (dict(out=None), INVALID), (dict(ld_B=31), INVALID), (dict(ld_C=31), INVALID),
    (dict(ld_x=7), INVALID), (dict(ld_dt=7), INVALID), (dict(ld_z=7), INVALID), (dict(ld_out=7), INVALID), (dict(n_slots=1), INVALID),
    (dict(state_stride=100), INVALID), (dict(A=P + 2), ALIGNMENT), (dict(z=P + 2), ALIGNMENT), (dict(state_out=P + 2), ALIGNMENT),
    (dict(saved=P + 4), ALIGNMENT), (dict(saved_bytes=16), WORKSPACE),
]


@pytest.mark.parametrize("change,status", SCAN_BAD)
def test_scan_refusals(change, status):
    assert tdx.tdx_selective_scan(scan(**change)) == status, tdx.tdx_last_error()


@pytest.mark.parametrize("change,status", [(dict(saved=None), INVALID), (dict(saved_bytes=0), WORKSPACE), (dict(dout=None), INVALID), (dict(dz=None), INVALID),
                                           (dict(dA=None), INVALID), (dict(dB=None), INVALID), (dict(ld_dC=2), INVALID), (dict(dstate_in=P + 1), ALIGNMENT)])
def test_scan_bwd_refusals(change, status):
    assert tdx.tdx_selective_scan_bwd(scan(**change)) == status, tdx.tdx_last_error()


@pytest.mark.parametrize("change,status", [(dict(state_in=None), INVALID), (dict(state_out=None), INVALID), (dict(groups=5), INVALID), (dict(out=None), INVALID)])
def test_scan_step_refusals(change, status):
    assert tdx.tdx_selective_scan_step(scan(**change)) == status, tdx.tdx_last_error()


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), INVALID), (dict(K=-1), INVALID), (dict(dtype=4), INVALID), (dict(group_size=0), INVALID), (dict(x=None), INVALID), (dict(weight=None), INVALID),
    (dict(scales=None), INVALID), (dict(y=None), INVALID), (dict(ld_x=63), INVALID), (dict(ld_y=7), INVALID), (dict(x=P + 1), ALIGNMENT),
    (dict(scales=P + 1), ALIGNMENT), (dict(K=1 << 32, ld_x=1 << 32), UNSUPPORTED)])
def test_w4_refusals(change, status):
    assert tdx.tdx_gemm_w4(w4(**change)) == status, tdx.tdx_last_error()


def test_w4_quantize_refusals():
    base = dict(N=4, K=64, group_size=32, dtype=tdx.TDX_F32, w=P, ld_w=64, weight=P, scales=P)
    for change in (dict(N=-1), dict(K=-1), dict(dtype=3), dict(group_size=0), dict(group_size=33), dict(w=None), dict(weight=None), dict(scales=None), dict(ld_w=63)):
        assert tdx.tdx_w4_quantize(**{**base, **change}) == INVALID, change
    assert tdx.tdx_w4_quantize(**{**base, "w": P + 2}) == ALIGNMENT
    assert tdx.tdx_w4_quantize(**{**base, "N": 0, "w": None}) == tdx.TDX_OK


def test_empty_problems_need_no_device_and_no_pointers():
    assert tdx.tdx_causal_conv1d(tdx.tdx_conv1d_args(width=4)) == tdx.TDX_OK
    assert tdx.tdx_causal_conv1d_step(tdx.tdx_conv1d_args(width=4)) == tdx.TDX_OK
    assert tdx.tdx_causal_conv1d_bwd(tdx.tdx_conv1d_args(width=4)) == tdx.TDX_OK
    assert tdx.tdx_selective_scan(tdx.tdx_scan_args(states=16, groups=1)) == tdx.TDX_OK
    assert tdx.tdx_selective_scan_bwd(tdx.tdx_scan_args(states=16, groups=1)) == tdx.TDX_OK
    assert tdx.tdx_selective_scan_step(tdx.tdx_scan_args(states=16, groups=1)) == tdx.TDX_OK
    assert tdx.tdx_gemm_w4(tdx.tdx_w4_args(group_size=32, K=64)) == tdx.TDX_OK


def test_null_blocks_are_refused():
    L = tdx.lib()
    size = ctypes.c_size_t(0)
    for name in ("tdx_causal_conv1d", "tdx_causal_conv1d_bwd", "tdx_causal_conv1d_step", "tdx_selective_scan", "tdx_selective_scan_bwd",
                 "tdx_selective_scan_step", "tdx_gemm_w4"):
        assert getattr(L, name)(None, None) == INVALID
    for name in ("tdx_causal_conv1d_workspace_size", "tdx_selective_scan_workspace_size", "tdx_selective_scan_saved_size"):
        assert getattr(L, name)(None, ctypes.byref(size)) == INVALID


def test_sizes():
    st, n = tdx.tdx_selective_scan_saved_size(scan())
    assert st == tdx.TDX_OK and n >= 2 * 8 * 16 * 4                    # a state per sequence at least
    packed = scan(seq_offsets=P, rows=1000, max_len=900)
    assert tdx.tdx_selective_scan_saved_size(packed)[1] == (1000 // 8 + 2) * 8 * 16 * 4
    forward, both = tdx.tdx_selective_scan_workspace_size(scan(saved=None)), tdx.tdx_selective_scan_workspace_size(scan())
    assert forward == (tdx.TDX_OK, 0) and both[0] == tdx.TDX_OK and both[1] > 0
    assert tdx.tdx_selective_scan_workspace_size(scan(saved=None, max_len=4096, rows=8192))[1] > 0      # few channels: cut into chunks
    st, n = tdx.tdx_causal_conv1d_workspace_size(conv())
    assert st == tdx.TDX_OK and n % 256 == 0 and n >= 2 * 8 * 5 * 4


def test_blocks_take_known_fields_only():
    with pytest.raises(TypeError):
        tdx.tdx_scan_args(chanels=3)
    with pytest.raises(TypeError):
        tdx.tdx_conv1d_args(x=1.5)


def test_block_layouts_match_the_header():
    """The ctypes blocks have the header's fields in the header's order."""
    import os
    import re
    text = open(os.path.join(os.path.dirname(__file__), "..", "include", "tdx.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    for cls in (tdx.tdx_conv1d_args, tdx.tdx_scan_args, tdx.tdx_w4_args):
        body = re.findall(r"typedef struct \{([^}]*)\} " + cls.__name__, text)[0]
        names, types = [], []
        for decl in body.split(";"):
            decl = decl.strip()
            if not decl:
                continue
            kind, rest = re.match(r"((?:const )?\w+\*?)\s*(.*)", decl, flags=re.S).groups()
            for name in rest.split(","):
                names.append(name.strip())
                types.append("ptr" if "*" in kind else kind)
        size = {"ptr": 8, "int64_t": 8, "size_t": 8, "int": 4}
        assert names == [n for n, _ in cls._fields_]
        assert [size[t] for t in types] == [ctypes.sizeof(t) for _, t in cls._fields_]


def test_a_packed_batch_of_no_sequences_has_no_work():
    """Rows that belong to no sequence make no pieces: nothing may be launched for them, as the offsets have one value only."""
    empty = dict(batch=0, max_len=500, rows=1000, seq_offsets=P)
    assert tdx.tdx_causal_conv1d_workspace_size(conv(**empty)) == (tdx.TDX_OK, 0)
    assert tdx.tdx_selective_scan_saved_size(scan(**empty)) == (tdx.TDX_OK, 0)
    assert tdx.tdx_causal_conv1d(conv(**empty)) == tdx.TDX_OK
    assert tdx.tdx_causal_conv1d_bwd(conv(**empty, dweight=None, dbias=None)) == tdx.TDX_OK
    assert tdx.tdx_selective_scan(scan(**empty)) == tdx.TDX_OK


def test_slots_of_a_step_without_states_are_checked_too():
    assert tdx.tdx_causal_conv1d_step(conv(width=1, slots=P + 2, n_slots=0)) == ALIGNMENT


def test_a_generous_max_len_does_not_cut_short_sequences():
    """No sequence is longer than all rows together, so a scan of few rows needs no workspace whatever max_len allows."""
    st, n = tdx.tdx_selective_scan_workspace_size(scan(seq_offsets=P, rows=60, max_len=32768, saved=None))
    assert (st, n) == (tdx.TDX_OK, 0)
