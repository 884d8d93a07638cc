"""GPU parity of the causal convolution (forward, backward, single tokens) with its 64-bit definition."""
import numpy as np
import pytest
import torch

import paper_2409_03864_b200 as tdx
import seq_reference as ref
from seq_util import DT, EPS, TORCH, Rows, assert_close, assert_close_but_infinities, f32, i32, offsets_of, seeded, workspace

pytestmark = pytest.mark.gpu

# rounding of the filter's sum, of silu and of the products behind it, in units of EPS * magnitude
def forward_factor(width):
    return (2 * width + 12) * EPS


def backward_factor(width, terms=0):
    return (4 * width + 32 + terms) * EPS


class Problem:
    def __init__(self, dtype, width, channels, lengths, packed, silu=1, bias=True, seed=0, pad=0, lead=0, states=True, order=None):
        rng = np.random.default_rng(seed)
        self.dtype, self.width, self.d, self.silu = dtype, width, channels, silu
        self.lengths, n = list(lengths), len(lengths)
        self.offsets = offsets_of(lengths) if packed else None
        self.rows = int(sum(lengths))
        self.seqs = ref.pieces(n, max(self.lengths, default=0), self.offsets)
        self.x = seeded(rng, (self.rows, channels), dtype)
        self.weight, self.bias = seeded(rng, (channels, width), "f32", 0.5), seeded(rng, (channels,), "f32", 0.3) * bool(bias)
        self.state = seeded(rng, (n, width - 1, channels), dtype) if states else np.zeros((n, width - 1, channels))
        self.dy, self.dstate = seeded(rng, (self.rows, channels), dtype), seeded(rng, (n, width - 1, channels), dtype)
        self.slots = list(range(n)) if order is None else order
        self.n_slots = max(self.slots, default=-1) + 2
        all_states = np.full((self.n_slots, width - 1, channels), 3.0)
        for b, s in enumerate(self.slots):
            if s >= 0:
                all_states[s] = self.state[b]
            else:
                self.state[b] = 0.0
        self.all_states = all_states
        self.dev_x = Rows(self.x, dtype, pad, lead)
        self.dev_w, self.dev_b = f32(self.weight), f32(self.bias) if bias else None
        self.dev_state = Rows(all_states, dtype)
        self.dev_offsets, self.dev_slots = i32(self.offsets), None if order is None else i32(order)
        self.args = tdx.tdx_conv1d_args(
            batch=n, max_len=max(self.lengths, default=0), rows=self.rows, channels=channels, width=width, dtype=DT[dtype], silu=silu,
            x=self.dev_x.ptr, ld_x=self.dev_x.ld, weight=self.dev_w, bias=self.dev_b, seq_offsets=self.dev_offsets,
            state_in=self.dev_state.ptr if states else None, slots=self.dev_slots, n_slots=self.n_slots)

    def forward(self, pad=0, lead=0, in_place=False, stream=None):
        self.y = Rows(np.zeros((self.rows, self.d)), self.dtype, pad, lead, fill=float("nan"))
        self.new_state = self.dev_state if in_place else Rows(np.full_like(self.all_states, 5.0), self.dtype)
        self.args.set(y=self.y.ptr, ld_y=self.y.ld, state_out=self.new_state.ptr)
        tdx.check(tdx.tdx_causal_conv1d(self.args, stream))
        torch.cuda.synchronize()

    def check_forward(self):
        o = ref.conv1d(self.x, self.weight, self.bias, self.silu, self.seqs, self.state)
        m = ref.conv1d(self.x, self.weight, self.bias, self.silu, self.seqs, self.state, magnitude=True)
        assert_close("y", self.y.host(), o["y"], m["y"], forward_factor(self.width), self.dtype)
        new, old = self.new_state.host(), self.all_states if self.new_state is self.dev_state else np.full_like(self.all_states, 5.0)
        for b, s in enumerate(self.slots):
            if s >= 0:
                assert np.array_equal(new[s], o["state"][b])          # copies, bit for bit
        for s in set(range(self.n_slots)) - set(self.slots):
            assert np.array_equal(new[s], old[s])                     # no other slot is touched
        assert self.y.guards_intact() and self.new_state.guards_intact() and self.dev_x.guards_intact()
        assert tdx.tdx_check_device_status() == 0

    def backward(self, pad=0, lead=0, with_state=True):
        n = len(self.lengths)
        self.dev_dy = Rows(self.dy, self.dtype, pad)
        self.dx = Rows(np.zeros((self.rows, self.d)), self.dtype, pad, lead, fill=float("nan"))
        self.dweight, self.dbias = f32(np.full_like(self.weight, np.nan)), f32(np.full_like(self.bias, np.nan))
        given = np.zeros_like(self.all_states)
        for b, s in enumerate(self.slots):
            if s >= 0:
                given[s] = self.dstate[b]
            else:
                self.dstate[b] = 0.0
        if not with_state:
            self.dstate[:] = 0.0
        self.dev_dstate, self.dstate_in = Rows(given, self.dtype), Rows(np.zeros_like(self.all_states), self.dtype, fill=float("nan"))
        self.ws = ws = workspace(tdx.tdx_causal_conv1d_workspace_size(self.args))
        self.args.set(dy=self.dev_dy.ptr, ld_dy=self.dev_dy.ld, dx=self.dx.ptr, ld_dx=self.dx.ld, dweight=self.dweight, dbias=self.dbias,
                      dstate_out=self.dev_dstate.ptr if with_state else None, dstate_in=self.dstate_in.ptr if with_state else None,
                      workspace=ws, workspace_bytes=ws.numel())
        tdx.check(tdx.tdx_causal_conv1d_bwd(self.args))
        torch.cuda.synchronize()
        assert n == len(self.seqs)

    def check_backward(self, with_state=True):
        a = (self.x, self.weight, self.bias, self.silu, self.seqs, self.state, self.dy, self.dstate)
        o, m = ref.conv1d(*a), ref.conv1d(*a, magnitude=True)
        few, many = backward_factor(self.width), backward_factor(self.width, self.rows)
        assert_close("dx", self.dx.host(), o["dx"], m["dx"], few, self.dtype)
        assert_close("dweight", self.dweight.double().cpu().numpy(), o["dweight"], m["dweight"], many)
        assert_close("dbias", self.dbias.double().cpu().numpy(), o["dbias"], m["dbias"], many)
        if with_state:
            got = self.dstate_in.host()
            for b, s in enumerate(self.slots):
                if s >= 0:
                    assert_close("dstate", got[s], o["dstate"][b], m["dstate"][b], few, self.dtype)
        assert self.dx.guards_intact() and self.dstate_in.guards_intact()
        assert tdx.tdx_check_device_status() == 0


SHAPES = [
    # width, channels, lengths, packed
    (4, 64, [37], False),
    (4, 256, [130, 130], False),           # several runs and blocks
    (4, 7, [1, 1, 1], False),              # single tokens, odd channels
    (3, 40, [5, 0, 1, 2, 70], True),       # an empty sequence, ones shorter than the filter
    (2, 33, [0, 0, 300], True),
    (1, 8, [9, 4], True),                  # no state at all
    (5, 24, [3, 129, 0], True),            # wide filter
    (8, 12, [2, 7, 40], True),
    (4, 1, [3], False),
    (4, 1026, [64, 65], True),             # rows of 2052 bytes (bf16): 4-byte accesses
    (4, 520, [17, 300], True),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward(shape, dtype):
    width, d, lengths, packed = shape
    p = Problem(dtype, width, d, lengths, packed)
    p.forward()
    p.check_forward()
    p.backward()
    p.check_backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("silu,bias,states", [(0, True, True), (1, False, True), (1, True, False), (0, False, False)])
def test_without_activation_bias_or_states(dtype, silu, bias, states):
    p = Problem(dtype, 4, 48, [21, 2, 33], True, silu=silu, bias=bias, states=states)
    p.forward()
    p.check_forward()
    p.backward(with_state=False)
    p.check_backward(with_state=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,lead", [(64, 0), (0, 64), (3, 0), (0, 1), (2, 2)])
def test_slices_of_wider_tensors(dtype, pad, lead):
    p = Problem(dtype, 4, 64, [40, 25], True, pad=pad, lead=lead)
    p.forward(pad, lead)
    p.check_forward()
    p.backward(pad, lead)
    p.check_backward()


@pytest.mark.parametrize("in_place", [False, True])
def test_states_in_slots(in_place):
    p = Problem("bf16", 4, 72, [2, 0, 140, 1, 3], True, order=[5, 2, 0, -1, 3])
    p.forward(in_place=in_place)
    p.check_forward()
    if not in_place:
        p.backward()
        p.check_backward()


def test_long_sequence_in_place_and_continued_from_its_state():
    """Two halves, the second from the state of the first, give the bits of the whole."""
    whole = Problem("bf16", 4, 128, [600], False, states=False)
    whole.forward()
    x = whole.dev_x
    state = torch.zeros(1, 3, 128, dtype=torch.bfloat16, device="cuda")
    y = torch.empty(600, 128, dtype=torch.bfloat16, device="cuda")
    for lo, hi in ((0, 1), (1, 258), (258, 600)):
        a = tdx.tdx_conv1d_args(batch=1, max_len=hi - lo, rows=hi - lo, channels=128, width=4, dtype=tdx.TDX_BF16, silu=1, x=x.view[lo:], ld_x=x.ld,
                                weight=whole.dev_w, bias=whole.dev_b, y=y[lo:], ld_y=128, state_in=state, state_out=state, n_slots=1)
        tdx.check(tdx.tdx_causal_conv1d(a))
    torch.cuda.synchronize()
    assert torch.equal(y, whole.y.view)
    assert torch.equal(state[0], x.view[-3:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width,d", [(4, 64), (4, 129), (2, 1000), (3, 30), (1, 16), (6, 10), (8, 8)])
@pytest.mark.parametrize("in_place", [False, True])
def test_single_tokens_equal_a_sequence(width, d, dtype, in_place):
    """Steps one token at a time give the bits of the forward pass over the sequence, whichever slots the states are in."""
    rng = np.random.default_rng(3)
    batch, length, slots = 5, 6, [4, 0, 6, 2, 5]
    p = Problem(dtype, width, d, [length] * batch, False, states=False)
    p.forward()
    state = [Rows(np.zeros((7, width - 1, d)), dtype) for _ in range(2)]
    y = Rows(np.zeros((batch, d)), dtype, 1)
    for t in range(length):
        now, after = (state[0], state[0]) if in_place else (state[t % 2], state[1 - t % 2])
        x = Rows(p.x.reshape(batch, length, d)[:, t], dtype, 2)
        a = tdx.tdx_conv1d_args(batch=batch, channels=d, width=width, dtype=DT[dtype], silu=1, x=x.ptr, ld_x=x.ld, weight=p.dev_w, bias=p.dev_b, y=y.ptr,
                                ld_y=y.ld, state_in=now.ptr, state_out=after.ptr, slots=i32(slots), n_slots=7)
        tdx.check(tdx.tdx_causal_conv1d_step(a))
        torch.cuda.synchronize()
        assert np.array_equal(y.host(), p.y.host().reshape(batch, length, d)[:, t])
    assert np.array_equal(after.host()[slots], p.new_state.host()[:batch])
    assert y.guards_intact() and all(s.guards_intact() for s in state)
    assert rng is not None


def test_padding_rows_of_a_step_and_slots_out_of_range():
    d, width = 40, 4
    state = Rows(np.ones((3, width - 1, d)), "f32")
    state.view[1] = float("nan")                          # the slot of nobody
    x, y = Rows(np.full((4, d), np.nan), "f32"), Rows(np.zeros((4, d)), "f32", fill=float("nan"))
    x.view[0] = 2.0
    w = f32(np.ones((d, width)))
    a = tdx.tdx_conv1d_args(batch=4, channels=d, width=width, dtype=tdx.TDX_F32, silu=0, x=x.ptr, ld_x=x.ld, weight=w, y=y.ptr, ld_y=y.ld,
                            state_in=state.ptr, state_out=state.ptr, slots=i32([2, -1, -7, -1]), n_slots=3)
    tdx.check(tdx.tdx_causal_conv1d_step(a))
    torch.cuda.synchronize()
    assert np.array_equal(y.host(), np.repeat([[5.0], [0.0], [0.0], [0.0]], d, axis=1))
    assert np.array_equal(state.host()[2], np.repeat([[1.0], [1.0], [2.0]], d, axis=1)) and (state.host()[0] == 1).all()
    assert np.isnan(state.host()[1]).all() and tdx.tdx_check_device_status() == 0
    a.set(slots=i32([0, 3, 2, -1]))
    tdx.check(tdx.tdx_causal_conv1d_step(a))
    assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
    assert tdx.tdx_check_device_status() == 0
    assert (y.host()[1] == 0).all()                       # treated as padding


def test_what_lies_outside_the_sequences_is_neither_read_nor_written():
    """Rows in front of, between (none) and behind the sequences hold NaN and infinity."""
    d = 64
    x = np.zeros((30, d))
    x[:4], x[25:] = np.nan, np.inf
    rng = np.random.default_rng(1)
    x[4:25] = rng.standard_normal((21, d))
    dev_x, y = Rows(x, "f32"), Rows(np.full((30, d), 9.0), "f32")
    dx, dy = Rows(np.full((30, d), 9.0), "f32"), Rows(np.where(np.isfinite(x), 1.0, np.nan), "f32")
    w, offsets = rng.standard_normal((d, 4)).astype(np.float32), [4, 10, 10, 25]
    dweight = f32(np.zeros((d, 4)))
    keep = f32(w), i32(offsets)
    a = tdx.tdx_conv1d_args(batch=3, max_len=15, rows=30, channels=d, width=4, dtype=tdx.TDX_F32, silu=1, x=dev_x.ptr, ld_x=d, weight=keep[0], y=y.ptr,
                            ld_y=d, seq_offsets=keep[1], dy=dy.ptr, ld_dy=d, dx=dx.ptr, ld_dx=d, dweight=dweight)
    ws = workspace(tdx.tdx_causal_conv1d_workspace_size(a))
    a.set(workspace=ws, workspace_bytes=ws.numel())
    tdx.check(tdx.tdx_causal_conv1d(a))
    tdx.check(tdx.tdx_causal_conv1d_bwd(a))
    torch.cuda.synchronize()
    seqs = [(4, 6), (10, 0), (10, 15)]
    clean = np.where(np.isfinite(x), x, 0.0)
    args = (clean, w.astype(np.float64), np.zeros(d), 1, seqs, np.zeros((3, 3, d)), np.ones((30, d)))
    o, m = ref.conv1d(*args), ref.conv1d(*args, magnitude=True)
    inside = slice(4, 25)
    assert_close("y", y.host()[inside], o["y"][inside], m["y"][inside], forward_factor(4))
    assert_close("dx", dx.host()[inside], o["dx"][inside], m["dx"][inside], backward_factor(4))
    assert_close("dweight", dweight.double().cpu().numpy(), o["dweight"], m["dweight"], backward_factor(4, 21))
    for t in (y, dx):
        assert (t.host()[:4] == 9).all() and (t.host()[25:] == 9).all()


def test_bad_offsets_are_reported_and_their_sequences_skipped():
    d = 32
    x, y = Rows(np.ones((10, d)), "f32"), Rows(np.full((10, d), 9.0), "f32")
    w = f32(np.ones((d, 2)))
    for offsets, good in (([0, 4, 11], slice(0, 4)), ([0, 4, 3], slice(0, 4)), ([0, 9, 10], slice(9, 10)), ([-2, 4, 8], slice(4, 8))):
        y.view[:] = 9.0
        o = i32(offsets)
        a = tdx.tdx_conv1d_args(batch=2, max_len=6, rows=10, channels=d, width=2, dtype=tdx.TDX_F32, silu=0, x=x.ptr, ld_x=d, weight=w, y=y.ptr, ld_y=d,
                                seq_offsets=o)
        tdx.check(tdx.tdx_causal_conv1d(a))
        assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
        got = y.host()
        assert (got[good] != 9).all()
        rest = np.ones(10, dtype=bool)
        rest[good] = False
        assert (got[rest] == 9).all()


def test_same_bits_every_time_and_on_another_stream():
    p = Problem("bf16", 4, 200, [300, 3, 90], True)
    p.forward()
    p.backward()
    first = [t.clone() for t in (p.y.view, p.dx.view, p.dweight, p.dbias)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.dev_x.view[:] = p.dev_x.view * 1.0              # work in front of the call on its own stream
        tdx.check(tdx.tdx_causal_conv1d(p.args, side))
        tdx.check(tdx.tdx_causal_conv1d_bwd(p.args, side))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, (p.y.view, p.dx.view, p.dweight, p.dbias)))


def test_empty_problems():
    p = Problem("f32", 4, 16, [0, 0, 0], True)
    p.forward()
    p.check_forward()
    p.backward()
    p.check_backward()
    assert (p.dweight == 0).all() and (p.dbias == 0).all()


def test_backward_of_a_packed_batch_of_no_sequences():
    """The parameters' gradients are zero, and rows that belong to no sequence stay what they are."""
    d, rows = 32, 1000
    x, dy, dx = Rows(np.full((rows, d), np.nan), "f32"), Rows(np.full((rows, d), np.nan), "f32"), Rows(np.full((rows, d), 9.0), "f32")
    w, offsets, dweight, dbias = f32(np.ones((d, 4))), i32([0]), f32(np.full((d, 4), np.nan)), f32(np.full(d, np.nan))
    a = tdx.tdx_conv1d_args(batch=0, max_len=500, rows=rows, channels=d, width=4, dtype=tdx.TDX_F32, silu=1, x=x.ptr, ld_x=d, weight=w, seq_offsets=offsets,
                            dy=dy.ptr, ld_dy=d, dx=dx.ptr, ld_dx=d, dweight=dweight, dbias=dbias)
    assert tdx.tdx_causal_conv1d_workspace_size(a) == (tdx.TDX_OK, 0)
    tdx.check(tdx.tdx_causal_conv1d_bwd(a))
    assert tdx.tdx_check_device_status() == 0
    assert (dweight == 0).all() and (dbias == 0).all() and (dx.host() == 9).all() and dx.guards_intact()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_single_tokens_of_width_one_need_neither_states_nor_slots(dtype):
    rng = np.random.default_rng(8)
    batch, d = 5, 24
    v, w, bias = seeded(rng, (batch, d), dtype), seeded(rng, (d, 1), "f32"), seeded(rng, (d,), "f32")
    x, y, dev_w, dev_b = Rows(v, dtype), Rows(np.zeros((batch, d)), dtype, fill=float("nan")), f32(w), f32(bias)
    a = tdx.tdx_conv1d_args(batch=batch, channels=d, width=1, dtype=DT[dtype], silu=1, x=x.ptr, ld_x=d, weight=dev_w, bias=dev_b, y=y.ptr, ld_y=d)
    tdx.check(tdx.tdx_causal_conv1d_step(a))
    assert tdx.tdx_check_device_status() == 0
    seqs, none = [(i, 1) for i in range(batch)], np.zeros((batch, 0, d))
    o, m = ref.conv1d(v, w, bias, 1, seqs, none), ref.conv1d(v, w, bias, 1, seqs, none, magnitude=True)
    assert_close("y", y.host(), o["y"], m["y"], forward_factor(1), dtype)
    # slots only tell which rows are padding
    slots = i32([7, -1, 0, 900, -3])
    a.set(slots=slots)
    tdx.check(tdx.tdx_causal_conv1d_step(a))
    assert tdx.tdx_check_device_status() == 0
    there = np.array([1, 0, 1, 1, 0])[:, None]
    assert_close("y", y.host(), o["y"] * there, m["y"] * there, forward_factor(1), dtype)


@pytest.mark.parametrize("offsets", [[0, 1000, 500, 2000], [0, 5000, 100, 2000], [0, 2000, -7, 1500], [1990, 3, 1000, 900]])
def test_offsets_that_do_not_ascend_are_reported(offsets):
    """Each call reports them, wherever they stand, and writes only into its tensors."""
    d, rows = 32, 2000
    x, y, dx = Rows(np.ones((rows, d)), "f32"), Rows(np.zeros((rows, d)), "f32", 3), Rows(np.zeros((rows, d)), "f32", 3)
    w, off, dweight = f32(np.ones((d, 4))), i32(offsets), f32(np.zeros((d, 4)))
    a = tdx.tdx_conv1d_args(batch=3, max_len=rows, rows=rows, channels=d, width=4, dtype=tdx.TDX_F32, silu=1, x=x.ptr, ld_x=x.ld, weight=w, y=y.ptr, ld_y=y.ld,
                            seq_offsets=off, dy=x.ptr, ld_dy=x.ld, dx=dx.ptr, ld_dx=dx.ld, dweight=dweight)
    ws = workspace(tdx.tdx_causal_conv1d_workspace_size(a))
    a.set(workspace=ws, workspace_bytes=ws.numel())
    tdx.check(tdx.tdx_causal_conv1d(a))
    assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
    tdx.check(tdx.tdx_causal_conv1d_bwd(a))
    assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
    assert x.guards_intact() and y.guards_intact() and dx.guards_intact()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", [2, 4, 6])
@pytest.mark.parametrize("where,value", [("x", np.inf), ("x", -np.inf), ("x", np.nan), ("dy", np.inf), ("state", np.inf)])
@pytest.mark.parametrize("silu", [0, 1])
def test_infinities_reach_the_rows_of_their_filter_only(silu, where, value, width, dtype):
    p = Problem(dtype, width, 36, [70, 9], True, silu=silu)
    {"x": p.x, "dy": p.dy, "state": p.state.reshape(-1, 36)}[where][1 if where == "state" and width > 2 else 0 if where == "state" else 33, 3] = value
    p.dev_x.view[:] = torch.from_numpy(p.x).cuda().to(TORCH[dtype])
    p.all_states[:2] = p.state
    p.dev_state.view[:] = torch.from_numpy(p.all_states.reshape(p.n_slots, -1)).cuda().to(TORCH[dtype])
    with np.errstate(all="ignore"):
        a = (p.x, p.weight, p.bias, silu, p.seqs, p.state)
        o, m = ref.conv1d(*a, p.dy, p.dstate), ref.conv1d(*a, p.dy, p.dstate, magnitude=True)
        if not silu:                                     # dx, dbias and dstate do not depend on x then, but the helper's sizes have 0 * |pre|
            clean = [np.where(np.isfinite(v), v, 0.0) for v in (p.x, p.state)]
            sizes = ref.conv1d(clean[0], p.weight, p.bias, silu, p.seqs, clean[1], p.dy, p.dstate, magnitude=True)
            m |= {k: sizes[k] for k in ("dx", "dbias", "dstate")} | {"dweight": np.where(np.isnan(m["dweight"]), sizes["dweight"], m["dweight"])}
        p.forward()
        p.backward()
        got = {"y": p.y.host(), "dx": p.dx.host(), "dweight": p.dweight.double().cpu().numpy(), "dbias": p.dbias.double().cpu().numpy(),
               "state": p.new_state.host()[:2], "dstate": p.dstate_in.host()[:2]}
        for k, v in got.items():
            factor = forward_factor(width) if k == "y" else backward_factor(width, p.rows if k in ("dweight", "dbias") else 0)
            assert_close_but_infinities(k, v, o[k], m[k], factor, "f32" if k in ("dweight", "dbias") else dtype)
    assert tdx.tdx_check_device_status() == 0
