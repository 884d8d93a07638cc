"""GPU parity of the selective scan (forward, backward, single tokens) with its 64-bit definition."""
import numpy as np
import pytest
import torch

import paper_2409_03864_b200 as tdx
import seq_reference as ref
from seq_util import DT, EPS, TORCH, Rows, assert_close, assert_close_but_infinities, f32, i32, offsets_of, seeded, workspace

pytestmark = pytest.mark.gpu


def factors(longest, states, channels, rows, reach):
    """What rounding may do, in units of the sums' magnitudes.  A decay is off by 2^-22 (the exponential) and by |dt' A| <= reach times
    the 10 EPS of dt' A; a state carries the errors of at most `longest` of them.  Gradients carry those of h, dh and y."""
    decay = longest * (2.0 ** -22 + 10 * reach * EPS)
    forward = decay + (longest + states + 24) * EPS
    return {"out": forward, "state": forward, "grad": 3 * forward, "over_channels": 3 * forward + channels * EPS, "over_rows": 3 * forward + rows * EPS}


class Problem:
    def __init__(self, dtype, states, channels, lengths, packed, groups=1, softplus=1, z=True, D=True, bias=True, with_states=True, seed=0, pad=0,
                 lead=0, order=None):
        rng = np.random.default_rng(seed)
        n, d, rows = states, channels, int(sum(lengths))
        self.dtype, self.n, self.d, self.rows, self.groups, self.softplus = dtype, n, d, rows, groups, softplus
        self.lengths, batch = list(lengths), len(lengths)
        longest = max(self.lengths, default=0)
        self.offsets = offsets_of(lengths) if packed else None
        seqs = ref.pieces(batch, longest, self.offsets)
        self.v = {
            "x": seeded(rng, (rows, d), dtype), "dt": seeded(rng, (rows, d), dtype, 0.5) if softplus else seeded(rng, (rows, d), dtype, lo=0.01, hi=0.3),
            "A": -seeded(rng, (d, n), "f32", lo=0.1, hi=4.0), "B": seeded(rng, (rows, groups * n), dtype), "C": seeded(rng, (rows, groups * n), dtype),
            "D": seeded(rng, (d,), "f32") * bool(D), "z": seeded(rng, (rows, d), dtype) if z else None,
            "dt_bias": (seeded(rng, (d,), "f32", lo=-5.0, hi=-1.0) if softplus else seeded(rng, (d,), "f32", lo=0.0, hi=0.1)) * bool(bias),
            "use_softplus": softplus, "groups": groups, "seqs": seqs, "state": seeded(rng, (batch, d, n), "f32") if with_states else np.zeros((batch, d, n))}
        v = self.v
        self.dout, self.dstate = seeded(rng, (rows, d), dtype), seeded(rng, (batch, d, n), "f32")
        self.slots = list(range(batch)) if order is None else order
        self.n_slots = max(self.slots, default=-1) + 2
        self.all_states = np.full((self.n_slots, d, n), 3.0)
        for b, s in enumerate(self.slots):
            if s >= 0:
                self.all_states[s] = v["state"][b]
            else:
                v["state"][b] = 0.0
        step = ref.softplus(v["dt"] + v["dt_bias"]) if softplus else np.abs(v["dt"] + v["dt_bias"])
        reach = float((step.max(0)[:, None] * np.abs(v["A"])).max()) if rows else 1.0
        self.f = factors(longest, n, d, rows, reach)
        self.dev = {k: Rows(v[k], dtype, pad, lead) for k in ("x", "dt", "B", "C") + (("z",) if z else ())}
        self.par = {k: f32(v[k]) for k in ("A",) + (("D",) if D else ()) + (("dt_bias",) if bias else ())}
        self.dev_state = Rows(self.all_states, "f32")
        self.dev_offsets, self.dev_slots = i32(self.offsets), None if order is None else i32(order)
        self.args = tdx.tdx_scan_args(
            batch=batch, max_len=longest, rows=rows, channels=d, states=n, groups=groups, dtype=DT[dtype], dt_softplus=softplus,
            **{k: t.ptr for k, t in self.dev.items()}, **{"ld_" + k: t.ld for k, t in self.dev.items()}, **self.par, seq_offsets=self.dev_offsets,
            state_in=self.dev_state.ptr if with_states else None, slots=self.dev_slots, n_slots=self.n_slots)

    def forward(self, pad=0, lead=0, in_place=False, save=False):
        self.out = Rows(np.zeros((self.rows, self.d)), self.dtype, pad, lead, fill=float("nan"))
        self.new_state = self.dev_state if in_place else Rows(np.full_like(self.all_states, 5.0), "f32")
        self.args.set(out=self.out.ptr, ld_out=self.out.ld, state_out=self.new_state.ptr)
        if save:
            self.saved = workspace(tdx.tdx_selective_scan_saved_size(self.args))
            self.args.set(saved=self.saved, saved_bytes=self.saved.numel())
        self.ws = workspace(tdx.tdx_selective_scan_workspace_size(self.args))
        self.args.set(workspace=self.ws, workspace_bytes=self.ws.numel())
        tdx.check(tdx.tdx_selective_scan(self.args))
        torch.cuda.synchronize()

    def check_forward(self):
        o, m = ref.scan(**self.v), ref.scan(**self.v, magnitude=True)
        assert_close("out", self.out.host(), o["out"], m["out"], self.f["out"], self.dtype)
        new, old = self.new_state.host(), self.all_states if self.new_state is self.dev_state else np.full_like(self.all_states, 5.0)
        for b, s in enumerate(self.slots):
            if s >= 0:
                assert_close("state", new[s], o["state"][b], m["state"][b], self.f["state"])
        for s in set(range(self.n_slots)) - set(self.slots):
            assert np.array_equal(new[s], old[s])
        assert self.out.guards_intact() and self.new_state.guards_intact()
        assert tdx.tdx_check_device_status() == 0

    def backward(self, pad=0, lead=0, with_state=True):
        g = self.groups * self.n
        shape = {"dx": self.d, "ddt": self.d, "dB": g, "dC": g} | ({"dz": self.d} if "z" in self.dev else {})
        self.g = {k: Rows(np.zeros((self.rows, w)), self.dtype, pad, lead, fill=float("nan")) for k, w in shape.items()}
        self.p = {"dA": f32(np.full((self.d, self.n), np.nan)), "dD": f32(np.full(self.d, np.nan)), "ddt_bias": f32(np.full(self.d, np.nan))}
        given = np.zeros_like(self.all_states)
        for b, s in enumerate(self.slots):
            if s >= 0:
                given[s] = self.dstate[b]
            else:
                self.dstate[b] = 0.0
        if not with_state:
            self.dstate[:] = 0.0
        self.dev_dout, self.dev_dstate = Rows(self.dout, self.dtype, pad), Rows(given, "f32")
        self.dstate_in = Rows(np.zeros_like(self.all_states), "f32", fill=float("nan"))
        self.args.set(dout=self.dev_dout.ptr, ld_dout=self.dev_dout.ld, **{k: t.ptr for k, t in self.g.items()},
                      **{"ld_" + k: t.ld for k, t in self.g.items()}, **self.p, dstate_out=self.dev_dstate.ptr if with_state else None,
                      dstate_in=self.dstate_in.ptr if with_state else None)
        self.ws.fill_(0xFF)
        tdx.check(tdx.tdx_selective_scan_bwd(self.args))
        torch.cuda.synchronize()

    def check_backward(self, with_state=True):
        extra = {"dout": self.dout, "dstate": self.dstate}
        o, m = ref.scan(**self.v, **extra), ref.scan(**self.v, **extra, magnitude=True)
        kind = {"dx": "grad", "ddt": "grad", "dz": "grad", "dB": "over_channels", "dC": "over_channels"}
        for k, t in self.g.items():
            assert_close(k, t.host(), o[k], m[k], self.f[kind[k]], self.dtype)
            assert t.guards_intact(), k
        for k, t in self.p.items():
            assert_close(k, t.double().cpu().numpy(), o[k], m[k], self.f["over_rows"])
        if with_state:
            got = self.dstate_in.host()
            for b, s in enumerate(self.slots):
                if s >= 0:
                    assert_close("dstate", got[s], o["dstate"][b], m["dstate"][b], self.f["grad"])
            for s in set(range(self.n_slots)) - set(self.slots):
                assert np.isnan(got[s]).all()
        assert tdx.tdx_check_device_status() == 0


SHAPES = [
    # states, channels, lengths, packed, groups
    (16, 64, [37], False, 1),
    (16, 32, [8, 8], False, 1),              # one backward tile, one channel tile
    (16, 33, [9, 1, 0, 70], True, 1),        # odd channels, an empty sequence
    (16, 40, [300], False, 1),               # cut into chunks: few channels, a long sequence
    (16, 48, [200, 0, 3, 150], True, 2),     # cut, packed, two groups
    (4, 130, [33, 20], True, 1),
    (3, 10, [1, 1, 1], False, 1),            # single tokens, states that do not fill a thread
    (8, 96, [65, 64], True, 3),
    (1, 5, [40], False, 5),                  # one state, a group per channel
    (20, 24, [31], False, 1),
    (64, 12, [70, 2], True, 2),
    (128, 6, [40], False, 1),
    (100, 9, [3, 129], True, 3),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward(shape, dtype):
    n, d, lengths, packed, groups = shape
    p = Problem(dtype, n, d, lengths, packed, groups)
    p.forward(save=True)
    p.check_forward()
    p.backward()
    p.check_backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("without", ["z", "D", "bias", "softplus", "states", "all"])
def test_optional_parts(dtype, without):
    off = lambda k: without not in (k, "all")  # noqa: E731
    p = Problem(dtype, 16, 72, [50, 0, 21], True, softplus=int(off("softplus")), z=off("z"), D=off("D"), bias=off("bias"), with_states=off("states"))
    p.forward(save=True)
    p.check_forward()
    p.backward(with_state=off("states"))
    p.check_backward(with_state=off("states"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,lead", [(32, 0), (0, 32), (3, 0), (0, 1)])
def test_slices_of_wider_tensors(dtype, pad, lead):
    p = Problem(dtype, 16, 64, [40, 25], True, pad=pad, lead=lead)
    p.forward(pad, lead, save=True)
    p.check_forward()
    p.backward(pad, lead)
    p.check_backward()


@pytest.mark.parametrize("lengths", [[2, 0, 60, 1, 3], [200, 0, 260, 1, 3]])
@pytest.mark.parametrize("in_place", [False, True])
def test_states_in_slots(in_place, lengths):
    p = Problem("f32", 16, 40, lengths, True, order=[5, 2, 0, -1, 3])
    p.forward(in_place=in_place, save=True)
    p.check_forward()
    if not in_place:
        p.backward()
        p.check_backward()


def test_a_forward_pass_that_saves_nothing_gives_the_same_bits():
    p = Problem("bf16", 16, 64, [100, 31], True)
    p.forward()
    first = p.out.view.clone(), p.new_state.view.clone()
    p.forward(save=True)
    assert torch.equal(first[0], p.out.view) and torch.equal(first[1], p.new_state.view)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,groups", [(16, 64, 1), (16, 37, 1), (5, 33, 3), (1, 16, 1), (8, 100, 2), (32, 40, 1), (128, 8, 1), (64, 7, 7)])
@pytest.mark.parametrize("in_place", [False, True])
def test_single_tokens_follow_a_sequence(n, d, groups, dtype, in_place):
    batch, length, slots = 4, 5, [4, 0, 6, 2]
    p = Problem(dtype, n, d, [length] * batch, False, groups, with_states=False)
    o, m = ref.scan(**p.v), ref.scan(**p.v, magnitude=True)
    state = [Rows(np.zeros((7, d, n)), "f32") for _ in range(2)]
    out = Rows(np.zeros((batch, d)), dtype, 1)
    order = i32(slots)
    for t in range(length):
        now, after = (state[0], state[0]) if in_place else (state[t % 2], state[1 - t % 2])
        rows = {k: Rows(p.v[k].reshape(batch, length, -1)[:, t], dtype, 1) for k in ("x", "dt", "B", "C", "z")}
        a = tdx.tdx_scan_args(batch=batch, channels=d, states=n, groups=groups, dtype=DT[dtype], dt_softplus=1, **{k: r.ptr for k, r in rows.items()},
                              **{"ld_" + k: r.ld for k, r in rows.items()}, **p.par, out=out.ptr, ld_out=out.ld, state_in=now.ptr, state_out=after.ptr,
                              slots=order, n_slots=7)
        tdx.check(tdx.tdx_selective_scan_step(a))
        torch.cuda.synchronize()
        assert_close("out", out.host(), o["out"].reshape(batch, length, d)[:, t], m["out"].reshape(batch, length, d)[:, t], p.f["out"], dtype)
    assert_close("state", after.host()[slots], o["state"], m["state"], p.f["state"])
    assert out.guards_intact() and all(s.guards_intact() for s in state) and tdx.tdx_check_device_status() == 0


def test_padding_rows_of_a_step_and_slots_out_of_range():
    d, n = 40, 16
    state = Rows(np.ones((3, d, n)), "f32")
    state.view[1] = float("nan")
    rows = {k: Rows(np.full((4, w), np.nan), "f32") for k, w in (("x", d), ("dt", d), ("B", n), ("C", n))}
    for r in rows.values():
        r.view[0] = 1.0
    out = Rows(np.zeros((4, d)), "f32", fill=float("nan"))
    A, slots = f32(np.zeros((d, n))), i32([2, -1, -7, -1])
    a = tdx.tdx_scan_args(batch=4, channels=d, states=n, groups=1, dtype=tdx.TDX_F32, dt_softplus=0, **{k: r.ptr for k, r in rows.items()},
                          **{"ld_" + k: r.ld for k, r in rows.items()}, A=A, out=out.ptr, ld_out=d, state_in=state.ptr, state_out=state.ptr, slots=slots,
                          n_slots=3)
    tdx.check(tdx.tdx_selective_scan_step(a))
    torch.cuda.synchronize()
    assert (out.host()[0] == 2 * n).all() and (out.host()[1:] == 0).all()
    assert (state.host()[2] == 2).all() and (state.host()[0] == 1).all() and np.isnan(state.host()[1]).all()
    assert tdx.tdx_check_device_status() == 0
    slots2 = i32([0, 3, 2, -1])
    a.set(slots=slots2)
    tdx.check(tdx.tdx_selective_scan_step(a))
    assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
    assert (out.host()[1] == 0).all()


@pytest.mark.parametrize("long", [False, True])
def test_what_lies_outside_the_sequences_is_neither_read_nor_written(long):
    k = 150 if long else 15
    lengths, front, back = [6, 0, k], 4, 5
    inner = Problem("f32", 16, 40, lengths, True, with_states=False)
    rows = front + inner.rows + back
    offsets = offsets_of(lengths) + front

    def widened(v, fill):
        w = np.full((rows, v.shape[1]), fill)
        w[front:front + inner.rows] = v
        return Rows(w, "f32")

    dev = {key: widened(inner.v[key], np.nan) for key in ("x", "dt", "B", "C", "z")}
    dout = widened(inner.dout, np.inf)
    outs = {key: widened(np.full((inner.rows, w), 9.0), 9.0) for key, w in
            (("out", 40), ("dx", 40), ("ddt", 40), ("dz", 40), ("dB", 16), ("dC", 16))}
    par = {key: f32(np.full(s, np.nan)) for key, s in (("dA", (40, 16)), ("dD", 40), ("ddt_bias", 40))}
    off = i32(offsets)
    a = tdx.tdx_scan_args(batch=3, max_len=max(lengths), rows=rows, channels=40, states=16, groups=1, dtype=tdx.TDX_F32, dt_softplus=1, seq_offsets=off,
                          **{key: t.ptr for key, t in {**dev, **outs, "dout": dout}.items()},
                          **{"ld_" + key: t.ld for key, t in {**dev, **outs, "dout": dout}.items()}, **inner.par, **par)
    saved = workspace(tdx.tdx_selective_scan_saved_size(a))
    a.set(saved=saved, saved_bytes=saved.numel())
    ws = workspace(tdx.tdx_selective_scan_workspace_size(a))
    a.set(workspace=ws, workspace_bytes=ws.numel())
    tdx.check(tdx.tdx_selective_scan(a))
    tdx.check(tdx.tdx_selective_scan_bwd(a))
    torch.cuda.synchronize()
    o, m = ref.scan(**inner.v, dout=inner.dout), ref.scan(**inner.v, dout=inner.dout, magnitude=True)
    for key, t in outs.items():
        got = t.host()
        factor = inner.f["out" if key == "out" else "over_channels" if key in ("dB", "dC") else "grad"]
        assert_close(key, got[front:front + inner.rows], o[key], m[key], factor)
        assert (got[:front] == 9).all() and (got[front + inner.rows:] == 9).all(), key
    for key, t in par.items():
        assert_close(key, t.double().cpu().numpy(), o[key], m[key], inner.f["over_rows"])


def test_bad_offsets_are_reported_and_their_sequences_skipped():
    d, n = 32, 16
    rows = {k: Rows(np.ones((10, w)), "f32") for k, w in (("x", d), ("dt", d), ("B", n), ("C", n))}
    out = Rows(np.full((10, d), 9.0), "f32")
    A = f32(np.zeros((d, n)))
    for offsets, good in (([0, 4, 11], slice(0, 4)), ([0, 4, 3], slice(0, 4)), ([0, 9, 10], slice(9, 10)), ([-2, 4, 8], slice(4, 8))):
        out.view[:] = 9.5
        off = i32(offsets)
        a = tdx.tdx_scan_args(batch=2, max_len=6, rows=10, channels=d, states=n, groups=1, dtype=tdx.TDX_F32, dt_softplus=0,
                              **{k: r.ptr for k, r in rows.items()}, **{"ld_" + k: r.ld for k, r in rows.items()}, A=A, out=out.ptr, ld_out=d, seq_offsets=off)
        tdx.check(tdx.tdx_selective_scan(a))
        assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
        got, rest = out.host(), np.ones(10, dtype=bool)
        rest[good] = False
        assert (got[good] != 9.5).all() and (got[rest] == 9.5).all()


def test_extreme_steps():
    """A step so long that the state is forgotten, one of zero (an exact copy of the state), and decays that underflow."""
    d, n = 32, 16
    rng = np.random.default_rng(5)
    dt = np.zeros((3, d))
    dt[1] = 1e4                                             # exp(-1e4 * A) = 0
    v = {"x": rng.standard_normal((3, d)), "dt": dt, "B": rng.standard_normal((3, n)), "C": rng.standard_normal((3, n))}
    v["x"][1] *= 1e-4
    rows = {k: Rows(t, "f32") for k, t in v.items()}
    out, state, A = Rows(np.zeros((3, d)), "f32"), Rows(np.ones((1, d, n)), "f32"), f32(-rng.uniform(0.5, 2, (d, n)))
    a = tdx.tdx_scan_args(batch=1, max_len=3, rows=3, channels=d, states=n, groups=1, dtype=tdx.TDX_F32, dt_softplus=0,
                          **{k: r.ptr for k, r in rows.items()}, **{"ld_" + k: r.ld for k, r in rows.items()}, A=A, out=out.ptr, ld_out=d,
                          state_in=state.ptr, state_out=state.ptr, n_slots=1)
    tdx.check(tdx.tdx_selective_scan(a))
    torch.cuda.synchronize()
    f = {k: r.host() for k, r in rows.items()}
    assert np.allclose(out.host()[0], f["C"][0].sum(), rtol=0, atol=1e-5)
    want = (f["dt"][1] * f["x"][1])[:, None] * f["B"][1]
    assert np.allclose(state.host()[0], want, rtol=1e-6, atol=0)
    assert np.allclose(out.host()[2], (want * f["C"][2]).sum(1), rtol=1e-5, atol=1e-5)


def test_gradients_against_differences_of_the_forward_pass():
    """Central differences of the fp32 forward pass: a step of 1e-2 leaves a truncation error of about 1e-4 of the sums' size and a
    rounding error of about 1e-5 / 1e-2."""
    p = Problem("f32", 16, 48, [60], False, with_states=False)
    p.forward(save=True)
    p.backward(with_state=False)
    rng = np.random.default_rng(9)
    grads = {k[1:]: t.host() for k, t in p.g.items()} | {k[1:]: t.double().cpu().numpy() for k, t in p.p.items()}
    for name in ("x", "dt", "B", "C", "z", "A", "D", "dt_bias"):
        direction = rng.standard_normal(p.v[name].shape)
        direction *= 1e-2 / np.sqrt(np.mean(direction ** 2))
        buf = p.dev[name].view if name in p.dev else p.par[name]
        kept, sums = buf.clone(), []
        for sign in (1, -1):
            buf[:] = kept + torch.from_numpy(sign * direction.reshape(tuple(buf.shape))).cuda().float()
            tdx.check(tdx.tdx_selective_scan(p.args))
            torch.cuda.synchronize()
            sums.append((p.out.host() * p.dout).sum())
        buf[:] = kept
        want, got = (sums[0] - sums[1]) / 2, (grads[name] * direction).sum()
        size = np.sqrt(((grads[name] * direction) ** 2).sum())
        assert abs(got - want) < 2e-2 * max(size, abs(want)), (name, got, want)


def test_same_bits_every_time_on_another_stream_and_in_a_graph():
    p = Problem("bf16", 16, 64, [300, 3, 90], True)
    p.forward(save=True)
    p.backward()
    outs = [p.out.view, *(t.view for t in p.g.values()), *p.p.values()]
    first = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.dev["x"].view[:] = p.dev["x"].view * 1.0
        tdx.check(tdx.tdx_selective_scan(p.args, side))
        tdx.check(tdx.tdx_selective_scan_bwd(p.args, side))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        stream = torch.cuda.current_stream()
        tdx.check(tdx.tdx_selective_scan(p.args, stream))
        tdx.check(tdx.tdx_selective_scan_bwd(p.args, stream))
    for t in outs:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs))


def test_empty_problems():
    p = Problem("f32", 16, 16, [0, 0, 0], True)
    p.forward(save=True)
    p.check_forward()
    p.backward()
    p.check_backward()
    assert all((t == 0).all() for t in p.p.values())


@pytest.mark.parametrize("groups", [1, 2])
def test_rows_of_a_rejected_sequence_get_no_gradients(groups):
    """A sequence in the middle is longer than max_len: everything else is as if it were not there, and its rows stay what they are."""
    lengths, d, n = [40, 300, 50], 40, 16
    p = Problem("f32", n, d, lengths, True, groups, with_states=False)
    p.args.set(max_len=100)
    p.v["seqs"] = [p.v["seqs"][0], (40, 0), p.v["seqs"][2]]
    p.forward(save=True)
    assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
    p.backward(with_state=False)
    assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
    o, m = ref.scan(**p.v, dout=p.dout), ref.scan(**p.v, dout=p.dout, magnitude=True)
    inside = np.r_[0:40, 340:390]
    for k, t in {"out": p.out, **p.g}.items():
        factor = p.f["out" if k == "out" else "over_channels" if k in ("dB", "dC") else "grad"]
        assert_close(k, t.host()[inside], o[k][inside], m[k][inside], factor)
        assert np.isnan(t.host()[40:340]).all(), k
    for k, t in p.p.items():
        assert_close(k, t.double().cpu().numpy(), o[k], m[k], p.f["over_rows"])


@pytest.mark.parametrize("channels", [32, 4800])            # cut into chunks, and one chunk a sequence
@pytest.mark.parametrize("offsets", [[0, 1000, 500, 2000], [0, 5000, 100, 2000], [0, 2000, -7, 1500], [1990, 3, 1000, 900]])
def test_offsets_that_do_not_ascend_are_reported(offsets, channels):
    """Each call reports them, wherever they stand, and writes only into its tensors."""
    rows, n = 2000, 4
    dev = {k: Rows(np.full((rows, w), 0.5), "f32") for k, w in (("x", channels), ("dt", channels), ("B", n), ("C", n), ("dout", channels))}
    outs = {k: Rows(np.zeros((rows, w)), "f32", 4) for k, w in (("out", channels), ("dx", channels), ("ddt", channels), ("dB", n), ("dC", n))}
    off, A, dA = i32(offsets), f32(-np.ones((channels, n))), f32(np.zeros((channels, n)))
    a = tdx.tdx_scan_args(batch=3, max_len=rows, rows=rows, channels=channels, states=n, groups=1, dtype=tdx.TDX_F32, dt_softplus=1, A=A, dA=dA, seq_offsets=off,
                          **{k: t.ptr for k, t in {**dev, **outs}.items()}, **{"ld_" + k: t.ld for k, t in {**dev, **outs}.items()})
    saved = workspace(tdx.tdx_selective_scan_saved_size(a))
    a.set(saved=saved, saved_bytes=saved.numel())
    ws = workspace(tdx.tdx_selective_scan_workspace_size(a))
    a.set(workspace=ws, workspace_bytes=ws.numel())
    tdx.check(tdx.tdx_selective_scan(a))
    assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
    tdx.check(tdx.tdx_selective_scan_bwd(a))
    assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
    assert all(t.guards_intact() for t in {**dev, **outs}.values())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("where", ["x", "B", "C", "dt", "dout"])
@pytest.mark.parametrize("n,d,length", [(3, 10, 21), (16, 10, 21), (20, 16, 24), (16, 64, 37), (3, 10, 150), (16, 33, 150)])
def test_infinities_reach_what_depends_on_them_and_nothing_else(n, d, length, where, dtype):
    """One infinity among positive inputs, so that sums over states and channels have a definite sign.  States and channels that fill
    up a thread or a block, and rows behind the last of a tile, must add nothing."""
    p = Problem(dtype, n, d, [length], False, with_states=False)
    for k in ("x", "B", "C", "z", "D"):
        p.v[k] = np.abs(p.v[k]) + 2.0 ** -4
    p.v = {k: (torch.from_numpy(v).to(TORCH[dtype]).double().numpy() if k in ("x", "B", "C", "z") else v) for k, v in p.v.items()}
    p.dout = np.abs(p.dout)
    (p.dout if where == "dout" else p.v[where])[4, 1] = np.inf
    for k, t in p.dev.items():
        t.view[:] = torch.from_numpy(p.v[k]).cuda().to(TORCH[dtype])
    p.par["D"].copy_(torch.from_numpy(p.v["D"]))
    with np.errstate(all="ignore"):
        o, m = ref.scan(**p.v, dout=p.dout), ref.scan(**p.v, dout=p.dout, magnitude=True)
        p.forward(save=True)
        p.backward(with_state=False)
        got = {"out": p.out.host(), "state": p.new_state.host()[:1], **{k: t.host() for k, t in p.g.items()},
               **{k: t.double().cpu().numpy() for k, t in p.p.items()}}
        kind = {"out": "out", "state": "state", "dB": "over_channels", "dC": "over_channels", "dA": "over_rows", "dD": "over_rows", "ddt_bias": "over_rows"}
        for k, v in got.items():
            assert_close_but_infinities(k, v, o[k], m[k], p.f[kind.get(k, "grad")], dtype if k in ("out", "dx", "ddt", "dz", "dB", "dC") else "f32")
    assert tdx.tdx_check_device_status() == 0


@pytest.mark.parametrize("where", ["x", "B", "C", "dt"])
@pytest.mark.parametrize("n,d", [(3, 10), (16, 40), (20, 33), (100, 5)])
def test_infinities_in_single_tokens(n, d, where):
    batch = 3
    p = Problem("f32", n, d, [1] * batch, False)
    for k in ("x", "B", "C", "z", "D", "state"):
        p.v[k] = np.abs(p.v[k])
    p.v[where][1, 1] = np.inf
    for k, t in p.dev.items():
        t.view[:] = torch.from_numpy(p.v[k]).cuda().float()
    p.par["D"].copy_(torch.from_numpy(p.v["D"]))
    state, out = Rows(p.v["state"], "f32"), Rows(np.zeros((batch, d)), "f32", fill=float("nan"))
    p.args.set(out=out.ptr, ld_out=out.ld, state_in=state.ptr, state_out=state.ptr, n_slots=batch)
    with np.errstate(all="ignore"):
        o, m = ref.scan(**p.v), ref.scan(**p.v, magnitude=True)
        tdx.check(tdx.tdx_selective_scan_step(p.args))
        assert_close_but_infinities("out", out.host(), o["out"], m["out"], p.f["out"])
        assert_close_but_infinities("state", state.host(), o["state"], m["state"], p.f["state"])


LONGER = [
    # states, channels, lengths: every block goes through three tiles of rows or more
    (16, 1600, [100] * 3),           # one chunk a sequence: tiles of 32 rows
    (32, 800, [100] * 3),
    (8, 3200, [60] * 3),             # 16 rows
    (64, 400, [60] * 3),
    (4, 6400, [40] * 3),             # 8 rows
    (128, 200, [40] * 3),
    (12, 1600, [100] * 3),           # states that do not fill up the last thread
    (16, 3200, [500]),               # chunks of 128 rows
    (32, 1600, [500]),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", LONGER)
def test_many_tiles_a_block(shape, dtype):
    n, d, lengths = shape
    p = Problem(dtype, n, d, lengths, False)
    p.forward(save=True)
    p.check_forward()
    p.backward()
    # Among so many values some lie next to the root of silu'(z) = s (1 + z (1 - s)), whose rounding goes by the size of the terms
    # of the sum, not by the sum: dz is compared with that size, and taken out of the common check.
    extra = {"dout": p.dout, "dstate": p.dstate}
    o, m = ref.scan(**p.v, **extra), ref.scan(**p.v, **extra, magnitude=True)
    z, s = p.v["z"], ref.sigmoid(p.v["z"])
    y = m["out"] / np.abs(z * s)
    assert_close("dz", p.g["dz"].host(), o["dz"], np.abs(p.dout) * y * s * (1 + np.abs(z) * (1 - s)), p.f["grad"], dtype)
    assert p.g.pop("dz").guards_intact()
    p.check_backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,batch", [(16, 4096, 100), (12, 4095, 100), (64, 4096, 40), (4, 9000, 50)])
def test_single_tokens_of_many_rows(n, d, batch, dtype):
    """More rows than the grid has: a warp goes through several of them, some without a slot."""
    slots = [(5 * b) % (batch + 1) for b in range(batch)]
    slots[batch // 2::9] = [-1] * len(slots[batch // 2::9])
    p = Problem(dtype, n, d, [1] * batch, False, order=slots)
    state, out = Rows(p.all_states, "f32"), Rows(np.zeros((batch, d)), dtype, 1, fill=float("nan"))
    p.args.set(out=out.ptr, ld_out=out.ld, state_in=state.ptr, state_out=state.ptr)
    tdx.check(tdx.tdx_selective_scan_step(p.args))
    assert tdx.tdx_check_device_status() == 0
    o, m = ref.scan(**p.v), ref.scan(**p.v, magnitude=True)
    there = (np.array(slots) >= 0)[:, None]
    assert_close("out", out.host(), o["out"] * there, m["out"] * there, p.f["out"], dtype)
    got = state.host()
    for b, s in enumerate(slots):
        if s >= 0:
            assert_close("state", got[s], o["state"][b], m["state"][b], p.f["state"])
    for s in set(range(p.n_slots)) - set(slots):
        assert np.array_equal(got[s], p.all_states[s])
    assert out.guards_intact() and state.guards_intact()


@pytest.mark.parametrize("lengths", [[20, 0, 33, 1], [150, 0, 90, 3]])
def test_a_generous_max_len_changes_nothing(lengths):
    p = Problem("f32", 16, 40, lengths, True, order=[2, 0, 3, 1])
    p.args.set(max_len=32768)
    p.forward(save=True)
    p.check_forward()
    p.backward()
    p.check_backward()


def kept_states(L, e, d, n, step_by_step):
    """States of ones behind L rows whose inputs are zero and whose steps are e, all with A = -1."""
    A, state = f32(-np.ones((d, n))), torch.ones(1, d, n, device="cuda")
    zero, bc, dt, out = (torch.zeros(L, w, device="cuda") for w in (d, n, d, d))
    dt[:] = torch.from_numpy(e).cuda().float()
    a = tdx.tdx_scan_args(batch=1, max_len=L, rows=L, channels=d, states=n, groups=1, dtype=tdx.TDX_F32, dt_softplus=0, x=zero, ld_x=d, dt=dt, ld_dt=d, A=A, B=bc,
                          ld_B=n, C=bc, ld_C=n, out=out, ld_out=d, state_in=state, state_out=state, n_slots=1)
    ws = workspace(tdx.tdx_selective_scan_workspace_size(a))
    a.set(workspace=ws, workspace_bytes=ws.numel())
    for _ in range(L if step_by_step else 1):
        tdx.check((tdx.tdx_selective_scan_step if step_by_step else tdx.tdx_selective_scan)(a))
    torch.cuda.synchronize()
    return state[0].double().cpu().numpy()


@pytest.mark.parametrize("step_by_step", [False, True])
@pytest.mark.parametrize("lo,hi", [(0.002, 0.006), (0.006, 0.02), (0.02, 0.1)])
def test_decays_are_right_on_average(lo, hi, step_by_step):
    """A state takes in the error of one decay per row.  Over 8192 different decays the mean error of a row has to be well below what
    the rounding of a single one may be (2^-25): below half of it."""
    L, d, n = 64, 8192, 4
    e = np.random.default_rng(0).uniform(lo, hi, d).astype(np.float32).astype(np.float64)
    got = kept_states(L, e, d, n, step_by_step)
    want = np.exp(-L * e)[:, None]
    assert abs(((got - want) / want).mean()) / L < 2.0 ** -26


@pytest.mark.parametrize("step_by_step", [False, True])
@pytest.mark.parametrize("d,n", [(64, 16), (40, 3), (9, 100)])
def test_a_step_of_zero_keeps_the_state(d, n, step_by_step):
    assert (kept_states(45, np.zeros(d), d, n, step_by_step) == 1).all()
