"""GPU parity of the linear attention with decay with its 64-bit definition, one row after the other."""
import numpy as np
import pytest
import torch

import layer_reference as ref
import paper_2409_03864_b200 as tdx
from seq_util import DT, EPS, TORCH, Rows, assert_close, f32, i32, offsets_of, seeded, workspace

pytestmark = pytest.mark.gpu
CANARY = -77.0


class Case:
    def __init__(self, dtype, lengths, heads, dk, dv, shares=(1, 1, 1), states=True, pad=0, lead=0, packed=None, spare=0, seed=0, decay=None, step=False):
        rng = self.rng = np.random.default_rng(seed)
        self.dtype, self.lengths, self.heads, self.dk, self.dv = dtype, lengths, heads, dk, dv
        self.own = [heads // s for s in shares]
        self.rows = sum(lengths) + spare
        self.pad, self.lead, self.spare, self.step = pad, lead, spare, step
        self.packed = len(set(lengths)) > 1 or spare > 0 if packed is None else packed
        self.q, self.k, self.v = (seeded(rng, (self.rows, h, d), dtype) for h, d in zip(self.own, (dk, dk, dv)))
        self.dout = seeded(rng, (self.rows, heads, dv), dtype)
        self.scale = float(np.float32(dk ** -0.5))
        d = np.log1p(-np.exp2(-np.linspace(0.7, 9.0, heads))) if decay is None else np.full(heads, decay)
        self.log_decay = d.astype(np.float32).astype(np.float64)
        count = len(lengths)
        self.n_slots = count + 2
        self.slots = rng.permutation(self.n_slots)[:count]
        self.states = states
        self.state = seeded(rng, (count, heads, dk, dv), "f32") if states else np.zeros((count, heads, dk, dv))
        self.dstate = seeded(rng, (count, heads, dk, dv), "f32") if states else None
        self.dev = {n: self.rows_of(getattr(self, n)) for n in ("q", "k", "v", "dout")}
        self.cache, self.dcache = (self.slots_of(v) if states else None for v in (self.state, self.dstate))

    def rows_of(self, v, fill=None):
        return Rows(v, self.dtype, self.pad, self.lead, fill)

    def slots_of(self, v=None):
        t = torch.full((self.n_slots, self.heads, self.dk, self.dv), CANARY, device="cuda")
        if v is not None:
            t[torch.from_numpy(self.slots).cuda()] = f32(v)
        return t

    def args(self, **more):
        a = tdx.tdx_attention_args(
            batch=len(self.lengths), max_len=max(self.lengths), rows=self.rows, heads=self.heads, q_heads=self.own[0], k_heads=self.own[1], v_heads=self.own[2],
            dim_k=self.dk, dim_v=self.dv, dtype=DT[self.dtype], scale=self.scale)
        self.keep = [f32(self.log_decay), i32(offsets_of(self.lengths)) if self.packed else None, i32(self.slots)]
        a.set(log_decay=self.keep[0], seq_offsets=self.keep[1], slots=self.keep[2], n_slots=self.n_slots)
        for name, v in {**self.dev, **more}.items():
            a.set(**({name: v.ptr, "ld_" + name: v.ld} if isinstance(v, Rows) else {name: v}))
        if not self.step:
            ws = workspace(tdx.tdx_decay_attention_workspace_size(a))
            self.keep.append(ws)
            a.set(workspace=ws, workspace_bytes=ws.numel())
        return a

    def exact(self, size=False, grads=True):
        f = np.abs if size else np.asarray
        n = sum(self.lengths)
        return ref.decay_attention_all(f(self.q[:n]), f(self.k[:n]), f(self.v[:n]), self.log_decay, self.scale, self.lengths, f(self.state), f(self.dout[:n]) if grads else None,
                                       None if self.dstate is None else f(self.dstate))

    def factors(self):
        # fp32 sums over the rows of a sequence (each chunk, and each decay of the state), over a head and over shared heads, twice for
        # truncating accumulation; pieces of three bf16 lose about 3 EPS a product.  bf16: weights and the states that rows read are
        # rounded once each (half a step, 2^-8, of disjoint terms), and a state that is only read keeps 16 bits of its terms
        exact = (2 * (max(self.lengths) + self.dk + self.dv + self.heads) + 64) * EPS
        return exact, exact + (0.0 if self.dtype == "f32" else 2.0 ** -8 + 2.0 ** -15)

    def check(self, back=True):
        n = sum(self.lengths)
        want, size = self.exact(grads=back), self.exact(True, back)
        exact, rounded = self.factors()
        out, new = self.rows_of(np.zeros((self.rows, self.heads, self.dv)), fill=-5.0), self.slots_of()
        for store in ((new, None) if self.states else (None,)):
            a = self.args(out=out, state_in=self.cache, state_out=store)
            tdx.check(tdx.tdx_decay_attention(a))
            torch.cuda.synchronize()
            got = out.host()
            assert_close("out", got[:n], want["out"], size["out"], rounded, self.dtype)
            assert (got[n:] == -5.0).all() and out.guards_intact()
        if self.states:
            host = new.double().cpu().numpy()
            assert_close("state", host[self.slots], want["state"], size["state"], exact)
            others = np.setdiff1d(np.arange(self.n_slots), self.slots)
            assert (host[others] == CANARY).all()
        if back:
            g = {"d" + name: self.rows_of(np.zeros(v.shape), fill=-5.0) for name, v in (("q", self.q), ("k", self.k), ("v", self.v))}
            ds = self.slots_of()
            a = self.args(**g, state_in=self.cache, dstate_out=self.dcache, dstate_in=ds if self.states else None)
            tdx.check(tdx.tdx_decay_attention_bwd(a))
            torch.cuda.synchronize()
            first = {k: v.full.clone() for k, v in g.items()}
            for k, v in g.items():
                got = v.host()
                assert_close(k, got[:n], want[k], size[k], rounded, self.dtype)
                assert (got[n:] == -5.0).all() and v.guards_intact()
            if self.states:
                assert_close("dstate", ds.double().cpu().numpy()[self.slots], want["dstate"], size["dstate"], exact)
            tdx.check(tdx.tdx_decay_attention_bwd(a))            # the same bits again
            torch.cuda.synchronize()
            assert all(torch.equal(first[k], g[k].full) for k in g)
        tdx.check(tdx.tdx_check_device_status())
        return out


SHAPES = [
    # lengths, heads, dim_k, dim_v
    ([1], 1, 16, 16), ([64], 2, 64, 64), ([65, 65], 1, 32, 48), ([63, 1, 0, 130], 3, 64, 80), ([300], 2, 128, 128), ([5, 0, 70, 256], 4, 128, 64),
    ([129, 128], 2, 96, 128), ([40, 200], 5, 72, 24), ([1100], 1, 64, 64), ([700, 3, 513], 2, 128, 96), ([2, 3, 1], 16, 8, 8),
]


@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_prompts_and_gradients(shape, dtype, states):
    Case(dtype, *shape, states=states).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dims", [(1, 1), (7, 13), (65, 3), (127, 66), (10, 12), (128, 1)])
def test_odd_dims(dims, dtype):
    Case(dtype, [70, 0, 33], 2, *dims).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shares", [(1, 2, 2), (4, 1, 1), (1, 4, 1), (2, 4, 1), (4, 4, 4)])
def test_shared_heads(shares, dtype):
    Case(dtype, [90, 7], 4, 32, 64, shares).check()
    Case(dtype, [50], 4, 30, 20, shares, spare=3).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,lead,spare", [(8, 0, 0), (0, 8, 5), (1, 0, 0), (0, 1, 1), (4, 4, 0)])
def test_slices_of_wider_rows_and_rows_behind_the_last_sequence(dtype, pad, lead, spare):
    Case(dtype, [66, 30], 2, 64, 64, pad=pad, lead=lead, spare=spare).check()


@pytest.mark.parametrize("decay", [0.0, -1e-6, -0.5, -40.0, -1e30, 0.01])
def test_decays_from_keeping_everything_to_forgetting_at_once(decay):
    for dtype in ("f32", "bf16"):
        Case(dtype, [130, 65], 1, 16, 16, decay=decay).check()


def test_minus_infinity_is_a_decay_too():
    c = Case("f32", [70], 1, 16, 16, decay=float("-inf"))
    out = c.rows_of(np.zeros((70, 1, 16)))
    tdx.check(tdx.tdx_decay_attention(c.args(out=out, state_in=c.cache, state_out=c.slots_of())))
    torch.cuda.synchronize()
    want = c.scale * (c.q * c.k).sum(2, keepdims=True) * c.v
    assert_close("out", out.host(), want, c.scale * (np.abs(c.q * c.k)).sum(2, keepdims=True) * np.abs(c.v), c.factors()[0])


def test_state_in_place_and_without_slots():
    c = Case("bf16", [100, 0, 30], 2, 64, 64)
    out, new = c.rows_of(np.zeros((130, 2, 64))), c.slots_of()
    tdx.check(tdx.tdx_decay_attention(c.args(out=out, state_in=c.cache, state_out=new)))
    c.slots[1] = -1                                              # the empty sequence has no state now
    keep = c.cache.clone()
    tdx.check(tdx.tdx_decay_attention(c.args(out=out, state_in=c.cache, state_out=c.cache)))
    torch.cuda.synchronize()
    live = [int(c.slots[0]), int(c.slots[2])]
    assert torch.equal(c.cache[live], new[live])
    others = [i for i in range(c.n_slots) if i not in live]
    assert torch.equal(c.cache[others], keep[others])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,dk,dv,shares", [(1, 64, 64, (1, 1, 1)), (4, 128, 128, (1, 2, 2)), (3, 16, 20, (1, 3, 1)), (2, 33, 5, (1, 1, 1)), (2, 128, 1, (1, 1, 1)), (1, 1, 128, (1, 1, 1))])
def test_single_tokens(heads, dk, dv, shares, dtype):
    c = Case(dtype, [1] * 9, heads, dk, dv, shares, step=True)
    want, size = c.exact(grads=False), c.exact(True, False)
    c.slots[4] = -1
    live = c.slots >= 0
    out = c.rows_of(np.zeros((9, heads, dv)), fill=-5.0)
    factor = (2 * dk + 16) * EPS
    for new in (c.slots_of(), c.cache):                          # into another cache, then in place
        tdx.check(tdx.tdx_decay_attention_step(c.args(out=out, state_in=c.cache, state_out=new)))
        torch.cuda.synchronize()
        got, host = out.host(), new.double().cpu().numpy()
        assert_close("out", got[live], want["out"][live], size["out"][live], factor, dtype)
        assert (got[~live] == 0).all() and out.guards_intact()
        assert_close("state", host[c.slots[live]], want["state"][live], size["state"][live], 8 * EPS)


def test_tokens_after_a_prompt_are_a_longer_prompt():
    c = Case("f32", [50, 20], 2, 64, 32)
    out, new = c.rows_of(np.zeros((70, 2, 32))), c.slots_of()
    tdx.check(tdx.tdx_decay_attention(c.args(out=out, state_in=c.cache, state_out=new)))
    # the first 40 and 10 rows as prompts, the others as tokens
    whole = {n: c.dev[n] for n in ("q", "k", "v")}
    order = list(range(40)) + list(range(50, 60))
    parts = {n: c.rows_of(v.host()[order]) for n, v in whole.items()}
    d = Case("f32", [40, 10], 2, 64, 32)
    d.slots, d.cache = c.slots, c.cache
    d.dev.update(parts)
    cache, got = c.slots_of(), c.rows_of(np.zeros((50, 2, 32)))
    tdx.check(tdx.tdx_decay_attention(d.args(out=got, state_in=c.cache, state_out=cache)))
    s = Case("f32", [1, 1], 2, 64, 32, step=True)
    s.slots = c.slots
    tokens = []
    for t in range(10):
        s.dev.update({n: c.rows_of(v.host()[[40 + t, 60 + t]]) for n, v in whole.items()})
        one = c.rows_of(np.zeros((2, 2, 32)))
        tdx.check(tdx.tdx_decay_attention_step(s.args(out=one, state_in=cache, state_out=cache)))
        torch.cuda.synchronize()
        tokens.append(one.host())
    size = c.exact(True, False)
    want = out.host()
    factor = 2 * c.factors()[0]
    assert_close("tokens", np.stack(tokens), np.stack([want[40:50], want[60:70]], axis=1), np.stack([size["out"][40:50], size["out"][60:70]], axis=1), factor)
    assert_close("state", cache.double().cpu().numpy()[c.slots], new.double().cpu().numpy()[c.slots], size["state"], factor)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bad_offsets_and_slots_are_reported(dtype):
    for offsets, slots in (([0, 60, 40, 100], None), ([0, 60, 101, 120], None), ([0, 60, 60, 100], [0, 1, 99])):
        c = Case(dtype, [60, 10, 30], 1, 16, 16)
        out, new = c.rows_of(np.zeros((100, 1, 16)), fill=-5.0), c.slots_of()
        a = c.args(out=out, state_in=c.cache, state_out=new)
        bad = i32(offsets)
        a.set(seq_offsets=bad)
        if slots:
            wrong = i32(slots)
            a.set(slots=wrong)
        tdx.check(tdx.tdx_decay_attention(a))
        assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
        assert out.guards_intact()
    s = Case(dtype, [1, 1], 1, 16, 16, step=True)
    one, wrong = s.rows_of(np.zeros((2, 1, 16)), fill=-5.0), i32([1, 400])
    a = s.args(out=one, state_in=s.cache, state_out=s.cache)
    a.set(slots=wrong)
    tdx.check(tdx.tdx_decay_attention_step(a))
    assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
    assert (one.host()[1] == 0).all()


def test_no_rows_move_states_on_unchanged():
    c = Case("f32", [0, 0], 2, 16, 16)
    new, ds = c.slots_of(), c.slots_of()
    tdx.check(tdx.tdx_decay_attention(c.args(state_in=c.cache, state_out=new)))
    tdx.check(tdx.tdx_decay_attention_bwd(c.args(state_in=c.cache, dstate_out=c.dcache, dstate_in=ds)))
    torch.cuda.synchronize()
    at = torch.from_numpy(c.slots).cuda()
    assert torch.equal(new[at], c.cache[at]) and torch.equal(ds[at], c.dcache[at])


def test_values_that_are_not_finite_stay_in_their_sequence_and_head():
    c = Case("bf16", [70, 70], 2, 64, 64)
    c.dev["v"].view[30, 64:] = float("nan")                      # head 1 of the first sequence
    out = c.rows_of(np.zeros((140, 2, 64)))
    tdx.check(tdx.tdx_decay_attention(c.args(out=out, state_in=c.cache, state_out=c.slots_of())))
    torch.cuda.synchronize()
    got = out.host()
    assert np.isfinite(got[:, 0]).all() and np.isfinite(got[70:]).all() and np.isnan(got[30:70, 1]).all()


def test_captured_and_replayed():
    c = Case("bf16", [300, 80], 2, 64, 64)
    out, new = c.rows_of(np.zeros((380, 2, 64))), c.slots_of()
    g = {"dq": c.rows_of(np.zeros(c.q.shape)), "dk": c.rows_of(np.zeros(c.k.shape)), "dv": c.rows_of(np.zeros(c.v.shape))}
    a = c.args(out=out, state_in=c.cache, state_out=new, **g)
    tdx.check(tdx.tdx_decay_attention(a))
    tdx.check(tdx.tdx_decay_attention_bwd(a))
    torch.cuda.synchronize()
    first = [v.full.clone() for v in (out, *g.values())]
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        tdx.check(tdx.tdx_decay_attention(a, torch.cuda.current_stream()))
        tdx.check(tdx.tdx_decay_attention_bwd(a, torch.cuda.current_stream()))
    for v in (out, *g.values()):
        v.view.fill_(3.0)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, v.full) for x, v in zip(first, (out, *g.values())))


def test_workspace_refusals():
    c = Case("bf16", [1100], 1, 64, 64)
    out = c.rows_of(np.zeros((1100, 1, 64)), fill=-5.0)
    a = c.args(out=out, state_in=c.cache, state_out=c.slots_of())
    ws = c.keep[-1]
    assert ws.numel() > 0
    for change, status in ((dict(workspace=None, workspace_bytes=1 << 30), tdx.TDX_ERR_WORKSPACE), (dict(workspace=ws, workspace_bytes=ws.numel() // 2 - 1), tdx.TDX_ERR_WORKSPACE),
                           (dict(workspace=ws.data_ptr() + 16, workspace_bytes=1 << 30), tdx.TDX_ERR_ALIGNMENT)):
        assert tdx.tdx_decay_attention(a.set(**change)) == status, change
    torch.cuda.synchronize()
    assert (out.host() == -5.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 1])
def test_state_in_place_of_sequences_in_several_segments(dtype, pad):
    c = Case(dtype, [1300, 40], 1, 64, 64, pad=pad)
    one, two, new = c.rows_of(np.zeros((1340, 1, 64))), c.rows_of(np.zeros((1340, 1, 64))), c.slots_of()
    tdx.check(tdx.tdx_decay_attention(c.args(out=one, state_in=c.cache, state_out=new)))
    tdx.check(tdx.tdx_decay_attention(c.args(out=two, state_in=c.cache, state_out=c.cache)))
    torch.cuda.synchronize()
    at = torch.from_numpy(c.slots).cuda()
    size, factors = c.exact(True, False), c.factors()
    assert_close("out", two.host(), one.host(), size["out"], 2 * factors[1], dtype)
    assert_close("state", c.cache[at].double().cpu().numpy(), new[at].double().cpu().numpy(), size["state"], 2 * factors[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decays_that_leave_fp32_only_behind_a_short_sequence(dtype):
    # e^19 is small enough for every sum; e^127, of rows of the tile that the sequence does not have, is not
    Case(dtype, [20, 7], 1, 16, 16, decay=1.0).check()


def run_all(c):
    """Every output of the call and its backward pass, with and without states handed on."""
    outs = {}
    for tag, store in (("", c.slots_of()), (" alone", None)):
        out = c.rows_of(np.zeros((c.rows, c.heads, c.dv)), fill=-5.0)
        tdx.check(tdx.tdx_decay_attention(c.args(out=out, state_in=c.cache, state_out=store)))
        outs["out" + tag] = out.view
        if store is not None:
            outs["state"] = store
        g = {"d" + name: c.rows_of(np.zeros(v.shape), fill=-5.0) for name, v in (("q", c.q), ("k", c.k), ("v", c.v))}
        grad = None if store is None else c.slots_of()
        tdx.check(tdx.tdx_decay_attention_bwd(c.args(**g, state_in=c.cache, dstate_out=c.dcache, dstate_in=grad)))
        outs.update({k + tag: v.view for k, v in g.items()})
        if grad is not None:
            outs["dstate"] = grad
    torch.cuda.synchronize()
    return {k: v.clone() for k, v in outs.items()}


# two heads: the longer sequences are cut into segments; 150: a block has all chunks of a sequence
@pytest.mark.parametrize("heads", [2, 150])
@pytest.mark.parametrize("length", [5, 133, 261, 773, 901])      # a short chunk of 5 rows behind 0, 1, 2, 6 and 7 whole ones
@pytest.mark.parametrize("dtype,pad", [("bf16", 0), ("bf16", 1), ("f32", 0)])
def test_rows_of_others_that_are_not_finite_do_not_show(dtype, pad, length, heads):
    c = Case(dtype, [70, length, 90], heads, 16, 24, pad=pad, spare=130)
    before = tdx.tdx_kernel_launch_count()
    clean = run_all(c)
    cut = heads == 2 and length > 700                            # (the passes over the states and the kernel that joins them)
    assert (tdx.tdx_kernel_launch_count() - before > 8) == cut
    mine = slice(70, 70 + length)
    for name in ("q", "k", "v", "dout"):
        v = c.dev[name].view
        for part in (v[:70], v[70 + length:]):
            part[::3], part[1::3], part[2::3] = float("nan"), float("inf"), float("-inf")
    got = run_all(c)
    for k in clean:
        at = int(c.slots[1]) if k in ("state", "dstate") else mine
        assert bool(torch.isfinite(got[k][at]).all()), k
        assert torch.equal(got[k][at], clean[k][at]), k
    tdx.check(tdx.tdx_check_device_status())


@pytest.mark.parametrize("dtype,pad", [("bf16", 0), ("bf16", 1), ("f32", 0)])
@pytest.mark.parametrize("lengths", [[1] * 9 + [1500] + [0, 1, 2] * 9, [1500, 300, 1, 0, 255, 256, 257, 1200], [0, 0, 700], [1200, 0, 0]], ids=["many", "some", "first", "last"])
def test_long_sequences_among_short_ones(lengths, dtype, pad):
    c = Case(dtype, lengths, 2, 24, 40, pad=pad, spare=70)
    before = tdx.tdx_kernel_launch_count()
    c.check()
    assert tdx.tdx_kernel_launch_count() - before > 10           # (some sequences are cut)
    # the states in place are the same bits
    out, new = c.rows_of(np.zeros((c.rows, 2, 40))), c.slots_of()
    again = c.cache.clone()
    tdx.check(tdx.tdx_decay_attention(c.args(out=out, state_in=c.cache, state_out=new)))
    tdx.check(tdx.tdx_decay_attention(c.args(out=out, state_in=again, state_out=again)))
    torch.cuda.synchronize()
    if dtype == "bf16" and pad == 0:
        at = torch.from_numpy(c.slots).cuda()
        assert torch.equal(again[at], new[at])


# heads fill the SMs: a block has all chunks of a sequence; few heads: segments, and pieces of them, of several chunks
@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("lengths,heads,dk,dv", [([1100], 150, 16, 16), ([700, 0, 1000], 160, 8, 24), ([4096], 32, 16, 16), ([4500], 30, 24, 8), ([2600, 1900], 40, 16, 16)])
def test_many_chunks_a_block(lengths, heads, dk, dv, states):
    Case("bf16", lengths, heads, dk, dv, states=states).check()


@pytest.mark.parametrize("lengths,heads", [([700], 150), ([640, 597], 90), ([3000], 8), ([2500, 40], 24)])
def test_many_chunks_of_wide_heads_against_fp32(lengths, heads):
    c = Case("bf16", lengths, heads, 128, 128)
    names = ("q", "k", "v", "dout", "state", "dstate")

    def same_values(f):
        d = Case("f32", lengths, heads, 128, 128)
        for n in names:
            setattr(d, n, f(getattr(c, n)))
        d.slots = c.slots
        d.dev = {n: d.rows_of(getattr(d, n)) for n in ("q", "k", "v", "dout")}
        d.cache, d.dcache = d.slots_of(d.state), d.slots_of(d.dstate)
        return run_all(d)

    got, want, size = run_all(c), same_values(np.asarray), same_values(np.abs)
    exact, rounded = c.factors()
    at = torch.from_numpy(c.slots).cuda()
    for k in got:
        g, w, s = (v[k][at] if k.endswith("state") else v[k] for v in (got, want, size))
        # both are off, the fp32 kernel by `exact`
        factor, dtype = (2 * exact, "f32") if k.endswith("state") else (exact + rounded, "bf16")
        assert_close(k, *(v.double().cpu().numpy() for v in (g, w, s)), factor, dtype)


@pytest.mark.parametrize("dtype,pad", [("bf16", 0), ("bf16", 1), ("f32", 0)])
@pytest.mark.parametrize("batch", [3, 12])                       # slots for every sequence; for those of several segments
def test_bad_offsets_of_cut_sequences_are_reported(batch, dtype, pad):
    for offsets in ([0, 900, 400, 1500], [0, 1300, 1501, 1600], [-900, 0, 800, 1500]):
        c = Case(dtype, [700, 300, 500] + [0] * (batch - 3), 2, 16, 16, pad=pad)
        out, new = c.rows_of(np.zeros((1500, 2, 16)), fill=-5.0), c.slots_of()
        g = {"d" + n: c.rows_of(np.zeros(v.shape), fill=-5.0) for n, v in (("q", c.q), ("k", c.k), ("v", c.v))}
        bad = i32(offsets + offsets[-1:] * (batch - 3))
        grad = c.slots_of()
        a = c.args(out=out, state_in=c.cache, state_out=new, **g, dstate_out=c.dcache, dstate_in=grad)
        a.set(seq_offsets=bad, max_len=1400)
        ws = workspace(tdx.tdx_decay_attention_workspace_size(a))
        a.set(workspace=ws, workspace_bytes=ws.numel())
        for call in (tdx.tdx_decay_attention, tdx.tdx_decay_attention_bwd):
            tdx.check(call(a))
            assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
        assert out.guards_intact() and all(v.guards_intact() for v in g.values())
        others = np.setdiff1d(np.arange(c.n_slots), c.slots)
        assert bool((new[torch.from_numpy(others).cuda()] == CANARY).all())


def test_captured_once_and_replayed_with_other_lengths():
    lengths = [900, 5, 300] + [1] * 12
    c = Case("bf16", lengths, 2, 32, 16)
    out, new = c.rows_of(np.zeros((c.rows, 2, 16))), c.slots_of()
    a = c.args(out=out, state_in=c.cache, state_out=new)
    offsets = c.keep[1]
    tdx.check(tdx.tdx_decay_attention(a))
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        tdx.check(tdx.tdx_decay_attention(a, torch.cuda.current_stream()))
    for lengths in ([1] * 12 + [300, 5, 900], [80] * 14 + [97], [0] * 7 + [900, 0, 317] + [0] * 5):
        c.lengths = lengths
        offsets.copy_(torch.from_numpy(offsets_of(lengths)))
        out.view.fill_(-5.0)
        graph.replay()
        torch.cuda.synchronize()
        want, size = c.exact(grads=False), c.exact(True, False)
        exact, rounded = c.factors()
        assert_close("out", out.host(), want["out"], size["out"], rounded, "bf16")
        assert_close("state", new.double().cpu().numpy()[c.slots], want["state"], size["state"], exact)
    tdx.check(tdx.tdx_check_device_status())
