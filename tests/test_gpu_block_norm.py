"""GPU parity of the block norm with its 64-bit definition."""
import numpy as np
import pytest
import torch

import layer_reference as ref
import paper_2409_03864_b200 as tdx
from seq_util import DT, EPS, Rows, assert_close, f32, seeded, workspace

pytestmark = pytest.mark.gpu
EPSILON = float(np.float32(1e-5))


class Case:
    def __init__(self, dtype, rows, d, group=0, norm_in=1, gate=True, residual=True, scale=True, weights=True, pad=0, lead=0, seed=0, magnitude=1.0):
        rng = np.random.default_rng(seed)
        self.dtype, self.rows, self.d, self.norm_in, self.rng = dtype, rows, d, norm_in, rng
        self.group = group or d
        self.pad, self.lead = pad, lead
        self.given = {"x": seeded(rng, (rows, d), dtype, magnitude)}
        if gate:
            self.given["gate"] = seeded(rng, (rows, d), dtype, 2.0)
        if residual:
            self.given["residual"] = seeded(rng, (rows, d), dtype)
        if scale:
            self.given["scale"] = seeded(rng, d, "f32")
        if weights and norm_in:
            self.given["weight_in"] = seeded(rng, d, "f32")
        if weights:
            self.given["weight_out"] = seeded(rng, d, "f32")
        self.dev = {k: (self.rows_of(v) if v.ndim == 2 else f32(v)) for k, v in self.given.items()}
        # serial additions of a sum: 16 channels a thread, 5 shuffles, 16 warps; wide rows channels / 512; odd groups one thread a
        # group.  Each rounds by EPS, a square root halves them; the functions and products are the other 64.
        self.ulps = 64 + self.group / 2 + d / 512
        # bf16 rows take the exponential by ex2.approx of v log2(e): |v| <= 12 here, so 12 x 1.45 x EPS and 4 EPS of ex2 and rcp
        self.factor = self.ulps * EPS + (24 * EPS if gate else 0.0)

    def rows_of(self, v, fill=None):
        return Rows(v, self.dtype, self.pad, self.lead, fill)

    def args(self, **more):
        a = tdx.tdx_norm_args(rows=self.rows, channels=self.d, group=self.group if self.norm_in else 0, dtype=DT[self.dtype], norm_in=self.norm_in, eps=EPSILON)
        for k, v in {**self.dev, **more}.items():
            a.set(**({k: v.ptr, "ld_" + k: v.ld} if isinstance(v, Rows) else {k: v}))
        return a

    def forward(self, want=("sum", "y")):
        outs = {k: self.rows_of(np.zeros((self.rows, self.d)), fill=float("nan")) for k in want}
        tdx.check(tdx.tdx_block_norm(self.args(**outs)))
        torch.cuda.synchronize()
        exact = ref.block_norm_all(self.given, self.group, self.norm_in, EPSILON)
        sizes = ref.block_norm_sizes(self.given, self.group, self.norm_in, EPSILON)
        for k, v in outs.items():
            assert_close(k, v.host(), exact[k], sizes[k], self.factor, self.dtype)
            assert v.guards_intact()
        return outs

    def backward(self, with_sum=True, with_y=True, sums=True):
        dsum = seeded(self.rng, (self.rows, self.d), self.dtype) if with_sum else None
        dy = seeded(self.rng, (self.rows, self.d), self.dtype) if with_y else None
        more = {k: self.rows_of(v) for k, v in (("dsum", dsum), ("dy", dy)) if v is not None}
        outs = {"d" + k: self.rows_of(np.zeros((self.rows, self.d)), fill=float("nan")) for k in ("x", "gate", "residual") if k in self.given}
        if sums:
            outs.update({"d" + k: torch.full((self.d,), float("nan"), device="cuda") for k in ("weight_in", "scale", "weight_out") if k in self.given})
        a = self.args(**more, **outs)
        ws = workspace(tdx.tdx_block_norm_workspace_size(a))
        a.set(workspace=ws, workspace_bytes=ws.numel())
        tdx.check(tdx.tdx_block_norm_bwd(a))
        torch.cuda.synchronize()
        first = {k: (v.host() if isinstance(v, Rows) else v.double().cpu().numpy()) for k, v in outs.items()}
        exact = ref.block_norm_all(self.given, self.group, self.norm_in, EPSILON, dsum, dy)
        sizes = ref.block_norm_sizes(self.given, self.group, self.norm_in, EPSILON, dsum, dy)
        for k, v in first.items():
            if isinstance(outs[k], Rows):
                assert_close(k, v, exact[k], sizes[k], 3 * self.factor, self.dtype)
                assert outs[k].guards_intact()
            else:
                want = exact[k] if k in exact else np.zeros(self.d)
                assert_close(k, v, want, sizes.get(k, np.zeros(self.d)), 3 * self.factor + self.rows * EPS)
        tdx.check(tdx.tdx_block_norm_bwd(a))                     # the same bits again
        torch.cuda.synchronize()
        for k, v in outs.items():
            assert np.array_equal(first[k], v.host() if isinstance(v, Rows) else v.double().cpu().numpy())


SHAPES = [
    # rows, channels, group
    (1, 1, 0), (1, 8, 0), (5, 7, 0), (3, 64, 16), (4, 4096, 0), (4, 4096, 128), (33, 512, 64), (2, 2000, 40), (3, 2909, 0), (7, 1366, 2), (2, 8192, 0),
    (2, 8192, 4096), (3, 8191, 0), (2, 4098, 0), (2, 8200, 0), (3, 9000, 90), (1, 20000, 0), (300, 96, 32), (1000, 24, 8), (17, 768, 768), (5, 1000, 1),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward(shape, dtype):
    c = Case(dtype, *shape)
    c.forward()
    c.backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm_in", [0, 1])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("residual", [False, True])
def test_every_part_alone_and_together(dtype, norm_in, gate, residual):
    for scale, weights in ((True, True), (False, False)):
        c = Case(dtype, 6, 256, 64 if norm_in else 0, norm_in, gate, residual, scale, weights)
        c.forward()
        c.forward(("sum",))
        c.forward(("y",))
        c.backward()
        c.backward(with_y=False)
        c.backward(with_sum=False)
        c.backward(sums=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,lead", [(8, 0), (0, 8), (1, 0), (0, 1), (2, 2), (3, 4)])
def test_slices_of_wider_rows(dtype, pad, lead):
    c = Case(dtype, 9, 320, 64, pad=pad, lead=lead)
    c.forward()
    c.backward()


def test_parameters_that_are_not_16_byte_aligned():
    c = Case("bf16", 5, 128)
    for k in ("weight_in", "scale", "weight_out"):
        t = torch.zeros(129, device="cuda")
        t[1:] = c.dev[k]
        c.dev[k] = t[1:]
    c.forward()
    c.backward()


@pytest.mark.parametrize("d", [512, 9000])
def test_sum_in_place_of_the_residual_and_dresidual_of_dsum(d):
    c = Case("bf16", 4, d)
    outs = c.forward()
    y = c.rows_of(np.zeros((4, d)))
    tdx.check(tdx.tdx_block_norm(c.args(sum=c.dev["residual"], y=y)))
    torch.cuda.synchronize()
    assert np.array_equal(c.dev["residual"].host(), outs["sum"].host()) and np.array_equal(y.host(), outs["y"].host())


def test_a_row_of_zeros_and_rows_that_are_not_finite():
    c = Case("f32", 4, 64, gate=False)
    x = c.dev["x"].view
    x[0] = 0.0
    x[2, 5] = float("inf")
    x[3, 1] = float("nan")
    s, y = c.rows_of(np.zeros((4, 64))), c.rows_of(np.zeros((4, 64)))
    tdx.check(tdx.tdx_block_norm(c.args(sum=s, y=y)))
    torch.cuda.synchronize()
    assert np.array_equal(s.host()[0], c.given["residual"][0])    # a zero row is a zero row, not a NaN
    assert np.isfinite(s.host()[1]).all() and np.isfinite(y.host()[:2]).all()
    assert np.isnan(s.host()[2, 5]) and np.isnan(s.host()[3]).all()


def test_no_rows_give_zero_parameter_gradients_and_no_channels_nothing():
    g = [torch.full((32,), 7.0, device="cuda") for _ in range(3)]
    a = tdx.tdx_norm_args(rows=0, channels=32, dtype=tdx.TDX_BF16, norm_in=1, eps=1e-5, dweight_in=g[0], dscale=g[1], dweight_out=g[2])
    tdx.check(tdx.tdx_block_norm(a))
    tdx.check(tdx.tdx_block_norm_bwd(a))
    torch.cuda.synchronize()
    assert all((v == 0).all() for v in g)
    tdx.check(tdx.tdx_block_norm_bwd(tdx.tdx_norm_args(rows=3, channels=0, dtype=tdx.TDX_F32, eps=0.0)))


def test_captured_and_replayed_on_another_stream():
    c = Case("bf16", 37, 512, 64)
    outs = c.forward()
    c.backward()
    s, y, dx = (c.rows_of(np.zeros((37, 512))) for _ in range(3))
    dy = c.rows_of(seeded(c.rng, (37, 512), "bf16"))
    dgate, dres, dw = c.rows_of(np.zeros((37, 512))), c.rows_of(np.zeros((37, 512))), torch.zeros(512, device="cuda")
    a = c.args(sum=s, y=y, dy=dy, dx=dx, dgate=dgate, dresidual=dres, dweight_in=dw)
    ws = workspace(tdx.tdx_block_norm_workspace_size(a))
    a.set(workspace=ws, workspace_bytes=ws.numel())
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        tdx.check(tdx.tdx_block_norm(a, torch.cuda.current_stream()))
        tdx.check(tdx.tdx_block_norm_bwd(a, torch.cuda.current_stream()))
    for _ in range(2):
        s.full.fill_(-77.0)
        graph.replay()
    torch.cuda.synchronize()
    assert np.array_equal(s.host(), outs["sum"].host()) and np.array_equal(y.host(), outs["y"].host())
    again = dw.clone()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(again, dw) and bool(torch.isfinite(dw).all())


def test_workspace_refusals():
    c = Case("bf16", 5, 128)
    out = {"d" + k: c.rows_of(np.zeros((5, 128)), fill=-5.0) for k in ("x", "gate", "residual")}
    a = c.args(dy=c.rows_of(np.zeros((5, 128))), **out)
    ws = workspace(tdx.tdx_block_norm_workspace_size(a))
    for change, status in ((dict(workspace=None, workspace_bytes=1 << 30), tdx.TDX_ERR_WORKSPACE), (dict(workspace=ws, workspace_bytes=ws.numel() - 1), tdx.TDX_ERR_WORKSPACE),
                           (dict(workspace=ws.data_ptr() + 16, workspace_bytes=1 << 30), tdx.TDX_ERR_ALIGNMENT)):
        assert tdx.tdx_block_norm_bwd(a.set(**change)) == status
    torch.cuda.synchronize()
    assert all((v.host() == -5.0).all() for v in out.values())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,group", [(512, 0), (2000, 40), (4096, 128), (9000, 0)])
def test_dresidual_in_place_of_dsum(d, group, dtype):
    c = Case(dtype, 700, d, group)                               # (several rows for every set of threads)
    dsum, dy = (seeded(c.rng, (700, d), dtype) for _ in range(2))
    dev_dy, results = c.rows_of(dy), []
    for shared in (False, True):
        own = c.rows_of(dsum)
        outs = {"d" + k: c.rows_of(np.zeros((700, d)), fill=float("nan")) for k in ("x", "gate", "residual")}
        if shared:
            outs["dresidual"] = own
        outs.update({"d" + k: torch.full((d,), float("nan"), device="cuda") for k in ("weight_in", "scale", "weight_out")})
        a = c.args(dsum=own, dy=dev_dy, **outs)
        ws = workspace(tdx.tdx_block_norm_workspace_size(a))
        tdx.check(tdx.tdx_block_norm_bwd(a.set(workspace=ws, workspace_bytes=ws.numel())))
        torch.cuda.synchronize()
        results.append({k: v.full.clone() if isinstance(v, Rows) else v for k, v in outs.items()})
    for k, v in results[0].items():
        assert bool(torch.isfinite(v).all()) and torch.equal(v, results[1][k]), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(700, 4096, 0), (700, 8192, 0), (700, 4096, 128), (700, 2000, 40), (700, 2909, 0), (700, 9000, 0), (650, 9000, 90), (10000, 64, 16)])
def test_many_rows_for_every_set_of_threads(shape, dtype):
    c = Case(dtype, *shape)
    c.forward()
    c.backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm_in,gate,residual", [(0, False, False), (0, False, True), (1, True, False), (1, False, True)])
def test_many_rows_of_the_usual_parts(norm_in, gate, residual, dtype):
    c = Case(dtype, 700, 4096, 0, norm_in, gate, residual, scale=residual)
    c.forward(("sum",) if norm_in and not residual else ("y",) if not residual else ("sum", "y"))
    c.backward(with_sum=bool(norm_in or residual), with_y=not norm_in or residual)
