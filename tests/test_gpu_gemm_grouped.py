"""GPU parity of the products grouped by expert with their 64-bit definition."""
import numpy as np
import pytest
import torch

import layer_reference as ref
import paper_2409_03864_b200 as tdx
from seq_util import DT, EPS, TORCH, Rows, assert_close, i32, seeded, workspace

pytestmark = pytest.mark.gpu


def close(name, got, want, size, terms, dtype):
    # fp32: every product and addition rounds once (the tensor cores' pieces of an operand lose less than 2 EPS a product);
    # bf16: products are exact, sums are fp32, the tensor cores may truncate an addend instead of rounding it (2 EPS)
    assert_close(name, got, want, size, (2 * terms + 8) * EPS, dtype)


class Case:
    def __init__(self, dtype, lengths, n, k, first=0, spare=0, pad=0, lead=0, seed=0, rng=None):
        self.rng = rng or np.random.default_rng(seed)
        self.dtype, self.n, self.k, self.lengths = dtype, n, k, lengths
        self.offsets = first + np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
        self.rows = int(self.offsets[-1]) + spare
        self.pad, self.lead = pad, lead
        self.x, self.dy = (seeded(self.rng, (self.rows, d), dtype) for d in (k, n))
        self.w = seeded(self.rng, (len(lengths), n, k), dtype)
        self.dev = {"x": self.rows_of(self.x), "dy": self.rows_of(self.dy)}
        self.dev_w = torch.from_numpy(self.w).cuda().to(TORCH[dtype])
        self.dev_offsets = i32(self.offsets)

    def rows_of(self, v, fill=None):
        return Rows(v, self.dtype, self.pad, self.lead, fill)

    def args(self, **more):
        a = tdx.tdx_grouped_args(rows=self.rows, experts=len(self.lengths), N=self.n, K=self.k, dtype=DT[self.dtype], offsets=self.dev_offsets, weight=self.dev_w)
        for name, v in {**self.dev, **more}.items():
            a.set(**({name: v.ptr, "ld_" + name: v.ld} if isinstance(v, Rows) else {name: v}))
        self.ws = workspace(tdx.tdx_gemm_grouped_workspace_size(a))
        return a.set(workspace=self.ws, workspace_bytes=self.ws.numel())

    def check(self, back=True):
        inside = np.zeros(self.rows, dtype=bool)
        inside[self.offsets[0]:self.offsets[-1]] = True
        y = self.rows_of(np.zeros((self.rows, self.n)), fill=-5.0)
        tdx.check(tdx.tdx_gemm_grouped(self.args(y=y)))
        torch.cuda.synchronize()
        got = y.host()
        close("y", got[inside], ref.grouped(self.x, self.w, self.offsets)[inside], ref.grouped(abs(self.x), abs(self.w), self.offsets)[inside], self.k, self.dtype)
        assert (got[~inside] == -5.0).all() and y.guards_intact()
        if not back:
            return y
        dx = self.rows_of(np.zeros((self.rows, self.k)), fill=-5.0)
        tdx.check(tdx.tdx_gemm_grouped_dx(self.args(dx=dx)))
        torch.cuda.synchronize()
        wt = self.w.transpose(0, 2, 1)
        got = dx.host()
        close("dx", got[inside], ref.grouped(self.dy, wt, self.offsets)[inside], ref.grouped(abs(self.dy), abs(wt), self.offsets)[inside], self.n, self.dtype)
        assert (got[~inside] == -5.0).all() and dx.guards_intact()
        dw = torch.full((len(self.lengths) * self.n * self.k + 64,), -5.0, device="cuda", dtype=TORCH[self.dtype])
        tdx.check(tdx.tdx_gemm_grouped_dw(self.args(dweight=dw)))
        torch.cuda.synchronize()
        got = dw.double().cpu().numpy()
        assert (got[-64:] == -5.0).all()
        size = ref.grouped_dw(abs(self.dy), abs(self.x), self.offsets)
        close("dweight", got[:-64].reshape(self.w.shape), ref.grouped_dw(self.dy, self.x, self.offsets), size, max(max(self.lengths), 1), self.dtype)
        tdx.check(tdx.tdx_check_device_status())
        return y


SHAPES = [
    # rows of each expert, N, K
    ([1], 8, 8), ([1, 0, 2], 16, 64), ([5], 264, 40), ([0, 0, 3, 0], 128, 128), ([17, 1, 0, 33], 256, 72), ([64, 63, 65], 136, 200), ([130, 0, 1, 255, 256, 257], 520, 328),
    ([300], 1000, 520), ([2, 700, 3], 256, 1024), ([16] * 9, 384, 192), ([1] * 70, 64, 96), ([129, 127], 24, 2304), ([48, 80, 15, 16, 17], 2304, 64), ([1100, 0], 128, 128),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_products_and_gradients(shape, dtype):
    Case(dtype, *shape).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [([3, 0, 70], 33, 65), ([5, 9], 7, 1), ([20, 1], 1, 31), ([64, 2], 129, 130)])
def test_odd_sizes(shape, dtype):
    Case(dtype, *shape).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("first,spare,pad,lead", [(0, 5, 0, 0), (3, 0, 0, 0), (7, 130, 8, 0), (0, 1, 0, 8), (1, 1, 4, 4), (0, 0, 1, 0), (0, 0, 0, 1)])
def test_rows_of_no_expert_and_slices_of_wider_rows(dtype, first, spare, pad, lead):
    Case(dtype, [40, 0, 129], 136, 96, first, spare, pad, lead).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_integers_are_exact(dtype):
    c = Case(dtype, [37, 200, 0, 5], 272, 144)
    for name in ("x", "dy"):
        v = c.rng.integers(-2, 3, getattr(c, name).shape).astype(np.float64)
        setattr(c, name, v)
        c.dev[name] = c.rows_of(v)
    c.w = c.rng.integers(-2, 3, c.w.shape).astype(np.float64)
    c.dev_w = torch.from_numpy(c.w).cuda().to(TORCH[dtype])
    y = c.check()
    want = torch.from_numpy(ref.grouped(c.x, c.w, c.offsets)).to(TORCH[dtype]).double().numpy()
    assert np.array_equal(y.host(), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_not_finite_stay_with_their_expert(dtype):
    c = Case(dtype, [10, 3, 70], 64, 128, spare=4)
    for bad in (float("nan"), float("inf")):
        c.dev["x"].view[10:13] = bad                             # the rows of expert 1, and rows of none
        c.dev["x"].view[83:] = bad
        c.dev["dy"].view[10:13] = bad
        c.dev["dy"].view[83:] = bad
        y, dw = c.rows_of(np.zeros((c.rows, 64))), torch.zeros(3, 64, 128, device="cuda", dtype=TORCH[dtype])
        tdx.check(tdx.tdx_gemm_grouped(c.args(y=y)))
        tdx.check(tdx.tdx_gemm_grouped_dw(c.args(dweight=dw)))
        torch.cuda.synchronize()
        got = y.host()
        assert np.isfinite(got[:10]).all() and np.isfinite(got[13:83]).all() and not np.isfinite(got[10:13]).any()
        assert bool(torch.isfinite(dw[0]).all()) and bool(torch.isfinite(dw[2]).all()) and not bool(torch.isfinite(dw[1]).any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bad_offsets_are_reported_and_touch_nothing(dtype):
    for offsets in ([0, 5, 3, 8], [0, 4, 400, 401], [-3, 2, 4, 8]):
        c = Case(dtype, [3, 2, 3], 64, 64)
        c.dev_offsets = i32(offsets)
        y, dx = c.rows_of(np.zeros((c.rows, 64)), fill=-5.0), c.rows_of(np.zeros((c.rows, 64)), fill=-5.0)
        dw = torch.full((3, 64, 64), -5.0, device="cuda", dtype=TORCH[dtype])
        for call, out in ((tdx.tdx_gemm_grouped, {"y": y}), (tdx.tdx_gemm_grouped_dx, {"dx": dx}), (tdx.tdx_gemm_grouped_dw, {"dweight": dw})):
            tdx.check(call(c.args(**out)))
            assert tdx.tdx_check_device_status() == tdx.TDX_ERR_BOUNDS
        assert y.guards_intact() and dx.guards_intact() and bool(torch.isfinite(dw).all())
    tdx.check(tdx.tdx_check_device_status())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_to_sum_gives_zeros(dtype):
    y = torch.full((5, 8), -5.0, device="cuda", dtype=TORCH[dtype])
    a = tdx.tdx_grouped_args(rows=5, experts=2, N=8, K=0, dtype=DT[dtype], offsets=i32([0, 2, 4]), y=y, ld_y=8)
    tdx.check(tdx.tdx_gemm_grouped(a))
    dw = torch.full((2, 8, 16), -5.0, device="cuda", dtype=TORCH[dtype])
    b = tdx.tdx_grouped_args(rows=0, experts=2, N=8, K=16, dtype=DT[dtype], offsets=i32([0, 0, 0]), dweight=dw, ld_x=16, ld_dy=8)
    tdx.check(tdx.tdx_gemm_grouped_dw(b))
    torch.cuda.synchronize()
    assert bool((y[:4] == 0).all()) and bool((y[4] == -5).all()) and bool((dw == 0).all())


def test_captured_and_replayed_with_other_offsets():
    c = Case("bf16", [70, 0, 200, 30], 256, 128)
    y = c.rows_of(np.zeros((c.rows, 256)))
    a = c.args(y=y)
    tdx.check(tdx.tdx_gemm_grouped(a))
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        tdx.check(tdx.tdx_gemm_grouped(a, torch.cuda.current_stream()))
    for offsets in ([0, 300, 300, 300, 300], [0, 1, 2, 3, 300], [0, 70, 70, 270, 300]):
        c.dev_offsets.copy_(torch.tensor(offsets))
        y.view.fill_(-5.0)
        graph.replay()
        torch.cuda.synchronize()
        close("y", y.host(), ref.grouped(c.x, c.w, offsets), ref.grouped(abs(c.x), abs(c.w), offsets), c.k, "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [
    ([(37 * i) % 700 for i in range(24)], 2304, 64),             # several rounds of tiles, leftovers of every size
    ([(53 * i) % 151 for i in range(140)], 64, 72),              # more experts than are sorted
    ([i % 3 for i in range(1030)], 40, 64),                      # more experts than the tensor-core kernel takes
], ids=["rounds", "unsorted", "thousand"])
def test_many_tiles_and_experts(shape, dtype):
    Case(dtype, *shape).check()


# more than 512 rows an expert: tiles of 256 features for dw too; the last with more tiles than SMs
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [([600, 700, 513], 264, 264), ([900, 0, 1100], 264, 72), ([1300], 136, 520), ([601, 640, 560, 700], 2304, 1096)])
def test_many_rows_an_expert(shape, dtype):
    Case(dtype, *shape).check()
