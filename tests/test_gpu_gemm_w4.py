"""GPU parity of products with 4-bit weights, and of their quantisation, with 64-bit definitions."""
import numpy as np
import pytest
import torch

import paper_2409_03864_b200 as tdx
import seq_reference as ref
from seq_util import DT, EPS, TORCH, Rows, assert_close, seeded

pytestmark = pytest.mark.gpu


def run(dtype, m, n, k, group, zeros, seed=0, pad=0, lead=0, out_pad=0, shift=0):
    rng = np.random.default_rng(seed)
    groups = -(-k // group)
    x = seeded(rng, (m, k), dtype)
    pitch = (k + 1) // 2
    weight = rng.integers(0, 256, (n, pitch), dtype=np.uint8)
    scales = seeded(rng, (n, groups), dtype, lo=0.01, hi=0.1)
    z = rng.integers(0, 16, (n, groups), dtype=np.uint8) if zeros else None
    dev_x, y = Rows(x, dtype, pad, lead), Rows(np.zeros((m, n)), dtype, out_pad, fill=float("nan"))
    raw = torch.zeros(n * pitch + shift, dtype=torch.uint8, device="cuda")
    raw[shift:] = torch.from_numpy(weight.reshape(-1)).cuda()
    dev_s = torch.from_numpy(scales).cuda().to(TORCH[dtype])
    dev_z = torch.from_numpy(z).cuda() if zeros else None
    a = tdx.tdx_w4_args(M=m, N=n, K=k, group_size=group, dtype=DT[dtype], x=dev_x.ptr, ld_x=dev_x.ld, weight=raw.data_ptr() + shift, scales=dev_s,
                        zeros=dev_z, y=y.ptr, ld_y=y.ld)
    tdx.check(tdx.tdx_gemm_w4(a))
    torch.cuda.synchronize()
    w = ref.unpack_w4(weight, scales, z, k, group)
    # every product is exact; K additions, and a group's sum is scaled once
    assert_close("y", y.host(), x @ w.T, np.abs(x) @ np.abs(w).T, (k + 8) * EPS, dtype)
    assert y.guards_intact()
    return y


FAST = [
    # m, n, k, group
    (1, 16, 128, 128), (1, 1, 32, 32), (1, 17, 64, 64), (1, 100, 1280, 128), (2, 40, 96, 32), (3, 33, 192, 64), (7, 64, 2304, 128), (8, 50, 2304, 64),
    (9, 48, 512, 32), (16, 31, 1024, 128), (17, 64, 640, 64), (33, 20, 256, 32), (64, 130, 4096, 128), (5, 300, 8192, 128), (100, 16, 384, 128),
]


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", FAST)
def test_products(shape, dtype, zeros):
    run(dtype, *shape, zeros)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 5, 7, 3), (3, 9, 33, 16), (6, 4, 1, 1), (2, 8, 130, 128), (1, 6, 50, 200), (5, 3, 255, 64), (9, 12, 96, 96)])
def test_any_group_and_odd_k(shape, dtype):
    run(dtype, *shape, True)
    run(dtype, *shape, False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,lead,out_pad,shift", [(8, 0, 0, 0), (0, 8, 5, 0), (1, 0, 1, 0), (0, 1, 0, 0), (0, 0, 3, 1), (0, 0, 0, 4), (0, 0, 0, 8)])
def test_slices_and_unaligned_weights(dtype, pad, lead, out_pad, shift):
    for m in (1, 5):
        run(dtype, m, 40, 256, 128, True, pad=pad, lead=lead, out_pad=out_pad, shift=shift)
        run(dtype, m, 40, 256, 32, False, pad=pad, lead=lead, out_pad=out_pad, shift=shift)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_integers_are_exact(dtype):
    rng = np.random.default_rng(2)
    m, n, k, group = 4, 48, 512, 64
    x = rng.integers(-3, 4, (m, k)).astype(np.float64)
    weight, scales = rng.integers(0, 256, (n, k // 2), dtype=np.uint8), np.ones((n, k // group))
    weight[:, 5:] &= 0x99                              # sums stay below 256: exact in bf16 as well
    x[:, 40:] = 0
    dx, y = Rows(x, dtype), Rows(np.zeros((m, n)), dtype)
    dw, ds = torch.from_numpy(weight).cuda(), torch.from_numpy(scales).cuda().to(TORCH[dtype])
    a = tdx.tdx_w4_args(M=m, N=n, K=k, group_size=group, dtype=DT[dtype], x=dx.ptr, ld_x=k, weight=dw, scales=ds, y=y.ptr, ld_y=n)
    tdx.check(tdx.tdx_gemm_w4(a))
    want = x @ ref.unpack_w4(weight, scales, None, k, group).T
    want = torch.from_numpy(want).to(TORCH[dtype]).double().numpy()
    assert np.array_equal(y.host(), want)


def test_rows_with_infinities_and_nan_leave_the_others_alone():
    for dtype in ("f32", "bf16"):
        rng = np.random.default_rng(4)
        m, n, k = 6, 32, 256
        x = seeded(rng, (m, k), dtype)
        x[1, 7], x[3, 100], x[5, 0] = np.inf, np.nan, -np.inf
        weight = rng.integers(0, 256, (n, k // 2), dtype=np.uint8) & 0x77     # q < 8: q - 8 is never zero
        scales = np.full((n, 2), 0.5)
        dx, y = Rows(x, dtype), Rows(np.zeros((m, n)), dtype)
        dw, ds = torch.from_numpy(weight).cuda(), torch.from_numpy(scales).cuda().to(TORCH[dtype])
        a = tdx.tdx_w4_args(M=m, N=n, K=k, group_size=128, dtype=DT[dtype], x=dx.ptr, ld_x=k, weight=dw, scales=ds, y=y.ptr, ld_y=n)
        tdx.check(tdx.tdx_gemm_w4(a))
        w = ref.unpack_w4(weight, scales, None, k, 128)
        got, good = y.host(), [0, 2, 4]
        assert_close("y", got[good], x[good] @ w.T, np.abs(x[good]) @ np.abs(w).T, (k + 8) * EPS, dtype)
        assert (got[1] == -np.inf).all() and (got[5] == np.inf).all() and np.isnan(got[3]).all()


def test_k_of_zero_gives_zeros_and_empty_outputs_are_left_alone():
    y = Rows(np.ones((3, 5)), "f32")
    a = tdx.tdx_w4_args(M=3, N=5, K=0, group_size=128, dtype=tdx.TDX_F32, y=y.ptr, ld_y=5)
    tdx.check(tdx.tdx_gemm_w4(a))
    assert (y.host() == 0).all() and y.guards_intact()
    a.set(N=0)
    tdx.check(tdx.tdx_gemm_w4(a))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("n,k,group,pad", [(5, 256, 128, 0), (3, 70, 32, 2), (4, 33, 64, 0), (2, 96, 6, 1), (1, 1, 1, 0)])
def test_quantisation(n, k, group, pad, zeros, dtype):
    rng = np.random.default_rng(k)
    w = seeded(rng, (n, k), dtype)
    w[0, :min(group, k)] = 0.0                           # a group of zeros
    if n > 2:
        w[2] = np.abs(w[2])                              # a row of one sign
    groups = -(-k // group)
    dev = Rows(w, dtype, pad)
    q = torch.zeros(n, (k + 1) // 2, dtype=torch.uint8, device="cuda")
    s, z = torch.zeros(n, groups, dtype=TORCH[dtype], device="cuda"), torch.zeros(n, groups, dtype=torch.uint8, device="cuda")
    tdx.check(tdx.tdx_w4_quantize(n, k, group, DT[dtype], dev.ptr, dev.ld, q, s, z if zeros else None))
    torch.cuda.synchronize()
    scales, zero = s.double().cpu().numpy(), z.cpu().numpy() if zeros else None
    for g in range(groups):
        part = w[:, g * group:(g + 1) * group]
        lo, hi = np.minimum(part.min(1), 0), np.maximum(part.max(1), 0)
        want = (hi - lo) / 15 if zeros else np.abs(part).max(1) / 7
        want = np.where(want > 0, want, 1.0)
        # the fp32 quotient, then the rounding to the stored type
        assert np.all(np.abs(scales[:, g] - want) <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -22) * want)
    back = ref.unpack_w4(q.cpu().numpy(), scales, zero, k, group)
    of = np.arange(k) // group
    # half a step; the scale's own rounding moves the ends of the range by up to 8 steps' worth of its error, and with zeros the
    # zero's rounding can push an end out by half a step more
    steps = (1.0 if zeros else 0.5) + 15 * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -20)
    assert np.all(np.abs(back - w) <= steps * scales[:, of])
    codes = np.stack([q.cpu().numpy() & 15, q.cpu().numpy() >> 4], axis=2).reshape(n, -1)[:, :k]
    if not zeros:
        assert codes.min() >= 1
    assert (back[0, :min(group, k)] == 0).all()


def test_same_bits_on_another_stream():
    first = run("bf16", 3, 64, 1024, 128, True).view.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = run("bf16", 3, 64, 1024, 128, True).view.clone()
    side.synchronize()
    assert torch.equal(first, again)


@pytest.mark.parametrize("shape", [
    # m, n, k, group: where x, the scales and the ring of weights together pass the shared memory of a block ...
    (1, 4740, 28672, 64), (2, 4740, 14336, 32), (1, 40, 32768, 32), (1, 4740, 17408, 32), (4, 33, 8192, 32),
    # ... and where they just fit, for both numbers of row sets
    (1, 4768, 16384, 32), (1, 40, 16384, 32), (2, 4740, 8192, 32), (4, 4737, 8192, 64),
])
def test_long_rows_and_small_groups(shape):
    run("bf16", *shape, True)


def test_long_rows_and_small_groups_fp32():
    run("f32", 1, 4750, 10880, 32, True)
    run("f32", 1, 300, 10912, 32, False)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype,shape", [
    # more than two sets of 16 rows per SM, a ragged last set, and more steps of K than a warp has in flight
    ("bf16", (1, 4801, 10368, 128)), ("bf16", (8, 4740, 8192, 128)), ("bf16", (3, 4737, 10304, 64)), ("bf16", (5, 4752, 2112, 32)),
    ("f32", (2, 4740, 5376, 128)), ("f32", (1, 4801, 10816, 64)),
    # the same with one set a block
    ("bf16", (1, 100, 16512, 128)), ("bf16", (2, 33, 16384, 64)), ("f32", (1, 50, 10880, 32)),
])
def test_many_rows_of_weights_and_long_sums(dtype, shape, zeros):
    run(dtype, *shape, zeros)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,group", [(2, 64), (20, 128), (3, 48)])
def test_zeros_of_a_whole_byte(m, group, dtype):
    """A zero may be any byte; q - zero is then up to 255 in size."""
    rng = np.random.default_rng(6)
    n, k = 40, 384
    x, weight = seeded(rng, (m, k), dtype), rng.integers(0, 256, (n, k // 2), dtype=np.uint8)
    scales, z = seeded(rng, (n, k // group), dtype, lo=0.01, hi=0.1), rng.integers(0, 256, (n, k // group), dtype=np.uint8)
    dx, y, dw, dz = Rows(x, dtype), Rows(np.zeros((m, n)), dtype), torch.from_numpy(weight).cuda(), torch.from_numpy(z).cuda()
    ds = torch.from_numpy(scales).cuda().to(TORCH[dtype])
    a = tdx.tdx_w4_args(M=m, N=n, K=k, group_size=group, dtype=DT[dtype], x=dx.ptr, ld_x=k, weight=dw, scales=ds, zeros=dz, y=y.ptr, ld_y=n)
    tdx.check(tdx.tdx_gemm_w4(a))
    w = ref.unpack_w4(weight, scales, z, k, group)
    assert_close("y", y.host(), x @ w.T, np.abs(x) @ np.abs(w).T, (k + 8) * EPS, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantisation_of_the_widest_range(dtype):
    """max - min passes the largest number of the type, the scale does not."""
    w = torch.tensor([[3e38, -3e38, 1e38, 0.0], [3.3e38, 0.0, -1e38, 1.0]]).to(TORCH[dtype]).cuda()
    q, s, z = torch.zeros(2, 2, dtype=torch.uint8, device="cuda"), torch.zeros(2, 1, dtype=TORCH[dtype], device="cuda"), torch.zeros(2, 1, dtype=torch.uint8, device="cuda")
    tdx.check(tdx.tdx_w4_quantize(2, 4, 4, DT[dtype], w, 4, q, s, z))
    torch.cuda.synchronize()
    scales, values = s.double().cpu().numpy(), w.double().cpu().numpy()
    want = (values.max(1) - np.minimum(values.min(1), 0)) / 15
    assert np.all(np.abs(scales[:, 0] - want) <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -22) * want)
    back = ref.unpack_w4(q.cpu().numpy(), scales, z.cpu().numpy(), 4, 4)
    assert np.all(np.abs(back - values) <= (1.0 + 15 * 2.0 ** -8) * scales)
