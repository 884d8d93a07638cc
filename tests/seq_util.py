"""Device buffers and comparisons for the tests of the sequence operators."""
import numpy as np
import torch

import paper_2409_03864_b200 as tdx

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
DT = {"f32": tdx.TDX_F32, "bf16": tdx.TDX_BF16}
EPS = 2.0 ** -24                                  # half a unit in the last place of fp32
BITS = {"f32": 24, "bf16": 8}                     # significant bits
CANARY = -77.0


class Rows:
    """A tensor of `rows` rows of `width` values inside a wider allocation: `pad` values behind every row and a guard band of rows
    on either side, all holding a canary."""

    def __init__(self, values, dtype, pad=0, lead=0, fill=None):
        values = np.asarray(values, dtype=np.float64)
        self.shape = values.shape
        rows = values.shape[0]
        flat = values.reshape(rows, -1) if rows else values.reshape(0, int(np.prod(values.shape[1:])))
        self.width, self.lead = flat.shape[1], lead
        self.ld = self.width + pad + lead
        self.full = torch.full((rows + 2, max(self.ld, 1)), CANARY, dtype=TORCH[dtype], device="cuda")
        if rows and self.width:
            self.view[:] = torch.from_numpy(flat).cuda().to(TORCH[dtype]) if fill is None else fill

    @property
    def view(self):
        return self.full[1:-1, self.lead:self.lead + self.width]

    @property
    def ptr(self):
        return self.full.data_ptr() + (self.ld + self.lead) * self.full.element_size()

    def host(self):
        return self.view.double().cpu().numpy().reshape(self.shape)

    def guards_intact(self):
        f = self.full.float().clone()
        f[1:-1, self.lead:self.lead + self.width] = CANARY
        return bool((f == CANARY).all())


def seeded(rng, shape, dtype, scale=1.0, lo=None, hi=None):
    """Values that the type holds exactly, as float64."""
    v = rng.standard_normal(shape) * scale if lo is None else rng.uniform(lo, hi, shape)
    return torch.from_numpy(np.asarray(v)).to(TORCH[dtype]).double().numpy()


def f32(v):
    return torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).cuda()


def i32(v):
    return None if v is None else torch.tensor(list(v), dtype=torch.int32, device="cuda")


def half_ulp(v, dtype):
    """Half the distance between neighbouring numbers of the type at v (normal range)."""
    return np.ldexp(1.0, np.frexp(v)[1] - BITS[dtype] - 1)


def assert_close(name, got, want, magnitude, factor, dtype="f32"):
    """|got - want| <= factor * magnitude + the rounding to the output type."""
    tol = factor * magnitude + half_ulp(np.abs(want) + factor * magnitude, dtype) + 1e-37
    bad = ~(np.abs(got - want) <= tol)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{name}: {bad.sum()} of {bad.size} values off, first at {i}: {got[i]} instead of {want[i]}, tolerance {tol[i]:.3g}")


def assert_close_but_infinities(name, got, want, magnitude, factor, dtype="f32"):
    """What is infinite or undefined is so on both sides; the rest is close."""
    there = np.isfinite(want)
    wrong = np.argwhere(~((got == want) | (np.isnan(got) & np.isnan(want))) & ~there)
    assert not len(wrong), (name, wrong[0], got[tuple(wrong[0])], want[tuple(wrong[0])])
    assert_close(name, got[there], want[there], magnitude[there], factor, dtype)


def workspace(answer):
    status, size = answer
    tdx.check(status)
    return torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")      # NaN patterns: nothing may rely on zeros


def offsets_of(lengths):
    return np.concatenate([[0], np.cumsum(lengths)])
