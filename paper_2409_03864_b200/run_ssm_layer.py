"""A selective state-space layer on the library's operators: a prompt, then single tokens, and a training step.

  python -m paper_2409_03864_b200.run_ssm_layer [--width 512] [--lengths 37,1,200] [--tokens 8]

The layer maps rows u (width E) to rows of the same width: an input projection to 2 D channels (x and the gate z), the short
causal convolution with SiLU, a projection of its result to the low-rank step, B and C, a projection of the step to D channels, the
selective scan, and an output projection.  Prompts of different lengths run packed, with tdx_gemm for the projections; their
states go to slots of a cache, from which single tokens go on, with tdx_gemm_w4 for the projections.  The same tokens appended
to the prompts and run as prompts must give the same outputs (up to the rounding of 4-bit against bf16 weights, which is why the
prompts of the comparison run with the 4-bit weights too).  All work goes to the caller's current stream, the library's calls as well
as torch's.  Prompts and gradients make their buffers per call; single tokens work in buffers that are made once, so that a token
step can be captured in a CUDA graph (after one step outside of it).
"""
from __future__ import annotations

import argparse

import torch

from . import binding as tdx

BF16 = torch.bfloat16


def _call(function, *args):
    """A call of the library on the current stream, so that it comes after torch's work there and before what follows."""
    tdx.check(function(*args, stream=torch.cuda.current_stream()))


class Linear:
    """y = x W^T with bf16 weights for many rows and the same weights in 4 bits for few."""

    def __init__(self, n, k, g, group=64):
        w = (torch.randn(n, k, generator=g, device="cuda") / k ** 0.5).to(BF16)
        self.n, self.k, self.group = n, k, group
        self.packed = torch.empty(n, k // 2, dtype=torch.uint8, device="cuda")
        self.scales = torch.empty(n, k // group, dtype=BF16, device="cuda")
        self.zeros = torch.empty(n, k // group, dtype=torch.uint8, device="cuda")
        _call(tdx.tdx_w4_quantize, n, k, group, tdx.TDX_BF16, w, k, self.packed, self.scales, self.zeros)
        # the weights that the 4 bits stand for, so that prompts and single tokens run the same layer
        q = torch.stack([self.packed & 15, self.packed >> 4], dim=2).view(n, k // group, group).float()
        self.weight = ((q - self.zeros.float()[:, :, None]) * self.scales.float()[:, :, None]).view(n, k).to(BF16)

    def many(self, x, y):
        _call(tdx.tdx_gemm, x.shape[0], self.n, self.k, 0, 1, 1.0, tdx.TDX_BF16, x, self.weight, y)

    def few(self, x, y):
        _call(tdx.tdx_gemm_w4, tdx.tdx_w4_args(
            M=x.shape[0], N=self.n, K=self.k, group_size=self.group, dtype=tdx.TDX_BF16, x=x, ld_x=x.stride(0), weight=self.packed,
            scales=self.scales, zeros=self.zeros, y=y, ld_y=y.stride(0)))


class Layer:
    def __init__(self, width=512, expand=2, states=16, rank=64, filter_width=4, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.E, self.D, self.N, self.R, self.W = width, expand * width, states, rank, filter_width
        self.proj_in, self.proj_out = Linear(2 * self.D, width, g), Linear(width, self.D, g)
        self.proj_x = Linear(rank + 2 * states, self.D, g)
        self.proj_dt = Linear(self.D, rank, g, min(64, rank))
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.conv_w, self.conv_b = rand(self.D, filter_width) * 0.3, rand(self.D) * 0.1
        self.A = -torch.arange(1, states + 1, device="cuda").float().repeat(self.D, 1)
        self.skip = torch.ones(self.D, device="cuda")
        step = torch.exp(torch.rand(self.D, generator=g, device="cuda") * 4.6 - 6.9)
        self.dt_bias = step + torch.log(-torch.expm1(-step))

    def cache(self, slots):
        """Zero states for `slots` sequences."""
        return (torch.zeros(slots, self.W - 1, self.D, dtype=BF16, device="cuda"), torch.zeros(slots, self.D, self.N, device="cuda"))

    def buffers(self, rows):
        e = lambda n: torch.empty(rows, n, dtype=BF16, device="cuda")  # noqa: E731
        return {"xz": e(2 * self.D), "conv": e(self.D), "proj": e(self.R + 2 * self.N), "low": e(self.R), "dt": e(self.D), "y": e(self.D), "out": e(self.E)}

    def conv_args(self, b, **more):
        return tdx.tdx_conv1d_args(channels=self.D, width=self.W, dtype=tdx.TDX_BF16, silu=1, x=b["xz"], ld_x=2 * self.D, weight=self.conv_w,
                                   bias=self.conv_b, y=b["conv"], ld_y=self.D, **more)

    def scan_args(self, b, **more):
        p = b["proj"]
        return tdx.tdx_scan_args(
            channels=self.D, states=self.N, groups=1, dtype=tdx.TDX_BF16, dt_softplus=1, x=b["conv"], ld_x=self.D, dt=b["dt"], ld_dt=self.D, A=self.A,
            B=p[:, self.R:], ld_B=p.stride(0), C=p[:, self.R + self.N:], ld_C=p.stride(0), D=self.skip, z=b["xz"][:, self.D:], ld_z=2 * self.D,
            dt_bias=self.dt_bias, out=b["y"], ld_out=self.D, **more)

    def _run(self, u, b, apply, conv, scan):
        apply(self.proj_in, u, b["xz"])
        _call(*conv)
        apply(self.proj_x, b["conv"], b["proj"])
        b["low"].copy_(b["proj"][:, :self.R])
        apply(self.proj_dt, b["low"], b["dt"])
        _call(*scan)
        apply(self.proj_out, b["y"], b["out"])
        return b["out"]

    def prompts(self, u, lengths, cache, slots, keep=None):
        """Packed prompts; their states go to the cache.  keep: a dict that gets what a backward pass needs."""
        b = self.buffers(u.shape[0])
        offsets = torch.tensor([0] + list(lengths), device="cuda").cumsum(0).to(torch.int32)
        slots = torch.tensor(slots, dtype=torch.int32, device="cuda")
        common = dict(batch=len(lengths), max_len=max(lengths), rows=u.shape[0], seq_offsets=offsets, slots=slots, n_slots=cache[0].shape[0])
        conv, scan = self.conv_args(b, state_out=cache[0], **common), self.scan_args(b, state_out=cache[1], **common)
        if keep is not None:
            status, size = tdx.tdx_selective_scan_saved_size(scan)
            tdx.check(status)
            keep["saved"] = torch.empty(size, dtype=torch.uint8, device="cuda")
            scan.set(saved=keep["saved"], saved_bytes=size)
        status, size = tdx.tdx_selective_scan_workspace_size(scan)
        tdx.check(status)
        workspace = torch.empty(size, dtype=torch.uint8, device="cuda")
        scan.set(workspace=workspace, workspace_bytes=size)
        out = self._run(u, b, Linear.many, (tdx.tdx_causal_conv1d, conv), (tdx.tdx_selective_scan, scan))
        if keep is not None:
            keep.update(b=b, conv=conv, scan=scan, workspace=workspace, offsets=offsets, slots=slots)
        return out

    def tokens(self, u, cache, slots, b):
        """One token for each row of u, in place on the cache."""
        common = dict(batch=u.shape[0], slots=slots, n_slots=cache[0].shape[0])
        conv = self.conv_args(b, state_in=cache[0], state_out=cache[0], **common)
        scan = self.scan_args(b, state_in=cache[1], state_out=cache[1], **common)
        return self._run(u, b, Linear.few, (tdx.tdx_causal_conv1d_step, conv), (tdx.tdx_selective_scan_step, scan))

    def between_gradients(self, keep, dy):
        """Gradients of what stands between the projections for a gradient dy of the scan's output: d conv input, d dt, d B, d C, d z and
        the parameters'.  (The projections' are products that tdx_gemm computes with the operands transposed.)"""
        b, scan, conv = keep["b"], keep["scan"], keep["conv"]
        rows = dy.shape[0]
        e = lambda n: torch.empty(rows, n, dtype=BF16, device="cuda")  # noqa: E731
        g = {"dx": e(self.D), "ddt": e(self.D), "dB": e(self.N), "dC": e(self.N), "dz": e(self.D)}
        p = {"dA": torch.empty_like(self.A), "dD": torch.empty_like(self.skip), "ddt_bias": torch.empty_like(self.dt_bias)}
        scan.set(dout=dy, ld_dout=dy.stride(0), **g, **{"ld_" + k: v.stride(0) for k, v in g.items()}, **p, state_out=None)
        _call(tdx.tdx_selective_scan_bwd, scan)
        g["dconv_in"], p["dconv_w"], p["dconv_b"] = e(self.D), torch.empty_like(self.conv_w), torch.empty_like(self.conv_b)
        conv.set(dy=g["dx"], ld_dy=self.D, dx=g["dconv_in"], ld_dx=self.D, dweight=p["dconv_w"], dbias=p["dconv_b"], state_out=None)
        status, size = tdx.tdx_causal_conv1d_workspace_size(conv)
        tdx.check(status)
        workspace = torch.empty(size, dtype=torch.uint8, device="cuda")
        conv.set(workspace=workspace, workspace_bytes=size)
        _call(tdx.tdx_causal_conv1d_bwd, conv)
        assert b["y"].shape == dy.shape
        return g | p


def prompt_and_tokens(layer, lengths, tokens, seed=1):
    """Outputs of the last `tokens` rows of every sequence, once as single tokens after a prompt and once as part of the prompt."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    count, slots = len(lengths), [2 * i + 1 for i in range(len(lengths))]
    u = [torch.randn(n + tokens, layer.E, generator=g, device="cuda").to(BF16) for n in lengths]
    cache = layer.cache(2 * count + 1)
    layer.prompts(torch.cat([v[:n] for v, n in zip(u, lengths)]), lengths, cache, slots)
    b, order = layer.buffers(count), torch.tensor(slots, dtype=torch.int32, device="cuda")
    steps = []
    for t in range(tokens):
        steps.append(layer.tokens(torch.stack([v[n + t] for v, n in zip(u, lengths)]), cache, order, b).clone())
    whole_cache = layer.cache(2 * count + 1)
    whole = layer.prompts(torch.cat(u), [n + tokens for n in lengths], whole_cache, slots)
    ends = torch.tensor([n + tokens for n in lengths]).cumsum(0).tolist()
    want = torch.stack([whole[e - tokens:e] for e in ends], dim=1)
    return torch.stack(steps), want, cache, whole_cache


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--lengths", default="37,1,200")
    ap.add_argument("--tokens", type=int, default=8)
    a = ap.parse_args(argv)
    lengths = [int(v) for v in a.lengths.split(",")]
    layer = Layer(a.width)
    got, want, cache, whole = prompt_and_tokens(layer, lengths, a.tokens)
    off = (got.float() - want.float()).norm() / want.float().norm()
    print(f"{len(lengths)} prompts of {a.lengths} rows, then {a.tokens} tokens each: relative difference to longer prompts {off:.2e}, "
          f"states {(cache[1] - whole[1]).norm() / whole[1].norm():.2e}")
    keep = {}
    u = torch.randn(sum(lengths), layer.E, device="cuda").to(BF16)
    layer.prompts(u, lengths, layer.cache(len(lengths)), list(range(len(lengths))), keep)
    grads = layer.between_gradients(keep, torch.randn(sum(lengths), layer.D, device="cuda").to(BF16))
    _call(tdx.tdx_check_device_status)
    print("gradients:", ", ".join(f"{k} {v.float().norm():.3g}" for k, v in grads.items()))


if __name__ == "__main__":
    main()
