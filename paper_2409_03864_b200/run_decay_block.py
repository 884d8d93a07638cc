"""A block of linear attention with decay and experts on the library's operators: a prompt, then single tokens, and gradients.

  python -m paper_2409_03864_b200.run_decay_block [--width 256] [--lengths 130,1,40] [--tokens 6]

The block maps rows x (width E) to rows of the same width:

  h  = norm(x)                                  tdx_block_norm (only y)
  q, k, v, g = h W_in^T                         tdx_gemm; k and v have half as many heads as q
  o  = attention with decay of q, k, v          tdx_decay_attention, or _step on states in slots of a cache
  a  = norm of every head of o, times silu(g)   tdx_block_norm (groups of a head's channels, only the sum)
  s  = x + scale_1 norm(a W_out^T),  n = norm(s)    tdx_gemm, tdx_block_norm (all of it)
  e  = argmax of n W_router^T; rows sorted by e
  d  = silu(n W_up[e]^T) W_down[e]^T            tdx_gemm_grouped
  y  = s + scale_2 d                            tdx_block_norm (no norms)

The router is fixed (the experts' choice has no gradient).  All work goes to the caller's current stream, the library's calls as well as
torch's.  Sorting and the experts' activation are torch's.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as tdx

BF16 = torch.bfloat16
EPS = 1e-5


def _call(function, *args):
    """A call of the library on the current stream, so that it comes after torch's work there and before what follows."""
    tdx.check(function(*args, stream=torch.cuda.current_stream()))


def _new(*shape, dtype=BF16):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def _rows(**tensors):
    """Fields of an argument block for tensors of rows: their addresses and the distance of rows."""
    given = {k: v for k, v in tensors.items() if v is not None}
    return {**given, **{"ld_" + k: v.stride(0) for k, v in given.items()}}


def _workspace(args, answer):
    status, size = answer
    tdx.check(status)
    space = _new(max(size, 1), dtype=torch.uint8)
    args.set(workspace=space, workspace_bytes=size)
    return space


def _product(x, w):
    """x W^T"""
    y = _new(x.shape[0], w.shape[0])
    _call(tdx.tdx_gemm, x.shape[0], w.shape[0], w.shape[1], 0, 1, 1.0, tdx.TDX_BF16, x, w, y)
    return y


def _product_gradients(x, w, dy):
    dx, dw = _new(*x.shape), _new(*w.shape)
    _call(tdx.tdx_gemm, x.shape[0], w.shape[1], w.shape[0], 0, 0, 1.0, tdx.TDX_BF16, dy, w, dx)
    _call(tdx.tdx_gemm, w.shape[0], w.shape[1], x.shape[0], 1, 0, 1.0, tdx.TDX_BF16, dy, x, dw)
    return dx, dw


class Norm:
    """tdx_block_norm with its parameters; `keep` of forward() is what backward() takes."""

    def __init__(self, channels, group=0, inner=True, scale=False, outer=False):
        self.channels, self.group, self.inner = channels, group, inner
        one = lambda there, v=1.0: torch.full((channels,), v, device="cuda") if there else None  # noqa: E731
        self.weight_in, self.scale, self.weight_out = one(inner), one(scale, 0.5), one(outer)

    def _args(self, x, gate, residual, **more):
        return tdx.tdx_norm_args(rows=x.shape[0], channels=self.channels, group=self.group, dtype=tdx.TDX_BF16, norm_in=int(self.inner), eps=EPS,
                                 weight_in=self.weight_in, scale=self.scale, weight_out=self.weight_out, **_rows(x=x, gate=gate, residual=residual), **more)

    def forward(self, x, gate=None, residual=None, want_sum=True):
        total = _new(*x.shape) if want_sum else None
        y = _new(*x.shape) if self.weight_out is not None else None
        _call(tdx.tdx_block_norm, self._args(x, gate, residual, **_rows(sum=total, y=y)))
        return total, y, (x, gate, residual)

    def backward(self, keep, dsum, dy, dgate=None):
        """(dx, dgate, dresidual) and a dict of the parameters' gradients."""
        x, gate, residual = keep
        dx, dres = _new(*x.shape), _new(*x.shape) if residual is not None else None
        grads = {"d" + n: _new(self.channels, dtype=torch.float32) for n in ("weight_in", "scale", "weight_out") if getattr(self, n) is not None}
        a = self._args(x, gate, residual, **_rows(dsum=dsum, dy=dy, dx=dx, dgate=dgate, dresidual=dres), **grads)
        space = _workspace(a, tdx.tdx_block_norm_workspace_size(a))  # noqa: F841  (held until the call is enqueued)
        _call(tdx.tdx_block_norm_bwd, a)
        return dx, dres, grads


class Block:
    def __init__(self, width=256, heads=4, dim=64, experts=4, hidden=384, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rand = lambda *s: (torch.randn(*s, generator=g, device="cuda") / s[-1] ** 0.5).to(BF16)  # noqa: E731
        self.E, self.H, self.D, self.kv, self.experts, self.hidden = width, heads, dim, max(1, heads // 2), experts, hidden
        self.split = [heads * dim, self.kv * dim, self.kv * dim, heads * dim]
        self.w_in, self.w_out = rand(sum(self.split), width), rand(width, heads * dim)
        self.router, self.w_up, self.w_down = rand(experts, width), rand(experts, hidden, width), rand(experts, width, hidden)
        self.log_decay = torch.log1p(-torch.exp2(-torch.linspace(2.0, 7.0, heads, device="cuda")))
        self.norm_1 = Norm(width, inner=False, outer=True)
        self.norm_heads = Norm(heads * dim, group=dim)
        self.norm_2 = Norm(width, scale=True, outer=True)
        self.add = Norm(width, inner=False, scale=True)

    def cache(self, slots):
        return torch.zeros(slots, self.H, self.D, self.D, device="cuda")

    def attention_args(self, q, k, v, out, **more):
        return tdx.tdx_attention_args(heads=self.H, q_heads=self.H, k_heads=self.kv, v_heads=self.kv, dim_k=self.D, dim_v=self.D, dtype=tdx.TDX_BF16,
                                      scale=self.D ** -0.5, log_decay=self.log_decay, **_rows(q=q, k=k, v=v, out=out), **more)

    def grouped_args(self, offsets, w, **rows):
        x = rows.get("x", rows.get("dx"))
        a = tdx.tdx_grouped_args(rows=x.shape[0], experts=self.experts, N=w.shape[1], K=w.shape[2], dtype=tdx.TDX_BF16, offsets=offsets, weight=w, **_rows(**rows))
        self.space = _workspace(a, tdx.tdx_gemm_grouped_workspace_size(a))
        return a

    def _run(self, x, attend):
        keep = {}
        _, h, keep["norm_1"] = self.norm_1.forward(x, want_sum=False)
        qkvg = _product(h, self.w_in)
        q, k, v, g = qkvg.split(self.split, dim=1)
        o = _new(x.shape[0], self.H * self.D)
        attend(q, k, v, o)
        a, _, keep["heads"] = self.norm_heads.forward(o, gate=g)
        p = _product(a, self.w_out)
        s, n, keep["norm_2"] = self.norm_2.forward(p, residual=x)
        expert = _product(n, self.router).argmax(1)
        order = torch.argsort(expert, stable=True)
        offsets = torch.searchsorted(expert[order], torch.arange(self.experts + 1, device="cuda")).to(torch.int32)
        rows = n[order]
        u, down = _new(x.shape[0], self.hidden), _new(x.shape[0], self.E)
        _call(tdx.tdx_gemm_grouped, self.grouped_args(offsets, self.w_up, x=rows, y=u))
        act = torch.nn.functional.silu(u)
        _call(tdx.tdx_gemm_grouped, self.grouped_args(offsets, self.w_down, x=act, y=down))
        d = torch.empty_like(down)
        d[order] = down
        y, _, keep["add"] = self.add.forward(d, residual=s)
        keep.update(h=h, qkvg=qkvg, o=o, a=a, order=order, offsets=offsets, rows=rows, u=u, act=act)
        return y, keep

    def prompts(self, x, lengths, cache=None, slots=None):
        """Packed prompts; their states go to the cache.  Returns y and what gradients() takes."""
        offsets = torch.tensor([0] + list(lengths), device="cuda").cumsum(0).to(torch.int32)
        more = dict(batch=len(lengths), max_len=max(lengths), rows=x.shape[0], seq_offsets=offsets)
        if cache is not None:
            where = torch.tensor(slots, dtype=torch.int32, device="cuda")
            more.update(state_out=cache, slots=where, n_slots=cache.shape[0])
        held = []

        def attend(q, k, v, o):
            a = self.attention_args(q, k, v, o, **more)
            held.append((a, _workspace(a, tdx.tdx_decay_attention_workspace_size(a))))
            _call(tdx.tdx_decay_attention, a)

        y, keep = self._run(x, attend)
        keep.update(more={k: v for k, v in more.items() if k in ("batch", "max_len", "rows", "seq_offsets")}, held=held)
        return y, keep

    def tokens(self, x, cache, slots):
        """One token for each row of x, in place on the cache."""
        def attend(q, k, v, o):
            _call(tdx.tdx_decay_attention_step, self.attention_args(q, k, v, o, batch=x.shape[0], slots=slots, n_slots=cache.shape[0], state_in=cache, state_out=cache))

        return self._run(x, attend)[0]

    def gradients(self, keep, dy):
        """Gradients of x and of all parameters for a gradient dy of prompts() (without states)."""
        g = {}
        dd, ds, p = self.add.backward(keep["add"], dy, None)
        g["scale_2"] = p["dscale"]
        order, offsets = keep["order"], keep["offsets"]
        dd = dd[order]
        dact, drows = torch.empty_like(keep["act"]), torch.empty_like(keep["rows"])
        g["w_down"], g["w_up"] = torch.empty_like(self.w_down), torch.empty_like(self.w_up)
        a = self.grouped_args(offsets, self.w_down, x=keep["act"], dy=dd, dx=dact).set(dweight=g["w_down"])
        _call(tdx.tdx_gemm_grouped_dx, a)
        _call(tdx.tdx_gemm_grouped_dw, a)
        u = keep["u"].float()
        sig = torch.sigmoid(u)
        du = (dact.float() * sig * (1 + u * (1 - sig))).to(BF16)
        a = self.grouped_args(offsets, self.w_up, x=keep["rows"], dy=du, dx=drows).set(dweight=g["w_up"])
        _call(tdx.tdx_gemm_grouped_dx, a)
        _call(tdx.tdx_gemm_grouped_dw, a)
        dn = torch.empty_like(drows)
        dn[order] = drows
        dp, dx, p = self.norm_2.backward(keep["norm_2"], ds, dn)
        g["norm_2_in"], g["scale_1"], g["norm_2_out"] = p["dweight_in"], p["dscale"], p["dweight_out"]
        da, g["w_out"] = _product_gradients(keep["a"], self.w_out, dp)
        dqkvg = torch.empty_like(keep["qkvg"])
        dq, dk, dv, dg = dqkvg.split(self.split, dim=1)
        do, _, p = self.norm_heads.backward(keep["heads"], da, None, dgate=dg)
        g["norm_heads"] = p["dweight_in"]
        q, k, v, _ = keep["qkvg"].split(self.split, dim=1)
        args = self.attention_args(q, k, v, None, **keep["more"], **_rows(dout=do, dq=dq, dk=dk, dv=dv))
        space = _workspace(args, tdx.tdx_decay_attention_workspace_size(args))  # noqa: F841
        _call(tdx.tdx_decay_attention_bwd, args)
        dh, g["w_in"] = _product_gradients(keep["h"], self.w_in, dqkvg)
        dx_1, _, p = self.norm_1.backward(keep["norm_1"], None, dh)
        g["norm_1"] = p["dweight_out"]
        g["x"] = dx.float() + dx_1.float()
        return g


def prompt_and_tokens(block, lengths, tokens, seed=1):
    """Outputs of the last `tokens` rows of every sequence, once as single tokens after a prompt and once as part of the prompt."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    count, slots = len(lengths), [2 * i + 1 for i in range(len(lengths))]
    x = [torch.randn(n + tokens, block.E, generator=g, device="cuda").to(BF16) for n in lengths]
    cache, whole_cache = block.cache(2 * count + 1), block.cache(2 * count + 1)
    block.prompts(torch.cat([v[:n] for v, n in zip(x, lengths)]), lengths, cache, slots)
    where = torch.tensor(slots, dtype=torch.int32, device="cuda")
    steps = [block.tokens(torch.stack([v[n + t] for v, n in zip(x, lengths)]), cache, where) for t in range(tokens)]
    whole, _ = block.prompts(torch.cat(x), [n + tokens for n in lengths], whole_cache, slots)
    ends = torch.tensor([n + tokens for n in lengths]).cumsum(0).tolist()
    return torch.stack(steps), torch.stack([whole[e - tokens:e] for e in ends], dim=1), cache, whole_cache


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--lengths", default="130,1,40")
    ap.add_argument("--tokens", type=int, default=6)
    a = ap.parse_args(argv)
    lengths = [int(v) for v in a.lengths.split(",")]
    block = Block(a.width)
    got, want, cache, whole = prompt_and_tokens(block, lengths, a.tokens)
    off = (got.float() - want.float()).norm() / want.float().norm()
    print(f"{len(lengths)} prompts of {a.lengths} rows, then {a.tokens} tokens each: relative difference to longer prompts {off:.2e}, "
          f"states {(cache - whole).norm() / whole.norm():.2e}")
    x = torch.randn(sum(lengths), block.E, device="cuda").to(BF16)
    _, keep = block.prompts(x, lengths)
    grads = block.gradients(keep, torch.randn(x.shape, device="cuda").to(BF16))
    _call(tdx.tdx_check_device_status)
    print("gradients:", ", ".join(f"{k} {v.float().norm():.3g}" for k, v in grads.items()))


if __name__ == "__main__":
    main()
