"""Cases that measure the operators of a block with linear attention and experts: attention with a decay for each head, the
norms, gate and residual scale around a block, and products grouped by expert.

A case is a dict of plain values.  prepare() makes its inputs on the GPU from a seed, run() makes one pass: with
own = False in elementary fp32 torch operations, with own = True through the library's entry points.  exact() gives the
same outputs from the definitions in 64 bits.

  decay attention   S[t] = exp(log_decay[h]) S[t - 1] + k[t]^T v[t],   out[t] = scale * q[t] S[t]
  block norm        u = x * rstd(x) * weight_in (over groups of channels),  s = residual + scale * u * silu(gate),
                    y = s * rstd(s) * weight_out
  grouped product   y[t] = x[t] W[e]^T for the rows t of expert e,  dx[t] = dy[t] W[e],  dW[e] = sum_t dy[t]^T x[t]
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-5


def listed():
    return [
        # between two blocks, generation for four users: the stream's sum and the next block's norm, where latency counts
        {"name": "norm tokens", "kind": "norm", "dtype": "bf16", "rows": 4, "d": 4096, "group": 0, "gate": False, "residual": True},
        # the heads' norm and gate behind attention, a long prompt
        {"name": "norm heads", "kind": "norm", "dtype": "bf16", "rows": 8192, "d": 4096, "group": 128, "gate": True, "residual": False},
        # a training step: norm of a block's output, gate, scaled residual sum and the next block's norm, forward and backward
        {"name": "norm train", "kind": "norm_train", "dtype": "bf16", "rows": 8192, "d": 4096, "group": 0, "gate": True, "residual": True},
        # the same in fp32 with odd sizes and norms over groups of channels
        {"name": "norm train fp32", "kind": "norm_train", "dtype": "f32", "rows": 1023, "d": 2000, "group": 40, "gate": True, "residual": True},
        # generation for 64 users, two experts each: few rows an expert, some experts with none
        {"name": "experts tokens", "kind": "experts", "dtype": "bf16", "rows": 128, "experts": 32, "n": 2048, "k": 2048, "spread": 1.0, "spare": 0},
        # a prompt's rows, unevenly spread over the experts
        {"name": "experts prompt", "kind": "experts", "dtype": "bf16", "rows": 8192, "experts": 16, "n": 4096, "k": 2048, "spread": 1.0, "spare": 0},
        # a training step, forward and both gradients; a few rows have lost their expert
        {"name": "experts train", "kind": "experts_train", "dtype": "bf16", "rows": 8200, "experts": 8, "n": 2304, "k": 2048, "spread": 0.5, "spare": 9},
        # fp32, ragged
        {"name": "experts train fp32", "kind": "experts_train", "dtype": "f32", "rows": 1501, "experts": 5, "n": 1000, "k": 520, "spread": 1.0, "spare": 2},
        # one long prompt from a state
        {"name": "attention prompt", "kind": "attn", "dtype": "bf16", "lengths": "4096", "heads": 32, "kv": 32, "dk": 128, "dv": 128},
        # packed prompts in fp32, one empty, one a single token, keys and values shared by pairs of heads
        {"name": "attention prompts fp32", "kind": "attn", "dtype": "f32", "lengths": "700,1,0,33,1500,257", "heads": 6, "kv": 3, "dk": 64, "dv": 80},
        # a training step, forward and backward
        {"name": "attention train", "kind": "attn_train", "dtype": "bf16", "lengths": "2048,2048,2048,2048", "heads": 16, "kv": 16, "dk": 128, "dv": 128},
        # one token for each of 128 users whose states sit in slots of a cache; some batch rows are padding
        {"name": "attention step", "kind": "attn_step", "dtype": "bf16", "batch": 128, "heads": 32, "kv": 32, "dk": 64, "dv": 64},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_train", "norm_train", "experts", "experts", "experts_train", "attn", "attn", "attn_train", "attn_train", "attn_step"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    case = {"kind": kind, "dtype": dtype}
    if kind.startswith("norm"):
        group = rng.choice([0, 0, 32, 64, 128, 40])
        d = _log_int(rng, 200, 8192)
        d = max(1, d // group) * group if group else d
        rows = min(_log_int(rng, 1, 16384), (1 << 25) // d)
        return {**case, "rows": rows, "d": d, "group": group, "gate": rng.random() < 0.6, "residual": rng.random() < 0.6}
    if kind.startswith("experts"):
        train = kind == "experts_train"
        n, k = 8 * _log_int(rng, 16, 512), 8 * _log_int(rng, 16, 512)
        experts = min(_log_int(rng, 2, 64), max(2, (1 << 28) // (n * k)))
        most = int((1 << (35 if dtype == "bf16" else 32)) // (n * k) // (3 if train else 1))
        rows = max(2, min(_log_int(rng, 1, 16384), most))
        return {**case, "rows": rows, "experts": experts, "n": n, "k": k, "spread": round(rng.uniform(0.0, 1.5), 2), "spare": rng.choice([0, 0, 1, min(7, rows - 1)])}
    heads = _log_int(rng, 1, 32)
    kv = rng.choice([v for v in (heads, heads, heads // 2, heads // 4, 1) if v and heads % v == 0])
    case.update(heads=heads, kv=kv, dk=rng.choice([32, 64, 64, 72, 96, 128, 128]), dv=rng.choice([32, 64, 64, 80, 128, 128]))
    if kind == "attn_step":
        return {**case, "batch": _log_int(rng, 1, 256)}
    most = (1 << (24 if dtype == "bf16" else 22)) // (heads * max(case["dk"], case["dv"]))
    total = max(4, min(_log_int(rng, 16, 8192), most))
    count = min(_log_int(rng, 1, 8), total)
    if rng.random() < 0.4:
        lengths = [max(1, total // count)] * count
    else:
        cuts = sorted(rng.randint(0, total) for _ in range(count - 1))
        lengths = [b - a for a, b in zip([0] + cuts, cuts + [total])]
    return {**case, "lengths": ",".join(str(v) for v in lengths)}


# ------------------------------------------------------------------------------------------------ inputs


def _lengths(case):
    return [int(v) for v in case["lengths"].split(",")]


def _shares(case, seed):
    """Rows of each expert: shares that differ the more the larger `spread` is, about one expert in eight without rows."""
    g = torch.Generator().manual_seed(seed)
    share = torch.exp(case["spread"] * torch.randn(case["experts"], generator=g, dtype=torch.float64))
    share[torch.rand(case["experts"], generator=g) < 0.125] = 0.0
    share[int(torch.randint(case["experts"], (1,), generator=g))] += 0.5
    ends = torch.round(share.cumsum(0) / share.sum() * (case["rows"] - case["spare"])).to(torch.int64)
    return torch.cat([torch.zeros(1, dtype=torch.int64), ends])


def _pad_index(s, ends, longest, align):
    """[sequence, place] -> row, behind the last row where there is none; align = "left" or "right" within the places."""
    starts, counts = ends[:-1], ends[1:] - ends[:-1]
    place = torch.arange(longest, device="cuda")
    place = place[None, :] - (longest - counts[:, None] if align == "right" else 0)
    there = (place >= 0) & (place < counts[:, None])
    s["at"] = torch.where(there, starts[:, None] + place, s["rows"])
    s["place"] = place.clamp(min=0)
    s["counts"] = counts


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, t = case["kind"], _TYPES[case["dtype"]]
    s = {"kind": kind, "case": case, "type": t}

    def normal(*shape, scale=1.0, dtype=t):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

    def out(*shape, dtype=t):
        return torch.zeros(*shape, device="cuda", dtype=dtype)

    if kind.startswith("norm"):
        rows, d = s["rows"], s["d"] = case["rows"], case["d"]
        s["group"] = case["group"] or d
        f32 = torch.float32
        s["x"] = normal(rows, d, scale=0.7)
        s["gate"] = normal(rows, 2 * d)[:, d:] if case["gate"] else None  # the second half of a projection
        s["residual"] = normal(rows, d, scale=1.5) if case["residual"] else None
        s["weight_in"], s["weight_out"] = 1.0 + normal(d, scale=0.1, dtype=f32), 1.0 + normal(d, scale=0.1, dtype=f32)
        s["scale"] = 0.5 + normal(d, scale=0.1, dtype=f32) if case["residual"] else None
        s["sum"] = out(rows, d)
        s["y"] = out(rows, d) if case["residual"] else None
        if kind == "norm_train":
            s["dsum"] = normal(rows, d)
            s["dy"] = normal(rows, d) if case["residual"] else None
            s["dx"] = out(rows, d)
            s["dgate"] = out(rows, 2 * d)[:, d:] if case["gate"] else None
            s["dresidual"] = out(rows, d) if case["residual"] else None
            s["dweight_in"], s["dweight_out"] = out(d, dtype=f32), out(d, dtype=f32) if case["residual"] else None
            s["dscale"] = out(d, dtype=f32) if case["residual"] else None
    elif kind.startswith("experts"):
        rows, e, n, k = case["rows"], case["experts"], case["n"], case["k"]
        ends = _shares(case, seed)
        s["rows"], s["longest"] = rows, int((ends[1:] - ends[:-1]).max())
        ends = ends.cuda()
        s["offsets"] = ends.to(torch.int32)
        _pad_index(s, ends, s["longest"], "left")
        s["x"], s["weight"] = normal(rows, k), normal(e, n, k, scale=1.0 / math.sqrt(k))
        s["y"] = out(rows, n)
        if kind == "experts_train":
            s["dy"], s["dx"], s["dweight"] = normal(rows, n), out(rows, k), out(e, n, k)
    else:
        heads, kv, dk, dv = case["heads"], case["kv"], case["dk"], case["dv"]
        step, train = kind == "attn_step", kind == "attn_train"
        if step:
            batch = s["rows"] = case["batch"]
            s["n_slots"] = batch + 3
            slots = torch.randperm(s["n_slots"], generator=g, device="cuda")[:batch].to(torch.int32)
            slots[15::16] = -1
            s["slots"] = slots
        else:
            lengths = s["lengths"] = _lengths(case)
            s["rows"], s["n_slots"] = sum(lengths), len(lengths)
            ends = torch.tensor([0] + lengths, device="cuda").cumsum(0)
            # equal lengths are a dense batch, described by the length alone
            s["offsets"] = None if len(set(lengths)) == 1 else ends.to(torch.int32)
            _pad_index(s, ends, -(-max(lengths) // 64) * 64, "right")
        qkv = normal(s["rows"], heads * dk + kv * (dk + dv))  # three slices of one projection
        s["q"], s["k"], s["v"] = qkv.split([heads * dk, kv * dk, kv * dv], dim=1)
        s["scale"] = dk ** -0.5
        # from a head that keeps everything to one that forgets half in a token
        s["log_decay"] = torch.log1p(-torch.exp2(-torch.linspace(1.0, 9.0, heads, device="cuda", dtype=torch.float64))).float()
        s["log_decay"][-1] = 0.0 if heads > 1 else -0.01
        s["out"] = out(s["rows"], heads * dv)
        if train:
            s["dout"] = normal(s["rows"], heads * dv)
            dqkv = out(s["rows"], heads * dk + kv * (dk + dv))
            s["dq"], s["dk"], s["dv"] = dqkv.split([heads * dk, kv * dk, kv * dv], dim=1)
        else:
            s["state"], s["new_state"] = normal(s["n_slots"], heads, dk, dv, dtype=torch.float32), out(s["n_slots"], heads, dk, dv, dtype=torch.float32)
    if own:
        _describe(s)
    return s


# ------------------------------------------------------------------------------------------------ the library's calls


def _describe(s):
    """The argument blocks and workspaces that a program fills once and passes with every call."""
    import paper_2409_03864_b200 as tdx

    s["tdx"], case, kind = tdx, s["case"], s["kind"]
    dtype = tdx.TDX_BF16 if s["type"] == torch.bfloat16 else tdx.TDX_F32

    def rows_of(*names):
        given = {n: s[n] for n in names if s.get(n) is not None}
        return {**given, **{"ld_" + n: v.stride(0) for n, v in given.items()}}

    if kind.startswith("norm"):
        a = tdx.tdx_norm_args(
            rows=s["rows"], channels=s["d"], group=s["group"], dtype=dtype, norm_in=1, eps=_EPS, weight_in=s["weight_in"], scale=s["scale"],
            weight_out=s["weight_out"] if case["residual"] else None, **rows_of("x", "gate", "residual", "sum", "y"))
        if kind == "norm_train":
            a.set(dweight_in=s["dweight_in"], dweight_out=s["dweight_out"], dscale=s["dscale"], **rows_of("dsum", "dy", "dx", "dgate", "dresidual"))
            _workspace(s, a, tdx.tdx_block_norm_workspace_size(a))
    elif kind.startswith("experts"):
        a = tdx.tdx_grouped_args(rows=s["rows"], experts=case["experts"], N=case["n"], K=case["k"], dtype=dtype, offsets=s["offsets"], weight=s["weight"],
                                 dweight=s.get("dweight"), **rows_of("x", "y", "dy", "dx"))
        _workspace(s, a, tdx.tdx_gemm_grouped_workspace_size(a))
    else:
        step = kind == "attn_step"
        a = tdx.tdx_attention_args(
            batch=case["batch"] if step else len(s["lengths"]), max_len=1 if step else max(s["lengths"]), rows=s["rows"], heads=case["heads"],
            q_heads=case["heads"], k_heads=case["kv"], v_heads=case["kv"], dim_k=case["dk"], dim_v=case["dv"], dtype=dtype, scale=s["scale"],
            log_decay=s["log_decay"], seq_offsets=s.get("offsets"), slots=s.get("slots"), n_slots=s["n_slots"], state_in=s.get("state"),
            state_out=s.get("new_state"), **rows_of("q", "k", "v", "out", "dout", "dq", "dk", "dv"))
        if not step:
            _workspace(s, a, tdx.tdx_decay_attention_workspace_size(a))
    s["args"] = a


def _workspace(s, a, answer):
    status, size = answer
    s["tdx"].check(status)
    s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    a.set(workspace=s["workspace"], workspace_bytes=size)


def _call(s):
    tdx, a, kind = s["tdx"], s["args"], s["kind"]
    stream = torch.cuda.current_stream().cuda_stream
    if kind.startswith("norm"):
        tdx.check(tdx.tdx_block_norm(a, stream))
        if kind == "norm":
            return _there(s, "sum", "y")
        tdx.check(tdx.tdx_block_norm_bwd(a, stream))
        return _there(s, "sum", "y", "dx", "dgate", "dresidual", "dweight_in", "dweight_out", "dscale")
    if kind.startswith("experts"):
        tdx.check(tdx.tdx_gemm_grouped(a, stream))
        if kind == "experts":
            return _there(s, "y")
        tdx.check(tdx.tdx_gemm_grouped_dx(a, stream))
        tdx.check(tdx.tdx_gemm_grouped_dw(a, stream))
        return _there(s, "y", "dx", "dweight")
    if kind == "attn_step":
        tdx.check(tdx.tdx_decay_attention_step(a, stream))
        return _there(s, "out", "new_state")
    tdx.check(tdx.tdx_decay_attention(a, stream))
    if kind == "attn":
        return _there(s, "out", "new_state")
    tdx.check(tdx.tdx_decay_attention_bwd(a, stream))
    return _there(s, "out", "dq", "dk", "dv")


def _there(s, *names):
    return {n: s[n] for n in names if s[n] is not None}


# ------------------------------------------------------------------------------------------------ plain forms


def run(s):
    if own:
        return _call(s)
    kind = s["kind"]
    if kind.startswith("norm"):
        return _norm(s)
    if kind.startswith("experts"):
        return _experts(s)
    if kind == "attn_step":
        return _attn_step(s)
    return _attn(s)


def _rounded(s, **outputs):
    return {n: v.to(s["type"]) for n, v in outputs.items()}


def _norm(s):
    case, groups = s["case"], (s["rows"], s["d"] // s["group"], s["group"])
    x = s["x"].float().view(groups)
    rstd = torch.rsqrt((x * x).mean(2, keepdim=True) + _EPS)
    xhat = (x * rstd).view(s["rows"], s["d"])
    u = xhat * s["weight_in"]
    a = u
    if case["gate"]:
        gate = s["gate"].float()
        sig = 1.0 / (1.0 + torch.exp(-gate))
        a = u * (gate * sig)
    total = a
    if case["residual"]:
        total = s["residual"].float() + s["scale"] * a
        rstd_out = torch.rsqrt((total * total).mean(1, keepdim=True) + _EPS)
        shat = total * rstd_out
        outputs = _rounded(s, sum=total, y=shat * s["weight_out"])
    else:
        outputs = _rounded(s, sum=total)
    if s["kind"] == "norm":
        return outputs
    ds = s["dsum"].float()
    sums = {}
    if case["residual"]:
        dy = s["dy"].float()
        t = dy * s["weight_out"]
        ds = ds + rstd_out * (t - shat * (t * shat).mean(1, keepdim=True))
        sums = {"dweight_out": (dy * shat).sum(0), "dscale": (ds * a).sum(0)}
        outputs |= _rounded(s, dresidual=ds)
    da = ds * s["scale"] if case["residual"] else ds
    du = da
    if case["gate"]:
        outputs |= _rounded(s, dgate=da * u * sig * (1.0 + gate * (1.0 - sig)))
        du = da * (gate * sig)
    sums["dweight_in"] = (du * xhat).sum(0)
    t, xhat = (du * s["weight_in"]).view(groups), xhat.view(groups)
    dx = rstd * (t - xhat * (t * xhat).mean(2, keepdim=True))
    return {**outputs, **_rounded(s, dx=dx.view(s["rows"], s["d"])), **sums}


def _padded(s, v):
    """Rows by [sequence, place], zeros where there is none."""
    return torch.cat([v.float(), v.new_zeros(1, v.shape[1], dtype=torch.float32)])[s["at"]]


def _packed(s, v):
    """The rows of [sequence, place, ...] in their order, zeros for rows of no sequence."""
    flat = v.flatten(0, 1).flatten(1)
    rows = flat.new_zeros(s["rows"] + 1, flat.shape[1])
    rows[s["at"].flatten()] = flat
    return rows[:-1]


def _experts(s):
    w, x = s["weight"].float(), _padded(s, s["x"])
    outputs = _rounded(s, y=_packed(s, x @ w.transpose(1, 2)))
    if s["kind"] == "experts":
        return outputs
    dy = _padded(s, s["dy"])
    return {**outputs, **_rounded(s, dx=_packed(s, dy @ w), dweight=dy.transpose(1, 2) @ x)}


def _heads(s, v, count):
    """rows x (count * dim) -> [sequence, head, place, dim], with the heads that share one beside each other."""
    v = _padded(s, v)
    return v.view(*v.shape[:2], count, -1).transpose(1, 2).repeat_interleave(s["case"]["heads"] // count, dim=1)


def _shared(s, v, count):
    """[sequence, head, place, dim] -> rows x (count * dim), summed over the heads that share one."""
    v = v.unflatten(1, (count, -1)).sum(2)
    return _packed(s, v.transpose(1, 2))


def _powers(s, exponent):
    """exp(log_decay * exponent) for every head, in 64 bits and then rounded; 0 where the exponent is negative."""
    e = exponent.double()
    return torch.where(e >= 0, torch.exp(s["log_decay"].double().view(-1, *[1] * e.dim()) * e), 0.0).float()


def _decay_sum(s, q, k, v):
    """sum over j <= i of decay^(i - j) (q[i] . k[j]) v[j] in chunks of 64 places, and the state after the last place."""
    c = 64
    batch, heads, places, _ = q.shape
    q, k, v = (u.unflatten(2, (places // c, c)) for u in (q, k, v))
    i = torch.arange(c, device="cuda")
    within = ((q @ k.transpose(3, 4)) * _powers(s, i[:, None] - i)[:, None]) @ v
    each = (k * _powers(s, c - 1 - i)[:, None, :, None]).transpose(3, 4) @ v  # what a chunk adds to the state
    n = torch.arange(places // c + 1, device="cuda")
    before = _powers(s, c * (n[:, None] - 1 - n[:-1])) @ each.flatten(3)
    before = before.view(batch, heads, places // c + 1, *each.shape[3:])
    out = within + (q * _powers(s, i + 1)[:, None, :, None]) @ before[:, :, :-1]
    return out.flatten(2, 3), before[:, :, -1]


def _attn(s):
    case = s["case"]
    q, k, v = _heads(s, s["q"], case["heads"]) * s["scale"], _heads(s, s["k"], case["kv"]), _heads(s, s["v"], case["kv"])
    out, state = _decay_sum(s, q, k, v)
    if s["kind"] == "attn":
        far = _powers(s, s["place"] + 1).transpose(0, 1)[:, :, :, None]  # what is left of the state in front of the sequence
        out = out + far * (q @ s["state"])
        state = state + _powers(s, s["counts"]).t()[:, :, None, None] * s["state"]
        return {**_rounded(s, out=_shared(s, out, case["heads"])), "new_state": state}
    dout = _heads(s, s["dout"], case["heads"])
    dq = _decay_sum(s, dout, v, k)[0] * s["scale"]
    # the gradients of keys and values are the same sum from the last row to the first
    q, k, v, dout = (u.flip(2) for u in (q, k, v, dout))
    dk, dv = _decay_sum(s, v, dout, q)[0].flip(2), _decay_sum(s, k, q, dout)[0].flip(2)
    return _rounded(s, out=_shared(s, out, case["heads"]), dq=_shared(s, dq, case["heads"]), dk=_shared(s, dk, case["kv"]), dv=_shared(s, dv, case["kv"]))


def _attn_step(s):
    case, slots = s["case"], s["slots"].long()
    live = slots >= 0
    share = case["heads"] // case["kv"]
    q = s["q"].float().unflatten(1, (case["heads"], -1)) * s["scale"]
    k, v = (s[n].float().unflatten(1, (case["kv"], -1)).repeat_interleave(share, dim=1) for n in ("k", "v"))
    state = torch.exp(s["log_decay"])[:, None, None] * s["state"][slots.clamp(min=0)] + k[:, :, :, None] * v[:, :, None, :]
    out = (q[:, :, :, None] * state).sum(2).flatten(1) * live[:, None]
    new = torch.zeros_like(s["state"])
    new[slots[live]] = state[live]
    return {**_rounded(s, out=out), "new_state": new}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without


def work(case):
    kind, e = case["kind"], 2 if case["dtype"] == "bf16" else 4
    train = kind.endswith("train")
    if kind.startswith("norm"):
        rows, d, gate, residual = case["rows"], case["d"], case["gate"], case["residual"]
        # forward: x, gate and residual in, sum and y out; backward reads those and dsum, dy and writes dx, dgate, dresidual
        reads, writes = 1 + gate + residual, 1 + residual
        total = reads + writes + (reads + 1 + residual + 1 + gate + residual if train else 0)
        return {"bytes": rows * d * e * total + d * 4 * (1 + 2 * residual) * (3 if train else 1), "flops": rows * d * ((12 if gate else 6) + (30 if train else 0))}
    if kind.startswith("experts"):
        rows, n, k = case["rows"] - case["spare"], case["n"], case["k"]
        used = min(case["experts"], rows) * n * k
        bytes_ = (rows * (n + k) + used) * e
        return {"bytes": bytes_ * (3 if train else 1), "flops": 2 * rows * n * k * (3 if train else 1)}
    heads, kv, dk, dv = case["heads"], case["kv"], case["dk"], case["dv"]
    rows = case["batch"] if kind == "attn_step" else sum(_lengths(case))
    states = 0 if train else rows - rows // 16 if kind == "attn_step" else len(_lengths(case))
    into, outof = heads * dk + kv * (dk + dv), heads * dv
    per_row = into + outof + (into + outof + into if train else 0)
    return {"bytes": rows * per_row * e + 8 * states * heads * dk * dv, "flops": rows * heads * dk * dv * (4 + (10 if train else 0))}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    kind = case["kind"]
    if kind.startswith("norm"):
        return _exact_norm(case, s, f)
    if kind.startswith("experts"):
        return _exact_experts(case, s, f)
    return _exact_attn(case, s, f)


def _exact_norm(case, s, f):
    names = ["x", "weight_in"] + (["gate"] if case["gate"] else []) + (["residual", "scale", "weight_out"] if case["residual"] else [])
    leaf = {n: f[n].clone().requires_grad_() for n in names}
    x = leaf["x"].view(s["rows"], -1, s["group"])
    total = (x / torch.sqrt(x.square().mean(2, keepdim=True) + _EPS)).flatten(1) * leaf["weight_in"]
    if case["gate"]:
        total = total * torch.nn.functional.silu(leaf["gate"])
    outputs, loss = {}, 0.0
    if case["residual"]:
        total = leaf["residual"] + leaf["scale"] * total
        outputs["y"] = total / torch.sqrt(total.square().mean(1, keepdim=True) + _EPS) * leaf["weight_out"]
    outputs["sum"] = total
    if s["kind"] == "norm_train":
        loss = (total * f["dsum"]).sum() + ((outputs["y"] * f["dy"]).sum() if case["residual"] else 0.0)
        outputs |= {"d" + n: g for n, g in zip(names, torch.autograd.grad(loss, [leaf[n] for n in names]))}
    return {n: v.detach() for n, v in outputs.items()}


def _exact_experts(case, s, f):
    ends = s["offsets"].tolist()
    train = s["kind"] == "experts_train"
    outputs = {n: torch.zeros_like(f[n]) for n in (("y", "dx", "dweight") if train else ("y",))}
    for e, (lo, hi) in enumerate(zip(ends, ends[1:])):
        w = f["weight"][e]
        outputs["y"][lo:hi] = f["x"][lo:hi] @ w.t()
        if train:
            outputs["dx"][lo:hi] = f["dy"][lo:hi] @ w
            outputs["dweight"][e] = f["dy"][lo:hi].t() @ f["x"][lo:hi]
    return outputs


def _exact_attn(case, s, f):
    heads, kv, dk, dv = case["heads"], case["kv"], case["dk"], case["dv"]
    step, train = case["kind"] == "attn_step", case["kind"] == "attn_train"
    lengths = [1] * case["batch"] if step else _lengths(case)
    count, longest = len(lengths), max(lengths)
    first = [sum(lengths[:i]) for i in range(count)]
    head = torch.arange(heads, device="cuda") // (heads // kv)
    q, k, v = f["q"].view(-1, heads, dk), f["k"].view(-1, kv, dk), f["v"].view(-1, kv, dv)
    decay = torch.exp(f["log_decay"])[:, None, None]
    out = torch.zeros(s["rows"], heads, dv, dtype=torch.float64, device="cuda")
    if train:
        state = torch.zeros(count, heads, dk, dv, dtype=torch.float64, device="cuda")
        dout = f["dout"].view(-1, heads, dv)
        dq, dkk, dvv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    elif step:
        slots = s["slots"].long()
        state = f["state"][slots.clamp(min=0)]
    else:
        state = f["state"].clone()
    # every step takes the sequences that still have a row: the recurrence itself, one row after the other
    rows_at = []
    for t in range(longest):
        on = [i for i in range(count) if t < lengths[i]]
        rows_at.append((torch.tensor(on, device="cuda"), torch.tensor([first[i] + t for i in on], device="cuda")))
    for on, r in rows_at:
        here = decay * state[on] + k[r][:, head, :, None] * v[r][:, head, None, :]
        state[on] = here
        out[r] = s["scale"] * (q[r][:, :, None, :] @ here)[:, :, 0]
        if train:
            dq[r] = s["scale"] * (here @ dout[r][:, :, :, None])[:, :, :, 0]
    if step:
        live = slots >= 0
        new = torch.zeros_like(f["state"])
        new[slots[live]] = state[live]
        return {"out": (out * live[:, None, None]).flatten(1), "new_state": new}
    if not train:
        return {"out": out.flatten(1), "new_state": state}
    grad = torch.zeros_like(state)
    for on, r in reversed(rows_at):
        here = grad[on] + s["scale"] * q[r][:, :, :, None] * dout[r][:, :, None, :]
        into_k = (here @ v[r][:, head, :, None])[:, :, :, 0]
        into_v = (k[r][:, head, None, :] @ here)[:, :, 0]
        dkk[r] = into_k.view(len(r), kv, heads // kv, dk).sum(2)
        dvv[r] = into_v.view(len(r), kv, heads // kv, dv).sum(2)
        grad[on] = decay * here
    return {"out": out.flatten(1), "dq": dq.flatten(1), "dk": dkk.flatten(1), "dv": dvv.flatten(1)}
