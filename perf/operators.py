"""Cases that measure the operators of a state-space layer: the short causal convolution, the selective scan, and
products with 4-bit weights.

A case is a dict of plain values.  prepare() makes its inputs on the GPU from a seed, run() makes one pass: with
own = False in elementary fp32 torch operations, with own = True through the library's entry points.  exact() gives the
same outputs from the definitions in 64 bits.

  causal convolution   y[t, d] = act(bias[d] + sum_k weight[d, k] * x[t - (W - 1) + k, d]), rows before the sequence
                       from its state
  selective scan       h[t] = exp(dt[t, d] A[d, n]) h[t - 1] + dt[t, d] x[t, d] B[t, n]
                       out[t, d] = (sum_n C[t, n] h[t, d, n] + D[d] x[t, d]) * silu(z[t, d])
  4-bit product        y[m, n] = sum_k x[m, k] * scale[n, k / group] * (q[n, k] - zero[n, k / group])
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # generation of one token for one user: the projections of a layer with 4-bit weights, where latency counts
        {"name": "w4 one token", "kind": "w4", "dtype": "bf16", "m": 1, "n": 4096, "k": 4096, "group": 128, "zeros": False},
        # the same for a wide layer, weights with zero points
        {"name": "w4 one token, wide", "kind": "w4", "dtype": "bf16", "m": 1, "n": 8192, "k": 8192, "group": 128, "zeros": True},
        # generation for a batch of users, small groups
        {"name": "w4 batch of 24", "kind": "w4", "dtype": "bf16", "m": 24, "n": 8192, "k": 2304, "group": 64, "zeros": True},
        # fp32 activations, an odd number of outputs, the smallest groups
        {"name": "w4 fp32 ragged", "kind": "w4", "dtype": "f32", "m": 2, "n": 1000, "k": 4096, "group": 32, "zeros": True},
        # prompts of several users packed one after the other, one of them empty, one a single token
        {"name": "conv prompts", "kind": "conv", "dtype": "bf16", "lengths": "1900,1,0,517,2049,3", "d": 4096, "width": 4},
        # a training step's convolution, forward and backward
        {"name": "conv train", "kind": "conv_train", "dtype": "bf16", "lengths": "2048,2048,2048,2048", "d": 4096, "width": 4},
        # one token for each of 64 users whose states sit in slots of a cache; some batch rows are padding
        {"name": "conv step", "kind": "conv_step", "dtype": "bf16", "batch": 64, "d": 4096, "width": 4},
        # one long prompt
        {"name": "scan prompt", "kind": "scan", "dtype": "bf16", "lengths": "4096", "d": 4096, "n": 16, "groups": 1},
        # packed prompts in fp32, an odd number of channels, two groups of B and C
        {"name": "scan prompts fp32", "kind": "scan", "dtype": "f32", "lengths": "700,1,0,33,1500,257", "d": 1000, "n": 16, "groups": 2},
        # a training step's scan, forward and backward
        {"name": "scan train", "kind": "scan_train", "dtype": "bf16", "lengths": "2048,2048,2048,2048", "d": 2048, "n": 16, "groups": 1},
        # the same in fp32 with odd sizes and fewer states
        {"name": "scan train fp32", "kind": "scan_train", "dtype": "f32", "lengths": "509,509,509", "d": 1000, "n": 8, "groups": 2},
        # one token for each of 128 users
        {"name": "scan step", "kind": "scan_step", "dtype": "bf16", "batch": 128, "d": 4096, "n": 16, "groups": 1},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _off_3072(v, step=1):
    return v + step if v == 3072 else v


def draw(rng):
    kind = rng.choice(["w4", "w4", "conv", "conv_train", "conv_step", "scan", "scan", "scan_train", "scan_train", "scan_step"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "w4":
        group = rng.choice([32, 64, 128])
        return {"kind": kind, "dtype": dtype, "m": _log_int(rng, 1, 64), "n": _off_3072(_log_int(rng, 200, 9000)),
                "k": _off_3072(group * max(1, _log_int(rng, 256, 8192) // group), group), "group": group, "zeros": rng.random() < 0.5}
    d = _off_3072(_log_int(rng, 100, 4500))
    if kind in ("conv_step", "scan_step"):
        batch = _log_int(rng, 1, 256)
        if kind == "conv_step":
            return {"kind": kind, "dtype": dtype, "batch": batch, "d": d, "width": rng.choice([2, 3, 4, 4])}
    else:
        most = 1 << 23 if kind.startswith("scan") else 1 << 25
        total = max(8, min(_log_int(rng, 64, 12000), most // d))
        count = min(_log_int(rng, 1, 12), total)
        if kind.endswith("train") and rng.random() < 0.5:
            lengths = [max(1, total // count)] * count
        else:
            cuts = sorted(rng.randint(0, total) for _ in range(count - 1))
            lengths = [b - a for a, b in zip([0] + cuts, cuts + [total])]
        text = ",".join(str(_off_3072(v)) for v in lengths)
        if kind.startswith("conv"):
            return {"kind": kind, "dtype": dtype, "lengths": text, "d": d, "width": rng.choice([2, 3, 4, 4])}
    groups = rng.choice([1, 1, 2])
    d += d % groups
    n = rng.choice([4, 8, 16, 16, 16])
    case = {"kind": kind, "dtype": dtype, "d": _off_3072(d, groups), "n": n, "groups": groups}
    return {**case, "batch": batch} if kind == "scan_step" else {**case, "lengths": text}


# ------------------------------------------------------------------------------------------------ inputs


def _lengths(case):
    return [int(v) for v in case["lengths"].split(",")]


def _packed(s, case):
    """Row numbers of packed sequences: offsets, and for every row its sequence and its place in it."""
    lengths = _lengths(case)
    s["lengths"], s["rows"] = lengths, sum(lengths)
    # equal lengths are a dense batch, described by the length alone
    dense = len(set(lengths)) == 1
    ends = torch.tensor([0] + lengths, device="cuda").cumsum(0)
    s["offsets"] = None if dense else ends.to(torch.int32)
    s["starts"], s["counts"] = ends[:-1], ends[1:] - ends[:-1]
    s["seq"] = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), s["counts"])
    s["place"] = torch.arange(s["rows"], device="cuda") - s["starts"][s["seq"]]


def _slots(s, case, g):
    """A cache with a few more slots than users; about one batch row in sixteen is padding (slot -1)."""
    batch = case["batch"]
    s["n_slots"] = batch + 3
    slots = torch.randperm(s["n_slots"], generator=g, device="cuda")[:batch].to(torch.int32)
    slots[15::16] = -1
    s["slots"] = slots


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, t = case["kind"], _TYPES[case["dtype"]]
    s = {"kind": kind, "case": case, "type": t}

    def normal(*shape, scale=1.0, dtype=t):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

    def uniform(lo, hi, *shape, dtype=torch.float32):
        return (torch.rand(*shape, generator=g, device="cuda") * (hi - lo) + lo).to(dtype)

    def out(*shape, dtype=t):
        return torch.zeros(*shape, device="cuda", dtype=dtype)

    if kind == "w4":
        m, n, k, group = case["m"], case["n"], case["k"], case["group"]
        s["x"] = normal(m, k)
        s["weight"] = torch.randint(0, 256, (n, k // 2), generator=g, device="cuda", dtype=torch.uint8)
        s["scales"] = uniform(0.5, 1.5, n, k // group, dtype=t) * (0.2 / math.sqrt(k))
        s["zeros"] = torch.randint(4, 12, (n, k // group), generator=g, device="cuda", dtype=torch.uint8) if case["zeros"] else None
        s["y"] = out(m, n)
    elif kind.startswith("conv"):
        d, w = case["d"], case["width"]
        s["weight"], s["bias"] = normal(d, w, scale=0.5, dtype=torch.float32), normal(d, scale=0.1, dtype=torch.float32)
        if kind == "conv_step":
            _slots(s, case, g)
            rows, states = case["batch"], s["n_slots"]
        else:
            _packed(s, case)
            rows, states = s["rows"], len(s["lengths"])
        s["x"] = normal(rows, 2 * d)[:, :d]  # the convolved half of an input projection
        s["y"] = out(rows, d)
        if kind != "conv_train":
            s["state"], s["new_state"] = normal(states, w - 1, d), out(states, w - 1, d)
        else:
            s["dy"] = normal(rows, d)
            s["dx"] = out(rows, 2 * d)[:, :d]
            s["dweight"], s["dbias"] = out(d, w, dtype=torch.float32), out(d, dtype=torch.float32)
    else:
        d, n, groups = case["d"], case["n"], case["groups"]
        if kind == "scan_step":
            _slots(s, case, g)
            rows, states = case["batch"], s["n_slots"]
        else:
            _packed(s, case)
            rows, states = s["rows"], len(s["lengths"])
        s["x"], s["z"] = normal(rows, d), normal(rows, 2 * d)[:, d:]
        s["dt"] = normal(rows, d, scale=0.5)
        bc = normal(rows, 2 * groups * n)
        s["B"], s["C"] = bc[:, : groups * n], bc[:, groups * n:]
        s["A"] = -uniform(0.8, 1.2, d, n) * torch.arange(1, n + 1, device="cuda", dtype=torch.float32)
        s["D"] = uniform(0.5, 1.5, d)
        step = torch.exp(uniform(math.log(1e-3), math.log(1e-1), d))  # step sizes at the start of training
        s["dt_bias"] = step + torch.log(-torch.expm1(-step))
        s["out"] = out(rows, d)
        if kind != "scan_train":
            s["state"], s["new_state"] = normal(states, d, n, dtype=torch.float32), out(states, d, n, dtype=torch.float32)
        else:
            s["dout"] = normal(rows, d)
            s["dx"], s["ddt"], s["dz"] = out(rows, d), out(rows, d), out(rows, 2 * d)[:, d:]
            dbc = out(rows, 2 * groups * n)
            s["dB"], s["dC"] = dbc[:, : groups * n], dbc[:, groups * n:]
            s["dA"], s["dD"], s["ddt_bias"] = out(d, n, dtype=torch.float32), out(d, dtype=torch.float32), out(d, dtype=torch.float32)
    if own:
        _describe(s)
    return s


# ------------------------------------------------------------------------------------------------ the library's calls


def _describe(s):
    """The argument blocks and workspaces that a program fills once and passes with every call."""
    import paper_2409_03864_b200 as tdx

    s["tdx"], case = tdx, s["case"]
    dtype = tdx.TDX_BF16 if s["type"] == torch.bfloat16 else tdx.TDX_F32
    if s["kind"] == "w4":
        s["args"] = tdx.tdx_w4_args(
            M=case["m"], N=case["n"], K=case["k"], group_size=case["group"], dtype=dtype, x=s["x"], ld_x=s["x"].stride(0), weight=s["weight"],
            scales=s["scales"], zeros=s["zeros"], y=s["y"], ld_y=s["y"].stride(0))
        return
    step = s["kind"].endswith("step")
    common = dict(channels=case["d"], dtype=dtype, x=s["x"], ld_x=s["x"].stride(0))
    if step:
        common.update(batch=case["batch"], max_len=1, rows=case["batch"], slots=s["slots"], n_slots=s["n_slots"])
    else:
        common.update(batch=len(s["lengths"]), max_len=max(s["lengths"]), rows=s["rows"], seq_offsets=s["offsets"], n_slots=len(s["lengths"]))
    if "state" in s:
        common.update(state_in=s["state"], state_out=s["new_state"])
    if s["kind"].startswith("conv"):
        a = tdx.tdx_conv1d_args(**common, width=case["width"], silu=1, weight=s["weight"], bias=s["bias"], y=s["y"], ld_y=s["y"].stride(0))
        if s["kind"] == "conv_train":
            a.set(dy=s["dy"], ld_dy=s["dy"].stride(0), dx=s["dx"], ld_dx=s["dx"].stride(0), dweight=s["dweight"], dbias=s["dbias"])
            _workspace(s, a, tdx.tdx_causal_conv1d_workspace_size(a))
    else:
        a = tdx.tdx_scan_args(
            **common, states=case["n"], groups=case["groups"], dt_softplus=1, dt=s["dt"], ld_dt=s["dt"].stride(0), A=s["A"], B=s["B"],
            ld_B=s["B"].stride(0), C=s["C"], ld_C=s["C"].stride(0), D=s["D"], z=s["z"], ld_z=s["z"].stride(0), dt_bias=s["dt_bias"],
            out=s["out"], ld_out=s["out"].stride(0))
        if s["kind"] == "scan_train":
            a.set(dout=s["dout"], ld_dout=s["dout"].stride(0), dA=s["dA"], dD=s["dD"], ddt_bias=s["ddt_bias"],
                  **{k: s[k] for k in ("dx", "ddt", "dB", "dC", "dz")}, **{"ld_" + k: s[k].stride(0) for k in ("dx", "ddt", "dB", "dC", "dz")})
            status, size = tdx.tdx_selective_scan_saved_size(a)
            tdx.check(status)
            s["saved"] = torch.empty(size, dtype=torch.uint8, device="cuda")
            a.set(saved=s["saved"], saved_bytes=size)
        if not step:
            _workspace(s, a, tdx.tdx_selective_scan_workspace_size(a))
    s["args"] = a


def _workspace(s, a, answer):
    status, size = answer
    s["tdx"].check(status)
    s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    a.set(workspace=s["workspace"], workspace_bytes=size)


def _call(s):
    tdx, a, kind = s["tdx"], s["args"], s["kind"]
    stream = torch.cuda.current_stream().cuda_stream
    if kind == "w4":
        tdx.check(tdx.tdx_gemm_w4(a, stream))
        return s["y"]
    if kind == "conv":
        tdx.check(tdx.tdx_causal_conv1d(a, stream))
        return s["y"], s["new_state"]
    if kind == "conv_step":
        tdx.check(tdx.tdx_causal_conv1d_step(a, stream))
        return s["y"], s["new_state"]
    if kind == "conv_train":
        tdx.check(tdx.tdx_causal_conv1d(a, stream))
        tdx.check(tdx.tdx_causal_conv1d_bwd(a, stream))
        return {k: s[k] for k in ("y", "dx", "dweight", "dbias")}
    if kind == "scan":
        tdx.check(tdx.tdx_selective_scan(a, stream))
        return s["out"], s["new_state"]
    if kind == "scan_step":
        tdx.check(tdx.tdx_selective_scan_step(a, stream))
        return s["out"], s["new_state"]
    tdx.check(tdx.tdx_selective_scan(a, stream))
    tdx.check(tdx.tdx_selective_scan_bwd(a, stream))
    return {k: s[k] for k in ("out", "dx", "ddt", "dB", "dC", "dz", "dA", "dD", "ddt_bias")}


# ------------------------------------------------------------------------------------------------ plain forms


def run(s):
    if own:
        return _call(s)
    kind = s["kind"]
    if kind == "w4":
        return _w4(s)
    if kind == "conv_step":
        return _conv_step(s)
    if kind.startswith("conv"):
        return _conv(s)
    if kind == "scan_step":
        return _scan_step(s)
    return _scan(s)


def _w4(s):
    case = s["case"]
    n, k, group = case["n"], case["k"], case["group"]
    q = torch.stack([s["weight"] & 15, s["weight"] >> 4], dim=2).view(n, k // group, group).float()  # the low half is the even k
    zero = s["zeros"].float()[:, :, None] if s["zeros"] is not None else 8.0
    w = ((q - zero) * s["scales"].float()[:, :, None]).view(n, k)
    return (s["x"].float() @ w.t()).to(s["type"])


def _sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _gather_rows(s, width):
    """For every row its `width` convolved rows in a list of all states' rows and then all inputs."""
    back = torch.arange(width, device="cuda") - (width - 1)
    place = s["place"][:, None] + back
    states = len(s["lengths"]) * (width - 1)
    return torch.where(place >= 0, states + torch.arange(s["rows"], device="cuda")[:, None] + back, s["seq"][:, None] * (width - 1) + (width - 1) + place)


def _conv(s):
    case, t = s["case"], s["type"]
    w, d, count = case["width"], case["d"], len(s["lengths"])
    state = s["state"].float().view(-1, d) if "state" in s else torch.zeros(count * (w - 1), d, device="cuda")
    rows = torch.cat([state, s["x"].float()])
    at = _gather_rows(s, w)
    pre = s["bias"] + (rows[at] * s["weight"].t()).sum(1)
    sig = _sigmoid(pre)
    y = pre * sig
    if s["kind"] == "conv":
        # the state after a sequence: its last width - 1 rows, older ones from the state before it
        place = s["counts"][:, None] + torch.arange(w - 1, device="cuda") - (w - 1)
        old = torch.arange(count, device="cuda")[:, None] * (w - 1) + (w - 1) + place
        new = torch.where(place >= 0, count * (w - 1) + s["starts"][:, None] + place, old)
        return y.to(t), rows[new].to(t)
    dpre = s["dy"].float() * sig * (1.0 + pre * (1.0 - sig))
    dweight = (dpre[:, None, :] * rows[at]).sum(0).t().contiguous()
    # a row of x is used by the rows up to width - 1 after it in its sequence
    ahead = (w - 1) - torch.arange(w, device="cuda")
    later = s["place"][:, None] + ahead < s["counts"][s["seq"]][:, None]
    at = torch.where(later, torch.arange(s["rows"], device="cuda")[:, None] + ahead, 0)
    dx = (dpre[at] * later[:, :, None] * s["weight"].t()).sum(1)
    return {"y": y.to(t), "dx": dx.to(t), "dweight": dweight, "dbias": dpre.sum(0)}


def _conv_step(s):
    t, slots = s["type"], s["slots"].long()
    live = slots >= 0
    at = slots.clamp(min=0)
    rows = torch.cat([s["state"][at].float(), s["x"].float()[:, None]], dim=1)
    pre = s["bias"] + (rows * s["weight"].t()).sum(1)
    y = pre * _sigmoid(pre) * live[:, None]
    new = torch.zeros_like(s["state"])
    new[slots[live]] = rows[live][:, 1:].to(t)
    return y.to(t), new


def _softplus(v):
    return torch.where(v > 20.0, v, torch.log1p(torch.exp(v)))


def _per_channel(s, v):
    """rows x (groups * n) to rows x channels x n"""
    case = s["case"]
    return v.float().view(-1, case["groups"], case["n"]).repeat_interleave(case["d"] // case["groups"], dim=1)


def _per_group(s, v):
    """rows x channels x n to rows x (groups * n), summed over each group's channels"""
    case = s["case"]
    return v.view(-1, case["groups"], case["d"] // case["groups"], case["n"]).sum(2).view(-1, case["groups"] * case["n"])


def _recur(a, u, longest):
    """h[t] = a[t] h[t - 1] + u[t] for all t, by doubling: after each step a term covers twice as many rows.  a is 0 where a sequence starts."""
    reach = 1
    while reach < longest:
        u = torch.cat([u[:reach], u[reach:] + a[reach:] * u[:-reach]])
        a = torch.cat([a[:reach], a[reach:] * a[:-reach]])
        reach *= 2
    return u


def _scan(s):
    case, t = s["case"], s["type"]
    x, z, C = s["x"].float(), s["z"].float(), _per_channel(s, s["C"])
    pre = s["dt"].float() + s["dt_bias"]
    dt, B = _softplus(pre), _per_channel(s, s["B"])
    decay = torch.exp(dt[:, :, None] * s["A"])
    u = (dt * x)[:, :, None] * B
    first = (s["place"] == 0)[:, None, None]
    if "state" in s:
        u = u + torch.where(first, decay * s["state"][s["seq"]], 0.0)
    longest = max(s["lengths"])
    h = _recur(torch.where(first, 0.0, decay), u, longest)
    y = (h * C).sum(2) + s["D"] * x
    sig = _sigmoid(z)
    out = (y * z * sig).to(t)
    if s["kind"] == "scan":
        last = s["starts"] + s["counts"] - 1
        new = torch.where((s["counts"] > 0)[:, None, None], h[last.clamp(min=0)], s["state"])
        return out, new
    dout = s["dout"].float()
    dz = dout * y * sig * (1.0 + z * (1.0 - sig))
    dy = dout * z * sig
    # dh[t] = C[t] dy[t] + decay[t + 1] dh[t + 1]: the same recurrence from the last row to the first
    ends = s["place"] + 1 == s["counts"][s["seq"]]
    after = torch.where(ends[:, None, None], 0.0, torch.cat([decay[1:], decay[:1]]))
    dh = _recur(after.flip(0), (dy[:, :, None] * C).flip(0), longest).flip(0)
    before = torch.where(first, 0.0, torch.cat([h[:1], h[:-1]]))
    dlog = dh * before * decay
    through_u = (dh * B).sum(2)
    ddt = (dlog * s["A"]).sum(2) + through_u * x
    dpre = ddt * _sigmoid(pre)
    return {
        "out": out, "dx": (through_u * dt + dy * s["D"]).to(t), "ddt": dpre.to(t), "dB": _per_group(s, dh * (dt * x)[:, :, None]).to(t),
        "dC": _per_group(s, h * dy[:, :, None]).to(t), "dz": dz.to(t), "dA": (dlog * dt[:, :, None]).sum(0), "dD": (dy * x).sum(0), "ddt_bias": dpre.sum(0),
    }


def _scan_step(s):
    slots, x, z = s["slots"].long(), s["x"].float(), s["z"].float()
    live = slots >= 0
    dt = _softplus(s["dt"].float() + s["dt_bias"])
    h = torch.exp(dt[:, :, None] * s["A"]) * s["state"][slots.clamp(min=0)] + (dt * x)[:, :, None] * _per_channel(s, s["B"])
    y = (h * _per_channel(s, s["C"])).sum(2) + s["D"] * x
    new = torch.zeros_like(s["state"])
    new[slots[live]] = h[live]
    return (y * z * _sigmoid(z) * live[:, None]).to(s["type"]), new


# ------------------------------------------------------------------------------------------------ what a pass cannot do without


def work(case):
    kind, e = case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind == "w4":
        m, n, k = case["m"], case["n"], case["k"]
        per_group = e + (1 if case["zeros"] else 0)
        return {"bytes": n * k // 2 + n * (k // case["group"]) * per_group + (m * k + m * n) * e, "flops": 2 * m * n * k}
    d = case["d"]
    step, train = kind.endswith("step"), kind.endswith("train")
    rows = case["batch"] if step else sum(_lengths(case))
    states = 0 if train else case["batch"] if step else len(_lengths(case))
    if kind.startswith("conv"):
        w = case["width"]
        bytes_ = rows * d * e * (4 if train else 2) + 2 * states * (w - 1) * d * e + d * (w + 1) * 4 * (2 if train else 1)
        return {"bytes": bytes_, "flops": rows * d * ((2 * w + 5) + (4 * w + 8 if train else 0))}
    n, bc = case["n"], 2 * case["groups"] * case["n"]
    # forward: x, dt, z, B, C in and out out; backward reads those and dout again and writes five gradients
    per_row = (4 * d + bc) * e + ((3 * d + bc + d + 3 * d + bc) * e if train else 0)
    bytes_ = rows * per_row + d * (n + 2) * 4 * (2 if train else 1) + 2 * states * d * n * 4
    return {"bytes": bytes_, "flops": rows * d * n * (7 + (19 if train else 0)) + rows * d * (12 if train else 8)}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if kind == "w4":
        return _exact_w4(case, s, f)
    if kind.startswith("conv"):
        return _exact_conv(case, s, f)
    return _exact_scan(case, s, f)


def _exact_w4(case, s, f):
    n, k = case["n"], case["k"]
    byte = s["weight"].to(torch.int64)
    w = torch.empty(n, k, dtype=torch.float64, device="cuda")
    w[:, 0::2], w[:, 1::2] = (byte % 16).double(), (byte // 16).double()
    group = torch.arange(k, device="cuda") // case["group"]
    w -= s["zeros"].double()[:, group] if s["zeros"] is not None else 8
    w *= f["scales"][:, group]
    return torch.einsum("mk,nk->mn", f["x"], w)


def _exact_conv(case, s, f):
    d, w, kind = case["d"], case["width"], case["kind"]
    step, train = kind == "conv_step", kind == "conv_train"
    y = torch.zeros(f["x"].shape[0], d, dtype=torch.float64, device="cuda")
    dx, dweight, dbias = torch.zeros_like(y), torch.zeros(d, w, dtype=torch.float64, device="cuda"), torch.zeros(d, dtype=torch.float64, device="cuda")
    new = torch.zeros_like(f["state"]) if not train else None
    pieces = [(b, b + 1, int(v)) for b, v in enumerate(s["slots"].tolist())] if step else []
    first = 0
    for i, length in enumerate([] if step else _lengths(case)):
        pieces.append((first, first + length, i))
        first += length
    for lo, hi, slot in pieces:
        if slot < 0:
            continue
        before = torch.zeros(w - 1, d, dtype=torch.float64, device="cuda") if train else f["state"][slot]
        line = torch.cat([before, f["x"][lo:hi]])
        length = hi - lo
        if not train:
            new[slot] = line[length:]
        pre = f["bias"].expand(length, d).clone()
        for k in range(w):
            pre += f["weight"][:, k] * line[k:k + length]
        sig = torch.sigmoid(pre)
        y[lo:hi] = pre * sig
        if train:
            g = f["dy"][lo:hi] * (sig + pre * sig * (1 - sig))
            dline = torch.zeros_like(line)
            for k in range(w):
                dline[k:k + length] += f["weight"][:, k] * g
                dweight[:, k] += (g * line[k:k + length]).sum(0)
            dbias += g.sum(0)
            dx[lo:hi] = dline[w - 1:]
    return {"y": y, "dx": dx, "dweight": dweight, "dbias": dbias} if train else (y, new)


def _exact_scan(case, s, f):
    d, n, groups, kind = case["d"], case["n"], case["groups"], case["kind"]
    step, train = kind == "scan_step", kind == "scan_train"
    lengths = [1] * case["batch"] if step else _lengths(case)
    count, longest = len(lengths), max(lengths)
    # every sequence in a row of its own, so that one step of the recurrence takes all of them
    rows = torch.zeros(count, longest, dtype=torch.int64, device="cuda")
    there = torch.zeros(count, longest, dtype=torch.bool, device="cuda")
    first = 0
    for i, length in enumerate(lengths):
        rows[i, :length] = torch.arange(first, first + length, device="cuda")
        there[i, :length] = True
        first += length
    x, z = f["x"], f["z"]
    pre = f["dt"] + f["dt_bias"]
    dt = torch.nn.functional.softplus(pre, threshold=40.0)
    group = torch.arange(d, device="cuda") // (d // groups)
    B, C = f["B"].view(-1, groups, n), f["C"].view(-1, groups, n)
    if step:
        slots = s["slots"].long()
        h = f["state"][slots.clamp(min=0)] * (slots >= 0)[:, None, None]
    else:
        h = torch.zeros(count, d, n, dtype=torch.float64, device="cuda") if train else f["state"].clone()
    y = torch.zeros_like(x)
    kept = torch.zeros(longest, count, d, n, dtype=torch.float64, device="cuda") if train else None
    for t in range(longest):
        r, on = rows[:, t], there[:, t]
        if train:
            kept[t] = h
        moved = torch.exp(dt[r][:, :, None] * f["A"]) * h + (dt[r] * x[r])[:, :, None] * B[r][:, group]
        h = torch.where(on[:, None, None], moved, h)
        y[r[on]] = ((h * C[r][:, group]).sum(2) + f["D"] * x[r])[on]
    out = y * z * torch.sigmoid(z)
    if step:
        new = torch.zeros_like(f["state"])
        new[slots[slots >= 0]] = h[slots >= 0]
        return out * (slots >= 0)[:, None], new
    if not train:
        return out, h
    sig = torch.sigmoid(z)
    dz = f["dout"] * y * (sig + z * sig * (1 - sig))
    dy = f["dout"] * z * sig
    dx, ddt = torch.zeros_like(x), torch.zeros_like(x)
    dB, dC = torch.zeros(x.shape[0], groups, n, dtype=torch.float64, device="cuda"), torch.zeros(x.shape[0], groups, n, dtype=torch.float64, device="cuda")
    dA = torch.zeros_like(f["A"])
    dh = torch.zeros(count, d, n, dtype=torch.float64, device="cuda")
    for t in reversed(range(longest)):
        r, on = rows[:, t], there[:, t]
        live = on[:, None, None].double()
        decay = torch.exp(dt[r][:, :, None] * f["A"])
        now = decay * kept[t] + (dt[r] * x[r])[:, :, None] * B[r][:, group]
        dh = (dh + dy[r][:, :, None] * C[r][:, group]) * live  # a sequence that ends before row t has no gradient yet
        inner = (dh * B[r][:, group]).sum(2)
        log = dh * decay * kept[t]
        dx[r[on]] = (inner * dt[r] + dy[r] * f["D"])[on]
        ddt[r[on]] = (inner * x[r] + (log * f["A"]).sum(2))[on]
        dA += (log * dt[r][:, :, None]).sum(0)
        dB[r[on]] = (dh * (dt[r] * x[r])[:, :, None]).view(count, groups, d // groups, n).sum(2)[on]
        dC[r[on]] = (now * dy[r][:, :, None]).view(count, groups, d // groups, n).sum(2)[on]
        dh = dh * decay
    dpre = ddt * torch.sigmoid(pre)
    return {"out": out, "dx": dx, "ddt": dpre, "dB": dB.flatten(1), "dC": dC.flatten(1), "dz": dz, "dA": dA, "dD": (dy * x).sum(0), "ddt_bias": dpre.sum(0)}
