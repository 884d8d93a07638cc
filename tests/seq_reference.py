"""Plain 64-bit definitions of the sequence operators (numpy, one row after the other), for the tests.

Every function also computes the size of its sums: with magnitude = True all signed inputs are replaced by their absolute
values (the decays exp(dt' A) stay what they are), which bounds what rounding can do to each output."""
import numpy as np


def sigmoid(v):
    return np.where(v >= 0, 1.0 / (1.0 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1.0 + np.exp(-np.abs(v))))


def softplus(v):
    return np.maximum(v, 0.0) + np.log1p(np.exp(-np.abs(v)))


def pieces(batch, max_len, offsets):
    """(first row, length) of every sequence."""
    if offsets is None:
        return [(b * max_len, max_len) for b in range(batch)]
    return [(int(offsets[b]), int(offsets[b + 1] - offsets[b])) for b in range(batch)]


def conv1d(x, weight, bias, silu, seqs, state, dy=None, dstate=None, magnitude=False):
    """state: per sequence (width - 1) x channels.  Returns a dict: y, state, and with dy the gradients."""
    if magnitude:
        x, weight, state = np.abs(x), np.abs(weight), np.abs(state)
        bias = np.abs(bias)
        dy = None if dy is None else np.abs(dy)
        dstate = None if dstate is None else np.abs(dstate)
    width = weight.shape[1]
    w1 = width - 1
    out = {"y": np.zeros_like(x), "state": np.zeros_like(state)}
    if dy is not None:
        out |= {"dx": np.zeros_like(x), "dstate": np.zeros_like(state), "dweight": np.zeros_like(weight), "dbias": np.zeros_like(bias)}
    for i, (first, length) in enumerate(seqs):
        e = np.concatenate([state[i], x[first:first + length]])
        out["state"][i] = e[length:]
        de = np.zeros_like(e)
        for t in range(length):
            pre = bias + (weight.T * e[t:t + width]).sum(0)
            s = sigmoid(pre)
            if magnitude:
                out["y"][first + t] = pre
                grad = np.full_like(pre, 1.1) if silu else np.ones_like(pre)     # |silu'| <= 1.0999
                slope = np.abs(pre) * (0.5 if silu else 0.0)                     # |silu''| <= 0.5: pre's own error
                grad = grad + slope
            else:
                out["y"][first + t] = pre * s if silu else pre
                grad = s * (1 + pre * (1 - s)) if silu else np.ones_like(pre)
            if dy is not None:
                g = dy[first + t] * grad
                de[t:t + width] += weight.T * g
                out["dweight"] += (g * e[t:t + width]).T
                out["dbias"] += g
        if dy is not None:
            if dstate is not None:
                de[length:] += dstate[i]
            out["dstate"][i] = de[:w1]
            out["dx"][first:first + length] = de[w1:]
    return out


def scan(x, dt, A, B, C, D, z, dt_bias, use_softplus, groups, seqs, state, dout=None, dstate=None, magnitude=False):
    """state: per sequence channels x states; z None for no gate.  Returns a dict: out, state, and with dout the gradients."""
    rows, d = x.shape
    n = A.shape[1]
    of = np.arange(d) // (d // groups)
    v = dt + dt_bias
    step = softplus(v) if use_softplus else v
    dstep = sigmoid(v) if use_softplus else np.ones_like(v)
    gate = np.ones_like(x) if z is None else z * sigmoid(z)
    dgate = None if z is None else sigmoid(z) * (1 + z * (1 - sigmoid(z)))
    Aw = A
    if magnitude:
        x, B, C, D, gate, state, Aw = (np.abs(q) for q in (x, B, C, D, gate, state, A))
        dgate = None if z is None else np.abs(dgate)
        dout = None if dout is None else np.abs(dout)
        dstate = None if dstate is None else np.abs(dstate)
    weight = np.abs(step) if magnitude else step
    B, C = B.reshape(rows, groups, n), C.reshape(rows, groups, n)
    out = {"out": np.zeros_like(x), "state": state.copy()}
    if dout is not None:
        out |= {k: np.zeros_like(x) for k in ("dx", "ddt")}
        out |= {"dz": None if z is None else np.zeros_like(x), "dB": np.zeros_like(B), "dC": np.zeros_like(C), "dA": np.zeros_like(A), "dD": np.zeros_like(D),
                "dstate": np.zeros_like(state)}
    for i, (first, length) in enumerate(seqs):
        h, before, decays, ys = state[i].copy(), [], [], []
        for t in range(first, first + length):
            a = np.exp(step[t][:, None] * A)
            before.append(h)
            decays.append(a)
            h = a * h + (weight[t] * x[t])[:, None] * B[t][of]
            ys.append((h * C[t][of]).sum(1) + D * x[t])
            out["out"][t] = ys[-1] * gate[t]
        out["state"][i] = h
        if dout is None:
            continue
        q = np.zeros_like(h) if dstate is None else dstate[i].copy()
        for t in range(first + length - 1, first - 1, -1):
            k = t - first
            g = dout[t] * gate[t]
            now = before[k + 1] if k + 1 < length else h
            if z is not None:
                out["dz"][t] = dout[t] * ys[k] * dgate[t]
            dh = q + g[:, None] * C[t][of]
            np.add.at(out["dC"][t], of, now * g[:, None])
            np.add.at(out["dB"][t], of, dh * (weight[t] * x[t])[:, None])
            through = (dh * B[t][of]).sum(1)
            q = decays[k] * dh
            log = q * before[k]
            out["dx"][t] = through * weight[t] + g * D
            out["ddt"][t] = ((log * Aw).sum(1) + through * x[t]) * dstep[t]
            out["dA"] += log * weight[t][:, None]
            out["dD"] += g * x[t]
        out["dstate"][i] = q
    if dout is not None:
        out["dB"], out["dC"] = out["dB"].reshape(rows, groups * n), out["dC"].reshape(rows, groups * n)
        out["ddt_bias"] = out["ddt"].sum(0)
    return out


def unpack_w4(weight, scales, zeros, k, group):
    """N x K in 64 bits from bytes, scales and zeros (None: 8)."""
    q = np.stack([weight & 15, weight >> 4], axis=2).reshape(weight.shape[0], -1)[:, :k].astype(np.float64)
    at = np.arange(k) // group
    zero = 8.0 if zeros is None else zeros.astype(np.float64)[:, at]
    return (q - zero) * scales[:, at]
