"""Plain definitions, in 64 bits on the CPU, of the operators of a block with linear attention and experts, and the sizes of the terms
that their tolerances go by."""
import numpy as np
import torch

F64 = torch.float64


def _t(v, grad=False):
    return None if v is None else torch.as_tensor(np.asarray(v), dtype=F64).clone().requires_grad_(grad)


def block_norm(x, group, norm_in, eps, weight_in=None, gate=None, scale=None, residual=None, weight_out=None):
    """(sum, y) as tensors; inputs may require gradients."""
    u = x
    if norm_in:
        g = x.reshape(x.shape[0], -1, group)
        u = (g / torch.sqrt((g * g).mean(2, keepdim=True) + eps)).reshape(x.shape)
        u = u if weight_in is None else u * weight_in
    a = u if gate is None else u * gate * torch.sigmoid(gate)
    s = a if scale is None else a * scale
    s = s if residual is None else residual + s
    y = s / torch.sqrt((s * s).mean(1, keepdim=True) + eps)
    return s, (y if weight_out is None else y * weight_out)


def block_norm_all(given, group, norm_in, eps, dsum=None, dy=None):
    """Outputs and, with dsum or dy, gradients of every input that is given; as numpy."""
    leaf = {k: _t(v, True) for k, v in given.items()}
    s, y = block_norm(group=group, norm_in=norm_in, eps=eps, **leaf)
    out = {"sum": s.detach().numpy(), "y": y.detach().numpy()}
    if dsum is not None or dy is not None:
        loss = 0.0
        loss = loss + (s * _t(dsum)).sum() if dsum is not None else loss
        loss = loss + (y * _t(dy)).sum() if dy is not None else loss
        names = [k for k in leaf if leaf[k] is not None]
        grads = torch.autograd.grad(loss, [leaf[k] for k in names], allow_unused=True)
        out.update({"d" + k: (np.zeros_like(np.asarray(given[k])) if g is None else g.numpy()) for k, g in zip(names, grads)})
    return out


def block_norm_sizes(given, group, norm_in, eps, dsum=None, dy=None):
    """For every output the sum of the absolute values of the terms that it is made of."""
    n = {k: (None if given.get(k) is None else np.abs(np.asarray(given[k], dtype=np.float64))) for k in
         ("x", "weight_in", "gate", "scale", "residual", "weight_out")}
    rows, d = n["x"].shape
    one = np.ones(d)
    w_in = n["weight_in"] if n["weight_in"] is not None and norm_in else one
    k, w_out = (one if n[v] is None else n[v] for v in ("scale", "weight_out"))
    g = n["x"].reshape(rows, -1, group) if norm_in else None
    r1 = np.repeat(1.0 / np.sqrt((g * g).mean(2) + eps), group, axis=1) if norm_in else np.ones((rows, d))
    xh = n["x"] * r1
    if n["gate"] is not None:
        sig = 1.0 / (1.0 + np.exp(-np.asarray(given["gate"], dtype=np.float64)))
        act, slope = n["gate"] * sig, sig * (1.0 + n["gate"] * (1.0 - sig))
    else:
        act, slope = np.ones((rows, d)), None
    a = xh * w_in * act
    s = k * a + (0.0 if n["residual"] is None else n["residual"])
    exact, _ = block_norm(group=group, norm_in=norm_in, eps=eps, **{v: _t(given.get(v)) for v in n})
    r2 = 1.0 / np.sqrt((exact.numpy() ** 2).mean(1, keepdims=True) + eps)
    # the sum of squares is off by twice the terms' error
    grown = 1.0 + r2 * r2 * (s * s).mean(1, keepdims=True)
    sh = s * r2
    out = {"sum": s, "y": sh * w_out * grown}
    ds = np.zeros((rows, d)) if dsum is None else np.abs(dsum)
    if dy is not None:
        t = np.abs(dy) * w_out
        ds = ds + r2 * (t + sh * (t * sh).mean(1, keepdims=True)) * grown * 2
        out["dweight_out"] = (np.abs(dy) * sh * grown).sum(0)
    out["dresidual"], out["dscale"] = ds, (ds * a).sum(0)
    da = ds * k
    if slope is not None:
        out["dgate"] = da * xh * w_in * slope
    du = da * act
    out["dweight_in"] = (du * xh).sum(0)
    t = du * w_in
    if norm_in:
        m = np.repeat((t * xh).reshape(rows, -1, group).mean(2), group, axis=1)
        out["dx"] = r1 * (t + xh * m)
    else:
        out["dx"] = t
    return out


def grouped(x, weight, offsets):
    y = np.zeros((x.shape[0], weight.shape[1]))
    for e in range(weight.shape[0]):
        y[offsets[e]:offsets[e + 1]] = x[offsets[e]:offsets[e + 1]] @ weight[e].T
    return y


def grouped_dw(dy, x, offsets):
    return np.stack([dy[offsets[e]:offsets[e + 1]].T @ x[offsets[e]:offsets[e + 1]] for e in range(len(offsets) - 1)])


def decay_attention(q, k, v, log_decay, scale, lengths, state_in):
    """q, k, v: rows x own heads x dim (heads a multiple of each); state_in: sequences x heads x dim_k x dim_v.  -> out (rows x heads x dim_v), states."""
    heads = len(log_decay)
    q, k, v = (u.repeat_interleave(heads // u.shape[1], dim=1) for u in (q, k, v))
    decay = torch.exp(log_decay)[:, None, None]
    out, states, row = [], [], 0
    for b, length in enumerate(lengths):
        s = state_in[b]
        for t in range(row, row + length):
            s = decay * s + k[t][:, :, None] * v[t][:, None, :]
            out.append(scale * (q[t][:, None, :] @ s)[:, 0])
        row += length
        states.append(s)
    out = torch.stack(out) if out else q.new_zeros(0, heads, v.shape[2])
    return out, (torch.stack(states) if states else state_in)


def decay_attention_all(q, k, v, log_decay, scale, lengths, state_in, dout=None, dstate_out=None):
    """Outputs and gradients as numpy; the arguments as numpy."""
    leaf = [_t(u, True) for u in (q, k, v, state_in)]
    out, state = decay_attention(leaf[0], leaf[1], leaf[2], _t(log_decay), scale, lengths, leaf[3])
    res = {"out": out.detach().numpy(), "state": state.detach().numpy()}
    if dout is not None:
        loss = (out * _t(dout)).sum()
        if dstate_out is not None:
            loss = loss + (state * _t(dstate_out)).sum()
        if loss.requires_grad:
            grads = torch.autograd.grad(loss, leaf, allow_unused=True)
            res.update({n: (np.zeros_like(np.asarray(u)) if g is None else g.numpy()) for n, g, u in zip(("dq", "dk", "dv", "dstate"), grads, (q, k, v, state_in))})
        else:
            res.update({n: np.zeros_like(np.asarray(u)) for n, u in zip(("dq", "dk", "dv", "dstate"), (q, k, v, state_in))})
    return res
