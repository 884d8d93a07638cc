"""The block's operators together: prompts against single tokens, and gradients against those of the same formulas in 64 bits."""
import pytest
import torch

import paper_2409_03864_b200 as tdx
from paper_2409_03864_b200 import run_decay_block as rb

pytestmark = pytest.mark.gpu


def test_tokens_after_prompts_are_longer_prompts():
    block = rb.Block(128, heads=4, dim=32, hidden=96)
    got, want, cache, whole = rb.prompt_and_tokens(block, [70, 1, 33], 5)
    # The same formulas in another order: every step rounds to bf16 (2^-8 each, about ten of them in a row), except for rows whose
    # two best experts are so near that the rounding decides.
    off = (got.float() - want.float()).norm(dim=2) / want.float().norm(dim=2)
    assert (off > 10 * 2 ** -8).sum() <= 1
    assert (cache - whole).norm() <= 10 * 2 ** -8 * whole.norm()
    tdx.check(tdx.tdx_check_device_status())


def plain(block, leaf, lengths, expert):
    """The block in 64 bits with every intermediate as it is, the experts' choice given."""
    def norm(v, w, group=0):
        g = v.reshape(v.shape[0], -1, group or v.shape[1])
        v = (g / torch.sqrt((g * g).mean(2, keepdim=True) + rb.EPS)).reshape(v.shape)
        return v * w

    h = norm(leaf["x"], leaf["norm_1"])
    q, k, v, g = (h @ leaf["w_in"].t()).split(block.split, dim=1)
    share = block.H // block.kv
    q = q.view(-1, block.H, block.D)
    k, v = (u.reshape(-1, block.kv, block.D).repeat_interleave(share, dim=1) for u in (k, v))
    o, row = [], 0
    for n in lengths:
        i = torch.arange(n, device="cuda", dtype=torch.float64)
        w = torch.exp(block.log_decay.double()[:, None, None] * (i[:, None] - i).clamp(min=0)) * (i[:, None] >= i)
        a, b, c = (u[row:row + n].transpose(0, 1) for u in (q, k, v))
        o.append((((a @ b.transpose(1, 2)) * w * block.D ** -0.5) @ c).transpose(0, 1))
        row += n
    o = torch.cat(o).reshape(-1, block.H * block.D)
    a = norm(o, leaf["norm_heads"], block.D) * torch.nn.functional.silu(g)
    s = leaf["x"] + leaf["scale_1"] * norm(a @ leaf["w_out"].t(), leaf["norm_2_in"])
    n = norm(s, leaf["norm_2_out"])
    u = torch.einsum("tk,tnk->tn", n, leaf["w_up"][expert])
    d = torch.einsum("tk,tnk->tn", torch.nn.functional.silu(u), leaf["w_down"][expert])
    return s + leaf["scale_2"] * d


def test_gradients_of_the_whole_block():
    block = rb.Block(128, heads=4, dim=32, hidden=96)
    lengths = [150, 0, 37, 1]
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x, dy = (torch.randn(sum(lengths), block.E, generator=g, device="cuda").to(rb.BF16) for _ in range(2))
    y, keep = block.prompts(x, lengths)
    grads = block.gradients(keep, dy)
    tdx.check(tdx.tdx_check_device_status())
    expert = torch.empty(x.shape[0], dtype=torch.int64, device="cuda")
    ends = keep["offsets"].tolist()
    for e in range(block.experts):
        expert[keep["order"][ends[e]:ends[e + 1]]] = e
    given = {"x": x, "w_in": block.w_in, "w_out": block.w_out, "w_up": block.w_up, "w_down": block.w_down, "norm_1": block.norm_1.weight_out,
             "norm_heads": block.norm_heads.weight_in, "norm_2_in": block.norm_2.weight_in, "scale_1": block.norm_2.scale, "norm_2_out": block.norm_2.weight_out,
             "scale_2": block.add.scale}
    leaf = {k: v.double().requires_grad_() for k, v in given.items()}
    want = plain(block, leaf, lengths, expert)
    exact = dict(zip(leaf, torch.autograd.grad((want * dy.double()).sum(), list(leaf.values()))))
    # about ten roundings to bf16 follow one another on the way to the output and as many on the way back, each at most 2^-8 of a value
    assert (y.double() - want).norm() <= 10 * 2 ** -8 * want.norm()
    assert set(exact) == set(grads)
    for k, v in exact.items():
        assert (grads[k].double() - v).norm() <= 20 * 2 ** -8 * v.norm(), k


def test_the_command_runs(capsys):
    rb.main(["--width", "64", "--lengths", "5,9", "--tokens", "2"])
    assert "gradients:" in capsys.readouterr().out
