"""The operators together, as the state-space layer example runs them."""
import numpy as np
import pytest
import torch

import paper_2409_03864_b200 as tdx
import seq_reference as ref
from paper_2409_03864_b200.run_ssm_layer import Layer, main, prompt_and_tokens

pytestmark = pytest.mark.gpu


def test_single_tokens_continue_prompts():
    """Every intermediate is rounded to bf16 (2^-8) in both runs, by kernels that sum in another order, so that now and then a
    value falls to the other side: five rounded intermediates in a row, each less than one unit off."""
    got, want, cache, whole = prompt_and_tokens(Layer(256), [37, 1, 200, 2], 6)
    size = want.float().norm()
    assert torch.isfinite(got.float()).all() and (got.float() - want.float()).norm() < 5 * 2.0 ** -8 * size
    assert (cache[0].float() - whole[0].float()).norm() < 2 * 2.0 ** -8 * whole[0].float().norm()
    assert (cache[1] - whole[1]).norm() < 5 * 2.0 ** -8 * whole[1].norm()
    assert (cache[1][0::2] == 0).all()                       # slots of nobody
    assert tdx.tdx_check_device_status() == 0


def test_gradients_between_the_projections():
    layer, lengths = Layer(64), [21, 1, 40]
    keep, rows = {}, sum(lengths)
    u = torch.randn(rows, 64, device="cuda").to(torch.bfloat16)
    layer.prompts(u, lengths, layer.cache(3), [0, 1, 2], keep)
    dy = torch.randn(rows, layer.D, device="cuda").to(torch.bfloat16)
    g = {k: v.double().cpu().numpy() for k, v in layer.between_gradients(keep, dy).items()}
    b = {k: v.double().cpu().numpy() for k, v in keep["b"].items()}
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    seqs, D, R, N = ref.pieces(3, 40, np.array([0, 21, 22, 62])), layer.D, layer.R, layer.N
    o = ref.scan(b["conv"], b["dt"], f(layer.A), b["proj"][:, R:R + N], b["proj"][:, R + N:], f(layer.skip), b["xz"][:, D:], f(layer.dt_bias), 1, 1, seqs,
                 np.zeros((3, D, N)), dout=f(dy))
    for k in ("dx", "ddt", "dB", "dC", "dz", "dA", "dD", "ddt_bias"):
        assert np.linalg.norm(g[k] - o[k]) < 2.0 ** -8 * np.linalg.norm(o[k]), k        # one rounding to bf16 at most
    c = ref.conv1d(b["xz"][:, :D], f(layer.conv_w), f(layer.conv_b), 1, seqs, np.zeros((3, layer.W - 1, D)), dy=g["dx"])
    for k, name in (("dconv_in", "dx"), ("dconv_w", "dweight"), ("dconv_b", "dbias")):
        assert np.linalg.norm(g[k] - c[name]) < 2.0 ** -8 * np.linalg.norm(c[name]), k


def test_the_command(capsys):
    main(["--width", "128", "--lengths", "9,0,17", "--tokens", "2"])
    assert "gradients" in capsys.readouterr().out


def test_on_another_stream():
    """Inputs that the side stream makes late, and states and buffers that it alone touches: the bits of the default stream."""
    layer, lengths = Layer(128), [30, 1, 7]
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    u, one = (torch.randn(n, layer.E, generator=g, device="cuda").to(torch.bfloat16) for n in (38, 3))

    def both():
        cache, b, slots = layer.cache(3), layer.buffers(3), torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda")
        outs = [layer.prompts(u * 1.0, lengths, cache, [2, 0, 1]).clone()]
        for _ in range(3):
            outs.append(layer.tokens(one * 1.0, cache, slots, b).clone())
        return outs + list(cache)

    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)                        # about 10 ms: what runs elsewhere runs before it
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert tdx.tdx_check_device_status() == 0


def test_single_tokens_in_a_graph():
    """A captured token step, replayed, gives the bits of the calls one by one."""
    layer, slots = Layer(128), torch.tensor([1, -1, 0, 3], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    rows = torch.randn(5, 4, layer.E, generator=g, device="cuda").to(torch.bfloat16)
    u = torch.zeros_like(rows[0])

    def five(step, cache):
        outs = []
        for r in rows:
            u.copy_(r)
            outs.append(step().clone())
        return outs + [c.clone() for c in cache]

    cache, b = layer.cache(4), layer.buffers(4)
    want = five(lambda: layer.tokens(u, cache, slots, b), cache)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = layer.tokens(u, cache, slots, b)
    for c in cache:
        c.zero_()
    got = five(lambda: graph.replay() or out, cache)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert (want[0][1] == 0).all() and tdx.tdx_check_device_status() == 0
