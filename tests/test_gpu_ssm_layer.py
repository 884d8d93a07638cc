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
