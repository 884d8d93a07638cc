"""The 64-bit definitions that the GPU tests compare with: their gradients against central differences, and the scan and
the convolution against closed forms."""
import numpy as np
import pytest

import seq_reference as ref


def directional(f, inputs, grads, rng, rel=1e-6):
    """sum over inputs of grad . direction == the central difference of f along the directions"""
    dirs = {k: rng.standard_normal(v.shape) for k, v in inputs.items()}
    h = 1e-5
    up = f(**{k: v + h * dirs[k] for k, v in inputs.items()})
    down = f(**{k: v - h * dirs[k] for k, v in inputs.items()})
    want = (up - down) / (2 * h)
    got = sum((grads[k] * dirs[k]).sum() for k in inputs)
    assert abs(got - want) <= rel * max(1.0, abs(want)), (got, want)


@pytest.mark.parametrize("silu", [0, 1])
@pytest.mark.parametrize("width", [1, 2, 4])
def test_conv1d_gradients_against_differences(width, silu):
    rng = np.random.default_rng(width)
    seqs, d = [(0, 5), (5, 0), (5, 1), (6, 2)], 3
    inputs = {"x": rng.standard_normal((8, d)), "weight": rng.standard_normal((d, width)), "bias": rng.standard_normal(d),
              "state": rng.standard_normal((4, width - 1, d))}
    dy, dstate = rng.standard_normal((8, d)), rng.standard_normal((4, width - 1, d))

    def loss(x, weight, bias, state):
        o = ref.conv1d(x, weight, bias, silu, seqs, state)
        return (o["y"] * dy).sum() + (o["state"] * dstate).sum()

    o = ref.conv1d(**{k: inputs[k] for k in ("x", "weight", "bias")}, silu=silu, seqs=seqs, state=inputs["state"], dy=dy, dstate=dstate)
    directional(loss, inputs, {"x": o["dx"], "weight": o["dweight"], "bias": o["dbias"], "state": o["dstate"]}, rng)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("softplus", [0, 1])
@pytest.mark.parametrize("groups", [1, 2])
def test_scan_gradients_against_differences(groups, softplus, gated):
    rng = np.random.default_rng(7)
    seqs, rows, d, n = [(0, 6), (6, 0), (6, 1)], 7, 4, 3
    inputs = {"x": rng.standard_normal((rows, d)), "dt": rng.uniform(0.1, 0.9, (rows, d)), "A": -rng.uniform(0.2, 2.0, (d, n)),
              "B": rng.standard_normal((rows, groups * n)), "C": rng.standard_normal((rows, groups * n)), "D": rng.standard_normal(d),
              "dt_bias": rng.uniform(0.0, 0.3, d), "state": rng.standard_normal((3, d, n))}
    if gated:
        inputs["z"] = rng.standard_normal((rows, d))
    dout, dstate = rng.standard_normal((rows, d)), rng.standard_normal((3, d, n))

    def call(z=None, state=None, **v):
        return ref.scan(**v, z=z, use_softplus=softplus, groups=groups, seqs=seqs, state=state, **extra)

    extra = {}

    def loss(**v):
        o = call(**v)
        return (o["out"] * dout).sum() + (o["state"] * dstate).sum()

    extra = {"dout": dout, "dstate": dstate}
    o = call(**inputs)
    extra = {}
    directional(loss, inputs, {k: o["dstate" if k == "state" else "d" + k] for k in inputs}, rng)


def test_scan_of_constant_inputs_is_a_geometric_sum():
    d, n, length, a, u = 2, 3, 9, -0.5, 0.25
    x, dt, B = np.ones((length, d)), np.full((length, d), u), np.ones((length, n))
    o = ref.scan(x, dt, np.full((d, n), a), B, np.ones((length, n)), np.zeros(d), None, np.zeros(d), 0, 1, [(0, length)], np.zeros((1, d, n)))
    w = np.exp(u * a)
    t = np.arange(length)
    assert np.allclose(o["out"], (n * u * (1 - w ** (t + 1)) / (1 - w))[:, None], rtol=1e-13)


def test_conv1d_with_a_unit_tap_shifts_the_rows():
    rng = np.random.default_rng(0)
    x, state = rng.standard_normal((6, 2)), rng.standard_normal((1, 3, 2))
    weight = np.zeros((2, 4))
    weight[:, 1] = 1.0                           # e[t + 1]: the row two before t
    o = ref.conv1d(x, weight, np.zeros(2), 0, [(0, 6)], state)
    assert np.array_equal(o["y"], np.concatenate([state[0, 1:], x[:4]]))
    assert np.array_equal(o["state"][0], x[3:])


def test_w4_bytes_hold_the_even_k_in_the_low_half():
    w = ref.unpack_w4(np.array([[0x21, 0x0F]], dtype=np.uint8), np.array([[1.0, 10.0]]), None, 3, 2)
    assert np.array_equal(w, [[1 - 8, 2 - 8, 70.0]])
