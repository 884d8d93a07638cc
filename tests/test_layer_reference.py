"""The 64-bit definitions that the block operators' GPU tests go by: gradients against differences, and hand-computed values."""
import numpy as np
import pytest

import layer_reference as ref


def differences(f, arrays, grads, rng, step=1e-6):
    """Directional derivatives of f along random directions, against the gradients' products with them."""
    for name, v in arrays.items():
        d = rng.standard_normal(v.shape)
        up, down = ({**arrays, name: v + s * step * d} for s in (1, -1))
        slope = (f(**up) - f(**down)) / (2 * step)
        assert abs(slope - (grads[name] * d).sum()) <= 1e-6 * (1 + abs(slope)), name


@pytest.mark.parametrize("norm_in", [0, 1])
@pytest.mark.parametrize("gate", [False, True])
def test_block_norm_gradients_are_slopes(norm_in, gate):
    rng = np.random.default_rng(1)
    rows, d, group, eps = 3, 12, 4, 1e-3
    given = {"x": rng.standard_normal((rows, d)), "scale": rng.standard_normal(d), "residual": rng.standard_normal((rows, d)),
             "weight_out": rng.standard_normal(d)}
    if norm_in:
        given["weight_in"] = rng.standard_normal(d)
    if gate:
        given["gate"] = rng.standard_normal((rows, d))
    dsum, dy = rng.standard_normal((rows, d)), rng.standard_normal((rows, d))

    def loss(**g):
        o = ref.block_norm_all(g, group, norm_in, eps)
        return (o["sum"] * dsum + o["y"] * dy).sum()

    o = ref.block_norm_all(given, group, norm_in, eps, dsum, dy)
    differences(loss, given, {k: o["d" + k] for k in given}, rng)
    sizes = ref.block_norm_sizes(given, group, norm_in, eps, dsum, dy)
    for k, v in sizes.items():
        if k in o:
            assert (np.abs(o[k]) <= v * (1 + 1e-9) + 1e-12).all(), k


def test_block_norm_by_hand():
    x = np.array([[3.0, 4.0, 0.0, 2.0]])
    s, y = ref.block_norm_all({"x": x}, 2, 1, 0.0)["sum"], None
    assert np.allclose(s, [[3 / np.sqrt(12.5), 4 / np.sqrt(12.5), 0.0, np.sqrt(2.0)]])
    y = ref.block_norm_all({"x": x, "residual": np.array([[0.0, 0.0, 3.0, 1.0]])}, 4, 0, 0.0)["y"]
    assert np.allclose(y, np.array([[3.0, 4.0, 3.0, 3.0]]) / np.sqrt(43 / 4))


def test_decay_attention_gradients_are_slopes():
    rng = np.random.default_rng(2)
    lengths, heads, dk, dv = [3, 0, 4], 4, 3, 2
    given = {"q": rng.standard_normal((7, 4, dk)), "k": rng.standard_normal((7, 2, dk)), "v": rng.standard_normal((7, 1, dv)),
             "state_in": rng.standard_normal((3, heads, dk, dv))}
    log_decay, dout, dstate = -rng.uniform(0, 1, heads), rng.standard_normal((7, heads, dv)), rng.standard_normal((3, heads, dk, dv))

    def loss(**g):
        o = ref.decay_attention_all(log_decay=log_decay, scale=0.7, lengths=lengths, **g)
        return (o["out"] * dout).sum() + (o["state"] * dstate).sum()

    o = ref.decay_attention_all(log_decay=log_decay, scale=0.7, lengths=lengths, dout=dout, dstate_out=dstate, **given)
    differences(loss, given, {"q": o["dq"], "k": o["dk"], "v": o["dv"], "state_in": o["dstate"]}, rng)


def test_decay_attention_by_hand():
    q, k, v = (np.array(x, dtype=float).reshape(2, 1, 1) for x in ([2, 3], [5, 7], [11, 13]))
    o = ref.decay_attention_all(q, k, v, np.log([0.5]), 10.0, [2], np.full((1, 1, 1, 1), 4.0))
    assert np.allclose(o["out"].ravel(), [10 * 2 * (2 + 55), 10 * 3 * (0.5 * 57 + 91)]) and np.isclose(o["state"].item(), 0.5 * 57 + 91)


def test_grouped_products_by_hand():
    x, w = np.arange(6.0).reshape(3, 2), np.stack([np.eye(2), 2 * np.eye(2)])
    assert np.array_equal(ref.grouped(x, w, [0, 1, 3]), [[0, 1], [4, 6], [8, 10]])
    assert np.array_equal(ref.grouped_dw(x, x, [0, 0, 1])[1], [[0, 0], [0, 1]])
