"""The fp64 oracle of the operators around the expert layer: its gradients against central differences of its own forward pass,
and its 8-bit codes against their definition."""
import numpy as np
import pytest

from oracle import block_oracle as orc


def _difference(f, x, direction, h=1e-6):
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


@pytest.mark.parametrize("T,d", [(1, 2), (3, 7), (5, 32)])
def test_layer_norm_gradients_are_its_differences(T, d):
    rng = np.random.default_rng(T * 100 + d)
    x, w, b, dy = rng.normal(size=(T, d)), rng.normal(size=d) + 1, rng.normal(size=d), rng.normal(size=(T, d))
    eps = 1e-2
    _, mean, rstd = orc.layer_norm(x, w, b, eps)
    dx, dw, db = orc.layer_norm_backward(dy, x, w, mean, rstd)
    for grad, at, f in ((dx, x, lambda v: (orc.layer_norm(v, w, b, eps)[0] * dy).sum()), (dw, w, lambda v: (orc.layer_norm(x, v, b, eps)[0] * dy).sum()),
                        (db, b, lambda v: (orc.layer_norm(x, w, v, eps)[0] * dy).sum())):
        u = rng.normal(size=at.shape)
        assert abs(_difference(f, at, u) - (grad * u).sum()) < 1e-6 * (1 + np.abs(grad * u).sum())


@pytest.mark.parametrize("kind", ["none", "relu", "silu", "gelu"])
def test_linear_gradients_are_its_differences(kind):
    rng = np.random.default_rng(5)
    x, W, b, dy = rng.normal(size=(4, 6)), rng.normal(size=(5, 6)), rng.normal(size=5), rng.normal(size=(4, 5))
    _, z = orc.linear(x, W, b, None, kind)
    dx, dW, db, _ = orc.linear_backward(dy, x, W, z, kind)
    for grad, at, f in ((dx, x, lambda v: (orc.linear(v, W, b, None, kind)[0] * dy).sum()), (dW, W, lambda v: (orc.linear(x, v, b, None, kind)[0] * dy).sum()),
                        (db, b, lambda v: (orc.linear(x, W, v, None, kind)[0] * dy).sum())):
        u = rng.normal(size=at.shape)
        assert abs(_difference(f, at, u) - (grad * u).sum()) < 1e-5 * (1 + np.abs(grad * u).sum())


@pytest.mark.parametrize("norm", ["softmax", "sigmoid"])
@pytest.mark.parametrize("masked", [False, True])
def test_balance_gradient_is_its_difference(norm, masked):
    rng = np.random.default_rng(7)
    T, E, k = 6, 9, 3
    s = rng.normal(size=(T, E))
    idx = np.argsort(-s, 1)[:, :k]
    mask = (np.arange(T) % 3 != 1) if masked else None
    counts, n = orc.expert_counts(idx, E, mask)
    dg = rng.normal(size=(T, k))
    ca, cz = 0.3, 0.2
    live = np.ones(T) if mask is None else mask.astype(float)

    def whole(v):        # the losses, and a loss whose gradient with respect to the gates is dg
        kept = np.take_along_axis(v, idx, 1)
        return orc.balance_loss(v, counts, n, ca, cz, mask)[0] + (orc.gates(kept, norm) * dg * live[:, None]).sum()

    grad = orc.balance_gradient(s, counts, n, ca, cz, mask, idx, dg, norm)
    for seed in range(3):
        u = np.random.default_rng(seed).normal(size=s.shape)
        assert abs(_difference(whole, s, u) - (grad * u).sum()) < 1e-6 * (1 + np.abs(grad * u).sum())


def test_balance_of_even_loads_is_one_and_counts_add_up():
    E, k = 8, 2
    idx = np.stack([np.arange(16) % E, (np.arange(16) + 3) % E], 1)
    counts, n = orc.expert_counts(idx, E)
    assert counts.tolist() == [4] * E and n == 16
    assert abs(orc.balance_loss(np.zeros((16, E)), counts, n, 1.0, 0.0)[1] - 1.0) < 1e-12
    counts, n = orc.expert_counts(idx, E, np.zeros(16))
    assert counts.sum() == 0 and n == 0 and orc.balance_loss(np.zeros((16, E)), counts, n, 1.0, 1.0, np.zeros(16)) == (0.0, 0.0, 0.0)


def test_adamw_first_step_moves_by_the_learning_rate():
    p, m, v = orc.adamw(np.array([1.0, -2.0]), np.array([0.5, -3.0]), np.zeros(2), np.zeros(2), 0.1, 0.9, 0.999, 0.0, 0.0, 1)
    assert np.allclose(p, [0.9, -1.9], atol=1e-12) and np.allclose(m, [0.05, -0.3]) and np.allclose(v, [0.00025, 0.009])


def test_codes_of_eight_bits():
    vals = orc.e4m3_values()
    assert vals[-1] == 448.0 and vals[1] == 2.0 ** -9 and (np.diff(vals) > 0).all()
    rng = np.random.default_rng(3)
    x = rng.normal(size=64) * np.exp(rng.normal(size=64) * 3)
    codes, exps = orc.encode8(x, False)
    back = orc.decode8(codes, exps)
    top = np.abs(x).reshape(2, 32).max(1).repeat(32)
    # half a step of a 3-bit mantissa, or half the smallest step at the low end
    assert (np.abs(back - x) <= np.maximum(np.abs(x) / 16, top / 448 * 2 * 2.0 ** -10) * (1 + 1e-12)).all()
    assert (2.0 ** (exps.astype(float) - 127) * 448 >= np.abs(x).reshape(2, 32).max(1)).all()
    again = orc.encode8(back, False)
    assert (orc.decode8(*again) == back).all()
    tiny = np.zeros(32)
    tiny[0], tiny[1] = 1.0, 1e-12
    assert orc.decode8(*orc.encode8(tiny, True))[1] > 0 and orc.decode8(*orc.encode8(tiny, False))[1] == 0
