"""Pins of the oracle of the operators around the layer, and the refusals that need no device."""
import ctypes as C

import numpy as np
import pytest

from oracle import around_oracle as ao
from paper_2607_23264_b200 import binding, build


def central(f, v, at, h):
    up, down = v.copy(), v.copy()
    up[at] += h
    down[at] -= h
    return (f(up) - f(down)) / (2 * h)


@pytest.mark.parametrize("offset", [0.0, 1.0])
def test_norm_gradients_against_differences(offset):
    rng = np.random.default_rng(0)
    s, gain, d, e = rng.standard_normal((3, 12)), rng.standard_normal(12), rng.standard_normal((3, 12)), rng.standard_normal((3, 12))
    dx, dg, _, _ = ao.rms_norm_backward(s, gain, d, e, 1e-3, offset)
    for at in np.ndindex(s.shape):
        assert abs(central(lambda v: (ao.rms_norm(v, gain, 1e-3, offset) * d).sum() + (v * e).sum(), s, at, 1e-5) - dx[at]) < 1e-7
    for c in range(12):
        assert abs(central(lambda v: (ao.rms_norm(s, v, 1e-3, offset) * d).sum(), gain, c, 1e-5) - dg[c]) < 1e-7


def test_norm_of_simple_rows():
    assert np.array_equal(ao.rms_norm(np.zeros((1, 8)), np.ones(8), 1e-6), np.zeros((1, 8)))
    assert np.allclose(ao.rms_norm(np.full((1, 8), 3.0), np.full(8, 2.0), 1e-12), 2.0)
    assert ao.residual_sum(np.array([[1.0]]), np.array([[2.0 ** -9]]))[0, 0] == 1.0          # a tie goes to the even number


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_balance_gradient_against_differences(score):
    rng = np.random.default_rng(1)
    T, E, k = 11, 6, 2
    x = 2 * rng.standard_normal((T, E))
    x[3, 1] = -np.inf
    ids = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    mask = rng.random(T) < 0.8
    kw = dict(offsets=[0, 4, 4, 10], mask=mask, sequences=3)
    counts, tokens, mean, loss = ao.balance_loss(x, ids, score, 0.7, 0.3, **kw)
    assert tokens[1] == 0 and (mean[1] == 0).all() and tokens[-1] == mask[:10].sum() and counts.sum() == k * tokens[-1]
    dx, _ = ao.balance_loss_backward(x, counts, tokens, k, score, 0.7, 0.3, 2.0, **kw)
    for at in np.ndindex(x.shape):
        if np.isfinite(x[at]):
            num = central(lambda v: 2.0 * ao.balance_loss(v, ids, score, 0.7, 0.3, **kw)[3].sum(), x, at, 1e-5)
            assert abs(num - dx[at]) < 1e-8, at
    assert (dx[10] == 0).all() and dx[3, 1] == 0


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_balance_values(score):
    E, k = 8, 2
    even = np.array([[(2 * t) % E, (2 * t + 1) % E] for t in range(16)])
    assert np.allclose(ao.balance_loss(np.zeros((16, E)), even, score, 0.5, 1.0)[3], [0.5, np.log(8) ** 2])
    one_sided = np.tile([0, 1], (16, 1))
    x = np.zeros((16, E))
    x[:, 2:] = -np.inf
    assert np.allclose(ao.balance_loss(x, one_sided, score, 0.5, 0.0)[3], [0.5 * E / k, 0.0])
    gone = np.full((16, E), -np.inf)
    _, tokens, mean, loss = ao.balance_loss(gone, even, score, 0.5, 1.0)
    assert tokens[-1] == 16 and (mean == 0).all() and (loss == 0).all()
    far, _ = ao.probabilities(np.array([[-200.0, -201.0, -400.0]]), "sigmoid")
    assert np.allclose(far, np.exp([[0, -1, -200]]) / (1 + np.exp(-1.0)))


def test_adapters_against_scalar_loops():
    rng = np.random.default_rng(2)
    x, a, b = rng.standard_normal((5, 16)), rng.standard_normal((3, 8, 16)), rng.standard_normal((3, 24, 8))
    y, scale = rng.standard_normal((5, 24)), np.array([1.0, 0.5, 2.0])
    got, size_t, size_y = ao.add_adapters(x, a, b, scale, [2, -1, 0], y, offsets=[0, 2, 3, 4])
    for r, i in enumerate([2, 2, -1, 0, -1]):
        for n in range(24):
            want = y[r, n]
            for j in range(8):
                want += 0.0 if i < 0 else scale[i] * b[i, n, j] * sum(x[r, c] * a[i, j, c] for c in range(16))
            assert abs(want - got[r, n]) < 1e-12
    assert (size_y <= size_t + 1e-12).all() and (size_t[[2, 4]] == 0).all()


def test_calls_without_a_context_are_refused():
    build.build()
    lib = binding.load_library()
    assert lib.moe_add_rms_norm(None, C.byref(binding.moe_rms_norm_args()), None) == 1
    assert lib.moe_rms_norm_backward(None, C.byref(binding.moe_rms_norm_grad_args()), None) == 1
    assert lib.moe_balance_loss(None, C.byref(binding.moe_balance_args()), None, None, None, None, None, 0, None) == 1
    assert lib.moe_balance_loss_backward(None, C.byref(binding.moe_balance_args()), None, None, None, None, None, None) == 1
    assert lib.moe_add_adapters(None, C.byref(binding.moe_adapter_args()), None) == 1
    assert lib.moe_rms_norm_scratch_bytes(None, 1, 8) == 0 and lib.moe_balance_scratch_bytes(None, 1) == 0
    assert lib.moe_adapter_scratch_bytes(None, 1, 8, 8) == 0


def test_binding_refuses_unknown_names():
    with pytest.raises(ValueError, match="form"):
        binding._lookup(binding.FORMS, "nvfp4", "form")
    with pytest.raises(ValueError, match="gain"):
        binding._gain_fp32(None)
