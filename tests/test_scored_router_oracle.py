"""Pins of the scored-routing oracle: the plain rule against the layer's own top-k, hand-worked groups, ties and masks,
and both gradients against central differences."""
import math

import numpy as np
import pytest

from oracle import moe_oracle as orc
from oracle import scored_router_oracle as sro
from oracle.scored_router_oracle import Rule

INF = math.inf


def test_plain_softmax_rule_is_the_layers_own_routing():
    rng = np.random.default_rng(0)
    logits = rng.standard_normal((50, 24)).astype(np.float32)
    logits[::5, 3] = logits[::5, 7]                      # ties
    ids, w = sro.route(logits, None, Rule(), 4)
    ref_ids, ref_w = orc.topk_route(logits, 4)
    assert np.array_equal(ids, ref_ids) and np.abs(w - ref_w).max() < 1e-12


def test_hand_worked_groups_and_bias():
    # four groups of two; sigmoid scores of 0 are 1/2.  The bias moves the choice, the weights stay those of the scores.
    x = np.array([2.0, -2.0, 0.0, 0.0, 1.0, 1.0, -1.0, 3.0])
    rule = Rule("sigmoid", 4, 2, 2, True, 2.0)
    s = 1 / (1 + np.exp(-x))
    # worth: {0,1}: 0.881+0.119 = 1.0; {2,3}: 1.0; {4,5}: 1.462; {6,7}: 0.269+0.953 = 1.222
    assert sro.select(x, None, rule, 2)[0] == [7, 4]
    bias = np.zeros(8)
    bias[2] = 1.0                                        # {2,3}: 2.0 now, and 2 is the best choice of all
    ids = sro.select(x, bias, rule, 3)[0]
    assert ids == [2, 4, 5]
    w = sro.weights(x, ids, rule)
    assert np.allclose(w, 2.0 * s[ids] / s[ids].sum()) and abs(w.sum() - 2.0) < 1e-12
    # ranked by the best expert alone: {6,7} (3.0) and {0,1} (2.0)
    assert sro.select(x, None, Rule("sigmoid", 4, 2, 1), 2)[0] == [7, 0]


def test_ties_go_to_the_lower_expert_and_group():
    x = np.zeros(8)
    assert sro.select(x, None, Rule("sigmoid", 4, 2, 2), 3)[0] == [0, 1, 2]
    assert sro.select(x, None, Rule("softmax"), 3)[0] == [0, 1, 2]


def test_masked_and_spoiled_tokens():
    x = np.array([-INF, 1.0, -INF, -INF])
    for score in ("softmax", "sigmoid"):
        ids = sro.select(x, None, Rule(score), 3)[0]
        assert ids == [1, 0, 2]
        w = sro.weights(x, ids, Rule(score))
        assert np.allclose(w, [1.0, 0.0, 0.0])
        nothing = np.full(4, -INF)
        assert sro.select(nothing, np.ones(4), Rule(score), 2)[0] == [0, 1]
        assert np.array_equal(sro.weights(nothing, [0, 1], Rule(score)), [0.0, 0.0])
        assert np.isnan(sro.weights(np.array([np.nan, 0.0, 1.0, 2.0]), [3, 2], Rule(score))).all()
        assert sro.select(np.array([np.nan, 0.0, 1.0, 2.0]), None, Rule(score), 4)[0] == [3, 2, 1, 0]
    # one unmasked expert is worth more than a group without any
    x = np.array([-INF, -5.0, -INF, -INF])
    assert sro.select(x, None, Rule("sigmoid", 2, 1, 2), 1)[0] == [1]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_routing_backward_is_the_central_difference_of_the_weights(score, renormalise):
    rng = np.random.default_rng(3)
    rule = Rule(score, 1, 1, 1, renormalise, 2.5)
    x = rng.standard_normal((3, 7))
    ids = np.array([[1, 4, 0], [6, 2, 3], [5, 0, 1]], dtype=np.int32)
    g = rng.standard_normal((3, 3))
    grad = sro.routing_backward(x, ids, g, rule)
    step = 1e-5
    for t in range(3):
        for e in range(7):
            up, dn = x[t].copy(), x[t].copy()
            up[e] += step
            dn[e] -= step
            diff = (sro.weights(up, ids[t], rule) - sro.weights(dn, ids[t], rule)) @ g[t] / (2 * step)
            assert abs(diff - grad[t, e]) < 1e-8


def test_combine_backward_is_the_central_difference_of_the_combine():
    rng = np.random.default_rng(4)
    T, k, H = 3, 2, 4
    y, w = rng.standard_normal((T * k, H)), rng.standard_normal((T, k))
    inv = rng.permutation(T * k)
    d_out = rng.standard_normal((T, H))
    d_y, d_w = sro.combine_backward(d_out, y, inv, w)
    loss = lambda y, w: float((orc.combine(y, inv, w) * d_out).sum())  # noqa: E731
    step = 1e-6
    for r in range(T * k):
        for c in range(H):
            e = np.zeros_like(y)
            e[r, c] = step
            assert abs((loss(y + e, w) - loss(y - e, w)) / (2 * step) - d_y[r, c]) < 1e-7
    for t in range(T):
        for j in range(k):
            e = np.zeros_like(w)
            e[t, j] = step
            assert abs((loss(y, w + e) - loss(y, w - e)) / (2 * step) - d_w[t, j]) < 1e-7
