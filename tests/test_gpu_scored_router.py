"""Scored routing and the gradients of the gate on the GPU against the fp64 oracle.

Ids.  Where logits and bias lie on a coarse grid, choice values are either equal on both sides or far apart, and ids
must match bit for bit.  For continuous logits an fp32 choice may order two experts differently whose exact choices are
closer than its rounding error: a differing slot must hold an expert whose exact choice is within 4e-6 of the oracle's.

Weights.  expf is within 2 ulp, its argument is rounded once (2^-24 |x - max| relative in the result), a sum of E <= 1024
terms in 32 lanes carries at most 37 roundings, divisions and the scale one each: below 1e-5 of the weight for |x| <= 30.
Gradients repeat these factors and one difference of two sums of k <= 32 terms: 1e-5 of (weight scale) x (largest |g|) x
(1 + k).  Dot products of H terms: 2^-24 x (H/32 + 8) of the sum of magnitudes."""
import math

import numpy as np
import pytest
import torch

from oracle import moe_oracle as orc
from oracle import scored_router_oracle as sro
from oracle.scored_router_oracle import Rule
from paper_2607_23264_b200 import binding, inputs as gen
from moe_testlib import DEV, bits_to_dev, dev_bf16_to_f64

pytestmark = pytest.mark.gpu


def gpu_rule(r: Rule):
    return binding.make_route_rule(r.score, r.n_group, r.topk_group, r.group_top, r.renormalise, r.weight_scale)


def run_route(logits, bias, rule, k, stream=None):
    T, E = logits.shape
    ctx = binding.Context(T, 64, 64, E, k)
    i32 = dict(dtype=torch.int32, device=DEV)
    o = dict(topk_ids=torch.full((T, k), -1, **i32), topk_w=torch.full((T, k), 7e30, device=DEV),
             counts=torch.full((E,), -1, **i32), offsets=torch.full((E + 1,), -1, **i32),
             perm=torch.full((T * k,), -1, **i32), inv_perm=torch.full((T * k,), -1, **i32))
    d_logits = torch.from_numpy(logits).to(DEV)
    d_bias = None if bias is None else torch.from_numpy(bias).to(DEV)
    torch.cuda.synchronize()
    ctx.moe_plan_routing_scored(d_logits, d_bias, gpu_rule(rule), **o, stream=stream)
    torch.cuda.synchronize()
    assert ctx.moe_last_device_status()[0] == 0
    return {n: t.cpu().numpy() for n, t in o.items()}


def check_plan(o, E):
    counts, offsets, perm, inv_perm = orc.plan_permutation(o["topk_ids"], E)
    for name, ref in (("counts", counts), ("offsets", offsets), ("perm", perm), ("inv_perm", inv_perm)):
        assert np.array_equal(o[name], ref), name


def check_weights(got, ids, logits, rule):
    for t in range(len(ids)):
        ref = sro.weights(logits[t], ids[t], rule)
        assert np.array_equal(np.isnan(got[t]), np.isnan(ref)), t
        if not np.isnan(ref).any():
            assert (np.abs(got[t] - ref) <= 1e-5 * np.abs(ref) + 1e-37).all(), (t, got[t], ref)


SHAPES = [  # T, E, k, n_group, topk_group
    (1, 1, 1, 1, 1), (1, 256, 8, 8, 4), (3, 7, 3, 1, 1), (70, 32, 4, 4, 2), (33, 33, 5, 3, 2), (65, 64, 6, 1, 1),
    (129, 96, 6, 6, 3), (40, 160, 6, 8, 3), (257, 256, 8, 8, 4), (50, 300, 32, 10, 3), (20, 512, 9, 32, 5),
    (37, 1000, 32, 25, 7), (600, 8, 2, 2, 1), (300, 24, 12, 24, 12), (2000, 48, 3, 1, 1),
    (130, 128, 7, 2, 1), (60, 1024, 12, 8, 5), (300, 256, 10, 16, 3), (9, 128, 4, 32, 32), (77, 512, 20, 4, 4),
]


@pytest.mark.parametrize("T,E,k,n_group,topk_group", SHAPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
def test_ids_on_a_grid_are_exact(T, E, k, n_group, topk_group, score, with_bias):
    rng = np.random.default_rng(T * 1000 + E)
    group_top = 2 if (T + E) % 2 and E // n_group >= 2 else 1
    rule = Rule(score, n_group, topk_group, group_top, bool(T % 2), 2.5)
    logits = (rng.integers(-24, 25, (T, E)) / 4).astype(np.float32)      # many exact ties
    if T > 2:
        logits[T // 2] = 0.0                                             # nothing but ties
    bias = (rng.integers(-3, 4, E) / (2 if score == "softmax" else 32)).astype(np.float32) if with_bias else None
    o = run_route(logits, bias, rule, k)
    ids, _ = sro.route(logits, bias, rule, k)
    same = (o["topk_ids"] == ids).all(1)
    for t in np.flatnonzero(~same):      # an equal-in-fp32 pair of different sums is the only other admissible order
        c = sro.choice_values(logits[t], bias, rule)
        if group_top == 2 and n_group > 1:
            size = E // n_group
            rank = c if bias is not None else sro.scores(logits[t], rule)
            worth = lambda e: np.sort(rank[e // size * size:(e // size + 1) * size])[-2:].sum()  # noqa: E731
            for a, b in zip(o["topk_ids"][t], ids[t]):
                assert abs(worth(a) - worth(b)) <= 4e-6 or abs(c[a] - c[b]) <= 4e-6, (t, a, b)
        else:
            assert (np.abs(c[o["topk_ids"][t]] - c[ids[t]]) <= 4e-6).all(), t
    # a softmax score far below the bias disappears in their fp32 sum: such choices tie on the GPU and not in fp64, and
    # only the bound above holds for them
    if not (score == "softmax" and with_bias):
        assert same.mean() >= (0.99 if with_bias or group_top == 2 else 1.0)
    check_weights(o["topk_w"], o["topk_ids"], logits, rule)
    check_plan(o, E)


@pytest.mark.parametrize("T,E,k,n_group,topk_group", SHAPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_continuous_logits(T, E, k, n_group, topk_group, score):
    rng = np.random.default_rng(T + 7 * E)
    rule = Rule(score, n_group, topk_group, 1 if E // n_group < 2 else 2, not T % 2, 1.0)
    logits = (3 * rng.standard_normal((T, E))).astype(np.float32)
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32)
    o = run_route(logits, bias, rule, k)
    ids, _ = sro.route(logits, bias, rule, k)
    assert (o["topk_ids"] == ids).all(1).mean() >= 0.99
    for t in np.flatnonzero((o["topk_ids"] != ids).any(1)):
        c = sro.choice_values(logits[t], bias, rule)
        kept = np.sort(c[o["topk_ids"][t]])[::-1]
        assert np.abs(kept - np.sort(c[ids[t]])[::-1]).max() <= 4e-6 or n_group > 1, t
        assert len(set(o["topk_ids"][t])) == k
    check_weights(o["topk_w"], o["topk_ids"], logits, rule)
    check_plan(o, E)


def test_the_plain_rule_is_moe_plan_routing():
    rng = np.random.default_rng(5)
    T, E, k = 500, 96, 6
    logits = rng.standard_normal((T, E)).astype(np.float32)
    logits[::7, 5] = logits[::7, 50]
    o = run_route(logits, None, Rule(), k)
    ids, w = orc.topk_route(logits, k)
    assert np.array_equal(o["topk_ids"], ids) and np.abs(o["topk_w"] - w).max() <= 1e-6
    check_plan(o, E)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("n_group,topk_group,group_top", [(1, 1, 1), (4, 2, 2), (4, 3, 1)])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("E", [40, 128])
def test_masked_infinite_and_nan_logits(score, renormalise, n_group, topk_group, group_top, with_bias, E):
    k = 6
    rng = np.random.default_rng(6)
    x = (rng.integers(-8, 9, (10, E)) / 4).astype(np.float32)
    x[0, :] = -math.inf                                 # nothing left
    x[1, 1:] = -math.inf                                # one expert left
    x[2, ::2] = -math.inf
    x[3, 3:] = np.finfo(np.float32).min                 # the type's lowest value: low, but not masked
    x[4, 5] = math.nan
    x[5, 9] = math.inf
    x[6, :] = math.nan
    x[7, E // 4:3 * E // 4] = -math.inf                             # two whole groups masked
    x[8, :] = 100.0 * np.sign(x[8] + 0.125)             # saturated scores
    x[9, 0], x[9, 1] = math.inf, math.inf
    bias = (rng.integers(-2, 3, E) / 2).astype(np.float32) if with_bias else None
    rule = Rule(score, n_group, topk_group, group_top, renormalise, 1.5)
    o = run_route(x, bias, rule, k)
    for t in range(10):
        got = o["topk_ids"][t]
        assert len(set(got)) == k and got.min() >= 0 and got.max() < E, t
        if t in (8, 9) or sro.spoiled(x[t], rule):
            continue                                    # saturated: order decided by last bits; spoiled: ids are free
        assert list(got) == sro.select(x[t], bias, rule, k)[0], t
    check_weights(o["topk_w"], o["topk_ids"], x, rule)
    check_plan(o, E)
    # gradients of the same rows
    g = rng.standard_normal((10, k)).astype(np.float32)
    d = run_backward(x, o["topk_ids"], g, rule)
    check_backward(d, x, o["topk_ids"], g, rule)


def run_backward(logits, ids, g, rule):
    T, E = logits.shape
    ctx = binding.Context(T, 64, 64, E, ids.shape[1])
    out = torch.full((T, E), 7e30, device=DEV)
    ctx.moe_routing_backward(torch.from_numpy(logits).to(DEV), torch.from_numpy(np.ascontiguousarray(ids)).to(DEV),
                             torch.from_numpy(g).to(DEV), gpu_rule(rule), out)
    torch.cuda.synchronize()
    assert ctx.moe_last_device_status()[0] == 0
    return out.cpu().numpy()


def check_backward(got, logits, ids, g, rule):
    ref = sro.routing_backward(logits.astype(np.float64), ids, g, rule)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    k = ids.shape[1]
    for t in range(len(ids)):
        if np.isnan(ref[t]).any():
            continue
        # the renormalised sigmoid divides by the sum S of the chosen scores: its factors are s (1 - s) / S <= 1
        bound = 1e-5 * rule.weight_scale * np.abs(g[t]).max() * (1 + k)
        assert np.abs(got[t] - ref[t]).max() <= bound, (t, np.abs(got[t] - ref[t]).max(), bound)


@pytest.mark.parametrize("T,E,k,n_group,topk_group", SHAPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_routing_backward(T, E, k, n_group, topk_group, score, renormalise):
    rng = np.random.default_rng(T + E)
    logits = (3 * rng.standard_normal((T, E))).astype(np.float32)
    rule = Rule(score, 1, 1, 1, renormalise, 2.5)
    ids = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    g = rng.standard_normal((T, k)).astype(np.float32)
    check_backward(run_backward(logits, ids, g, rule), logits, ids, g, rule)


def test_routing_backward_reports_an_id_out_of_range():
    ctx = binding.Context(4, 64, 64, 16, 2)
    ids = torch.tensor([[0, 1], [2, 16], [3, -1], [4, 5]], dtype=torch.int32, device=DEV)
    out = torch.full((4, 16), 7e30, device=DEV)
    ctx.moe_routing_backward(torch.zeros(4, 16, device=DEV), ids, torch.ones(4, 2, device=DEV),
                             binding.make_route_rule("sigmoid", renormalise=False), out)
    code, detail = ctx.moe_last_device_status()
    assert code == 4 and detail in (3, 5)
    ref = torch.zeros(4, 16)
    for t, e in ((0, 0), (0, 1), (1, 2), (2, 3), (3, 4), (3, 5)):
        ref[t, e] = 0.25
    assert torch.equal(out.cpu(), ref)
    assert ctx.moe_last_device_status() == (0, 0)


@pytest.mark.parametrize("T,H,E,k", [(1, 64, 1, 1), (5, 64, 4, 2), (33, 576, 8, 3), (7, 7168, 40, 32), (300, 1024, 16, 8),
                                     (64, 4096, 8, 2)])
@pytest.mark.parametrize("frozen", [False, True])
def test_combine_backward(T, H, E, k, frozen):
    rng = np.random.default_rng(T + H)
    ctx = binding.Context(T, H, 64, E, k)
    y_bits = gen.f32_to_bf16_bits(rng.standard_normal((T * k, H)).astype(np.float32))
    g_bits = gen.f32_to_bf16_bits(rng.standard_normal((T, H)).astype(np.float32))
    w = rng.standard_normal((T, k)).astype(np.float32)
    w[0, 0] = 0.0
    inv = rng.permutation(T * k).astype(np.int32)
    d_y = None if frozen else torch.full((T * k, H), float("nan"), dtype=torch.bfloat16, device=DEV)
    d_w = torch.full((T, k), float("nan"), device=DEV)
    args = (bits_to_dev(g_bits), bits_to_dev(y_bits), torch.from_numpy(inv).to(DEV), torch.from_numpy(w).to(DEV))
    ctx.moe_combine_backward(*args, d_y, d_w)
    torch.cuda.synchronize()
    y, g = gen.bf16_bits_to_f32(y_bits).astype(np.float64), gen.bf16_bits_to_f32(g_bits).astype(np.float64)
    ref_y, ref_w = sro.combine_backward(g, y, inv, w.astype(np.float64))
    _, mag = sro.combine_backward(np.abs(g), np.abs(y), inv, w)
    assert (np.abs(d_w.cpu().numpy() - ref_w) <= (H / 32 + 8) * 2.0 ** -24 * mag).all()
    if not frozen:
        got = dev_bf16_to_f64(d_y)
        assert (np.abs(got - ref_y) <= 2.0 ** -8 * np.abs(ref_y)).all()
    again = torch.empty_like(d_w)
    ctx.moe_combine_backward(*args, d_y, again)
    torch.cuda.synchronize()
    assert torch.equal(again, d_w)


def test_router_tuning_step_end_to_end():
    """combine -> d_out -> d_topk_w -> d_logits against central differences of the fp64 layer output."""
    rng = np.random.default_rng(11)
    T, H, E, k = 6, 128, 8, 3
    rule = Rule("sigmoid", 2, 2, 1, True, 2.0)
    logits = (rng.integers(-8, 9, (T, E)) / 4 + rng.permutation(E) / 64).astype(np.float32)
    o = run_route(logits, None, rule, k)
    y_bits = gen.f32_to_bf16_bits(rng.standard_normal((T * k, H)).astype(np.float32))
    g_bits = gen.f32_to_bf16_bits(rng.standard_normal((T, H)).astype(np.float32))
    y, g = gen.bf16_bits_to_f32(y_bits).astype(np.float64), gen.bf16_bits_to_f32(g_bits).astype(np.float64)
    ctx = binding.Context(T, H, 64, E, k)
    to = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    d_w = torch.empty(T, k, device=DEV)
    d_logits = torch.empty(T, E, device=DEV)
    ctx.moe_combine_backward(bits_to_dev(g_bits), bits_to_dev(y_bits), to(o["inv_perm"]), to(o["topk_w"]), None, d_w)
    ctx.moe_routing_backward(to(logits), to(o["topk_ids"]), d_w, gpu_rule(rule), d_logits)
    torch.cuda.synchronize()

    def loss(x):
        w = np.stack([sro.weights(x[t], o["topk_ids"][t], rule) for t in range(T)])
        return float((orc.combine(y, o["inv_perm"], w) * g).sum())

    step, got = 1e-4, d_logits.cpu().numpy()
    for t in range(T):
        for e in range(E):
            x = logits.astype(np.float64)
            up, dn = x.copy(), x.copy()
            up[t, e] += step
            dn[t, e] -= step
            assert abs((loss(up) - loss(dn)) / (2 * step) - got[t, e]) <= 1e-3


def test_another_stream_and_smaller_batches():
    rng = np.random.default_rng(9)
    rule = Rule("sigmoid", 4, 2, 2, True, 2.5)
    logits = (rng.integers(-24, 25, (100, 64)) / 4).astype(np.float32)
    side = torch.cuda.Stream()
    a, b = run_route(logits, None, rule, 4), run_route(logits, None, rule, 4, stream=side)
    assert all(np.array_equal(a[n], b[n]) for n in a)
    ctx = binding.Context(100, 64, 64, 64, 4)
    for T in (99, 1, 0):
        ctx.moe_set_active_tokens(T)
        i32 = dict(dtype=torch.int32, device=DEV)
        ids, w = torch.full((max(T, 1), 4), -1, **i32), torch.empty(max(T, 1), 4, device=DEV)
        counts, offsets = torch.full((64,), -1, **i32), torch.full((65,), -1, **i32)
        perm, inv = torch.full((max(T, 1) * 4,), -1, **i32), torch.full((max(T, 1) * 4,), -1, **i32)
        ctx.moe_plan_routing_scored(torch.from_numpy(logits[:max(T, 1)]).to(DEV), None, gpu_rule(rule), ids, w, counts,
                                    offsets, perm, inv)
        torch.cuda.synchronize()
        assert int(offsets[-1]) == 4 * T
        if T:
            assert np.array_equal(ids.cpu().numpy(), a["topk_ids"][:T])
        else:
            assert counts.eq(0).all() and ids.eq(-1).all()


def test_refusals():
    T, E, k = 8, 24, 6
    ctx = binding.Context(T, 64, 64, E, k)
    i32 = dict(dtype=torch.int32, device=DEV)
    x, w = torch.zeros(T, E, device=DEV), torch.zeros(T, k, device=DEV)
    ids, counts, offsets = torch.zeros(T, k, **i32), torch.zeros(E, **i32), torch.zeros(E + 1, **i32)
    perm, inv = torch.zeros(T * k, **i32), torch.zeros(T * k, **i32)

    def call(rule, x=x, bias=None):
        ctx.moe_plan_routing_scored(x, bias, rule, ids, w, counts, offsets, perm, inv)

    ok = dict(score="sigmoid", n_group=4, topk_group=2, group_top=2)
    call(binding.make_route_rule(**ok))
    bad_rules = [dict(ok, n_group=5), dict(ok, n_group=0), dict(ok, n_group=48), dict(ok, topk_group=0),
                 dict(ok, topk_group=5), dict(ok, group_top=3), dict(ok, group_top=0), dict(ok, n_group=24, topk_group=24),
                 dict(ok, n_group=12, topk_group=2), dict(ok, weight_scale=math.inf), dict(ok, weight_scale=math.nan)]
    for r in bad_rules:
        for f in (lambda rule: call(rule), lambda rule: ctx.moe_routing_backward(x, ids, w, rule, x)):
            with pytest.raises(binding.MoeError) as e:
                f(binding.make_route_rule(**r))
            assert e.value.code == 1, r
    raw = binding.make_route_rule(**ok)
    raw.score = 2
    with pytest.raises(binding.MoeError):
        call(raw)
    raw = binding.make_route_rule(**ok)
    raw.renormalise = 2
    with pytest.raises(binding.MoeError):
        call(raw)
    with pytest.raises(ValueError):
        binding.make_route_rule(score="tanh")
    flat = torch.zeros(T * E + 4, device=DEV)
    with pytest.raises(binding.MoeError) as e:              # misaligned
        call(binding.make_route_rule(**ok), x=flat[1:1 + T * E].view(T, E))
    assert e.value.code == 1
    with pytest.raises(binding.MoeError):
        call(binding.make_route_rule(**ok), x=None)
    with pytest.raises(ValueError):                         # strided
        call(binding.make_route_rule(**ok), x=torch.zeros(E, T, device=DEV).t())
    with pytest.raises(binding.MoeError):
        ctx.moe_combine_backward(None, x, inv, w, None, w)


def sigmoid_gradient_parts(x, ids, g, rule):
    """Per chosen slot, in 64 bits and from sigmoids of both signs (no 1 - s): the gradient, and the factor that its
    rounding errors are relative to."""
    xs = np.take_along_axis(x.astype(np.float64), ids.astype(np.int64), 1)
    e = np.exp(-np.abs(xs))
    s, c = np.where(xs >= 0, 1 / (1 + e), e / (1 + e)), np.where(xs >= 0, e / (1 + e), 1 / (1 + e))
    g = g.astype(np.float64) * rule.weight_scale
    if not rule.renormalise:
        return g * s * c, np.abs(g) * s * c
    q = s / s.sum(1, keepdims=True)
    return q * (g - (g * q).sum(1, keepdims=True)) * c, q * c * (np.abs(g) + (np.abs(g) * q).sum(1, keepdims=True))


@pytest.mark.parametrize("E,k", [(8, 2), (96, 6), (256, 8), (1024, 32)])
@pytest.mark.parametrize("renormalise", [True, False])
def test_sigmoid_gradient_of_saturated_logits(E, k, renormalise):
    """Every element against its own size where scores are near 0 or 1.  expf is within 2 ulp and a sigmoid adds two
    roundings, so s and 1 - s carry 3.6e-7; a product of them with g 1e-6, a share of a sum of 32 another 8e-7 and the mean
    of g as much again: 1.5e-6 without the sum, 4e-6 with it."""
    rng = np.random.default_rng(E + k)
    levels = np.array([-88.0, -80.0, -30.0, -4.0, 0.0, 5.0, 12.0, 17.0, 20.0, 40.0, 80.0, 88.0])
    x = (levels.repeat(4)[:, None] + rng.uniform(-0.5, 0.5, (48, E))).astype(np.float32)
    mixed = rng.choice(levels, (16, E)) + rng.uniform(-0.5, 0.5, (16, E))
    x = np.concatenate([x, mixed.astype(np.float32)])
    ids = np.stack([rng.permutation(E)[:k] for _ in x]).astype(np.int32)
    g = (rng.standard_normal((len(x), k)) * 10.0 ** rng.uniform(-2, 2, (len(x), 1))).astype(np.float32)
    rule = Rule("sigmoid", 1, 1, 1, renormalise, 2.5)
    got = run_backward(x, ids, g, rule)
    ref, size = sigmoid_gradient_parts(x, ids, g, rule)
    err = np.abs(np.take_along_axis(got, ids.astype(np.int64), 1) - ref)
    assert (err <= (4e-6 if renormalise else 1.5e-6) * size + 1e-44).all(), np.nanmax(err / (size + 1e-44))
    others = got.copy()
    np.put_along_axis(others, ids.astype(np.int64), 0.0, 1)
    assert not others.any()


def test_sigmoid_gradient_of_saturated_logits_against_differences():
    """The same where the slope is all that is left of the score: central differences of the fp64 weights."""
    x = np.array([[12.0, 12.5, 11.5, -3.0], [20.0, 19.0, 21.0, 0.0], [-20.0, -21.0, -19.5, 4.0]], dtype=np.float32)
    ids = np.tile(np.array([0, 1, 2], dtype=np.int32), (3, 1))
    g = np.array([[1.0, -2.0, 0.5]] * 3, dtype=np.float32)
    for renormalise in (True, False):
        rule = Rule("sigmoid", 1, 1, 1, renormalise, 1.0)
        got = run_backward(x, ids, g, rule)
        for t in range(3):
            for e in range(3):
                w = []
                for step in (1e-2, -1e-2):
                    v = x[t].astype(np.float64)
                    v[e] += step
                    w.append(sro.weights(v, ids[t], rule))
                # third derivative of a weight: at most its slope, so the difference is off by step^2 / 6 of it
                diff = float(((w[0] - w[1]) * g[t]).sum() / 2e-2)
                assert abs(got[t, e] - diff) <= 1e-4 * np.abs(got[t]).max(), (renormalise, t, e, got[t, e], diff)


def softmax_gradient_bound(x, ids, g, rule):
    """Per element [T,E]: what the rounding errors of a softmax gradient are relative to, s_e (|g_e| + sum_i |g_i| s_i)."""
    T, E = x.shape
    size = np.zeros((T, E))
    for t in range(T):
        sel = list(ids[t])
        a = np.abs(g[t].astype(np.float64)) * rule.weight_scale
        if rule.renormalise:
            q = sro.scores(x[t, sel], rule)
            size[t, sel] = q * (a + (a * q).sum())
        else:
            s = sro.scores(x[t], rule)
            full = np.zeros(E)
            full[sel] = a
            size[t] = s * (full + (a * s[sel]).sum())
    return size


@pytest.mark.parametrize("T,E,k,n_group,topk_group", SHAPES)
@pytest.mark.parametrize("renormalise", [True, False])
def test_softmax_gradient_element_by_element(T, E, k, n_group, topk_group, renormalise):
    """Every element against its own size, so that the small gradients of unchosen experts count.  For |x - max| <= 30: the
    argument's rounding 1.8e-6 and expf 2.4e-7 relative in an exponential; a sum of 1024 of them adds 37 roundings: 6.3e-6 in
    a score, 6.7e-6 in the weighted sum of k gradients: 1.5e-5 of the element's size with the remaining products."""
    rng = np.random.default_rng(T * 3 + E)
    x = np.clip(3 * rng.standard_normal((T, E)), -14, 14).astype(np.float32)
    rule = Rule("softmax", 1, 1, 1, renormalise, 2.5)
    ids = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    g = rng.standard_normal((T, k)).astype(np.float32)
    got = run_backward(x, ids, g, rule)
    ref = sro.routing_backward(x.astype(np.float64), ids, g, rule)
    size = softmax_gradient_bound(x, ids, g, rule)
    err = np.abs(got - ref)
    assert (err <= 1.5e-5 * size + 1e-37).all(), np.max(err / (size + 1e-37))


def admissible(ids, x, bias, rule, k):
    """Whether an fp32 choice may hold these experts: with choice values and groups' worths (fp64) that are off by at most
    2e-6 each, every expert is in a group that stays and among the k best of such groups."""
    c = sro.choice_values(x, bias, rule)
    E, size = len(c), len(c) // rule.n_group
    rank = c
    if bias is None and rule.group_top == 2:
        rank = np.where(np.isneginf(c), -math.inf, sro.scores(x, rule))
    worth = np.array([np.sort(rank[j * size:(j + 1) * size])[::-1][:rule.group_top].sum() for j in range(rule.n_group)])
    edge = np.sort(worth)[::-1][rule.topk_group - 1]
    may, must = worth >= edge - 4e-6, worth > edge + 4e-6
    mine = set(int(e) // size for e in ids)
    if not all(may[j] for j in mine) or len(set(ids)) != k:
        return False
    # the kept groups: all that have to stay, those that were used, and the best of the others
    kept = sorted(range(rule.n_group), key=lambda j: (not (must[j] or j in mine), -worth[j]))[:rule.topk_group]
    if must.sum() == rule.topk_group or may.sum() == rule.topk_group:
        kept = list(np.flatnonzero(may if may.sum() == rule.topk_group else must))
    open_ = np.concatenate([np.arange(j * size, (j + 1) * size) for j in kept])
    if not set(int(e) for e in ids) <= set(open_):
        return False
    if may.sum() > rule.topk_group:
        return True                                        # more than one set of groups may stay
    return bool(np.abs(np.sort(c[ids])[::-1] - np.sort(c[open_])[::-1][:k]).max() <= 4e-6)


@pytest.mark.parametrize("T,E,k,n_group,topk_group,group_top", [
    (2000, 256, 8, 8, 4, 2), (2000, 256, 8, 8, 4, 1), (1500, 128, 6, 4, 2, 2), (1500, 160, 6, 8, 3, 2),
    (1500, 96, 6, 6, 3, 1), (700, 512, 20, 16, 4, 2), (700, 1000, 32, 25, 7, 2), (400, 1024, 12, 32, 5, 2),
    (1000, 64, 4, 32, 9, 2), (1000, 24, 12, 24, 12, 1),
])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [True, False])
def test_grouped_choices_differ_only_within_rounding(T, E, k, n_group, topk_group, group_top, score, with_bias):
    rng = np.random.default_rng(T + 11 * E + k)
    rule = Rule(score, n_group, topk_group, group_top, True, 1.0)
    x = (3 * rng.standard_normal((T, E))).astype(np.float32)
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32) if with_bias else None
    o = run_route(x, bias, rule, k)
    ids, _ = sro.route(x, bias, rule, k)
    differ = np.flatnonzero((o["topk_ids"] != ids).any(1))
    assert len(differ) <= 0.01 * T
    for t in differ:
        assert admissible(o["topk_ids"][t], x[t], bias, rule, k), t
    check_plan(o, E)


def test_the_grouped_check_refuses_wrong_choices():
    """The check above on the oracle's own choices and on choices that are wrong (no kernel involved)."""
    rng = np.random.default_rng(2)
    rule, k = Rule("sigmoid", 8, 4, 2, True, 1.0), 8
    refused = 0
    for _ in range(200):
        x, bias = (3 * rng.standard_normal(256)).astype(np.float32), (0.1 * rng.standard_normal(256)).astype(np.float32)
        ids, c = sro.select(x, bias, rule, k)
        ids = np.array(ids)
        assert admissible(ids, x, bias, rule, k)
        groups = set(ids // 32)
        closed = [e for e in range(256) if e // 32 not in groups]
        best_closed = max(closed, key=lambda e: c[e])
        other = ids.copy()
        other[-1] = best_closed                                # an expert of a group that does not stay
        worse = ids.copy()
        worse[0] = min((e for e in range(256) if e // 32 == ids[0] // 32), key=lambda e: c[e])
        refused += (not admissible(other, x, bias, rule, k)) + (not admissible(worse, x, bias, rule, k))
    assert refused >= 390
