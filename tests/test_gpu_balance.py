"""The balance loss of a router, its counts and its gradient on the GPU against the oracle.

Bounds, in roundings of 2^-24: an exponential's argument x - max is rounded once (its size r, at most the logits' range, in
units of the result) and expf adds 2; the sum over up to 1024 experts adds 37, the quotient 2: a probability is within
(2 r + 43) of its value, for sigmoid scores (whose exponentials' arguments are at most the logit) alike.  A mean adds a slot's
tokens (4 a warp, 8 warps) and up to slots / 32 + 32 partial sums, all positive.  The gradient adds the weighted sum (37), u and the
products: (4 r + 140) of p (|u| + sum |u| p), and of the second loss's part, where the logarithm itself is within 4 + 43 / |log|."""
import numpy as np
import pytest
import torch

from oracle import around_oracle as ao
from oracle import scored_router_oracle as sro
from paper_2607_23264_b200 import binding
from moe_testlib import DEV

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def choose(rng, T, E, k):
    return np.argsort(rng.random((T, E)), axis=1)[:, :k].astype(np.int32)


def run_loss(ctx, x, ids, scratch=None, stream=None, **kw):
    S, E = kw.get("sequences", 1), x.shape[1]
    o = dict(counts=torch.full((S, E), -7, dtype=torch.int32, device=DEV),
             tokens=torch.full((S + 1,), -7, dtype=torch.int32, device=DEV),
             mean=torch.full((S, E), float("nan"), device=DEV), loss=torch.full((2,), float("nan"), device=DEV))
    if scratch is None:
        scratch = torch.full((ctx.balance_scratch_bytes(S),), 0xFF, dtype=torch.uint8, device=DEV)
    ctx.moe_balance_loss(x, ids, o["counts"], o["tokens"], o["mean"], o["loss"], scratch, stream=stream, **kw)
    return o


def case(rng, T, E, k, S, masked, spread=3.0):
    x = (spread * rng.standard_normal((T, E))).astype(np.float32)
    ids = choose(rng, T, E, k)
    offsets = None
    if S > 1:
        cuts = np.sort(rng.integers(0, T + 1, S))
        offsets = np.concatenate([[0], cuts]).astype(np.int32)       # the last tokens may lie behind every sequence
    mask = (rng.random(T) < 0.7).astype(np.uint8) if masked else None
    return x, ids, offsets, mask


CASES = [(1, 1, 1, 1, False), (1, 8, 2, 1, False), (7, 5, 3, 1, True), (31, 33, 4, 3, False), (33, 64, 6, 5, True),
         (1000, 96, 6, 1, False), (1000, 100, 32, 40, True), (4099, 64, 6, 13, True), (3000, 256, 8, 1, False), (513, 300, 5, 7, True),
         (700, 512, 8, 2, False), (300, 1024, 12, 1, True), (260, 1000, 3, 260, False), (16384, 256, 8, 1, False)]


@pytest.mark.parametrize("T,E,k,S,masked", CASES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("z_coef", [0.0, 0.02])
def test_loss_and_gradient_against_oracle(T, E, k, S, masked, score, z_coef):
    rng = np.random.default_rng(T * 5 + E + S)
    x, ids, offsets, mask = case(rng, T, E, k, S, masked)
    ctx = binding.Context(T, 64, 64, E, k)
    xd, how = dev(x), dict(score=score, coef=0.3, z_coef=z_coef, sequences=S, seq_offsets=dev(offsets), token_mask=dev(mask))
    o = run_loss(ctx, xd, dev(ids), **how)
    assert ctx.moe_last_device_status() == (0, 0)
    counts, tokens, mean, loss = ao.balance_loss(x, ids, score, 0.3, z_coef, offsets, mask, S)
    assert np.array_equal(o["counts"].cpu().numpy(), counts) and np.array_equal(o["tokens"].cpu().numpy(), tokens)
    r = float(x.max() - x.min())
    deep = 2 * r + 43 + 4 + 8 + T / 1024 + 32
    got = o["mean"].cpu().numpy().astype(np.float64)
    assert (np.abs(got - mean) <= deep * U * mean + 1e-38).all()
    lse = ao.probabilities(x, score)[1]
    assert abs(float(o["loss"][0]) - loss[0]) <= (deep + 50) * U * loss[0] + 1e-38
    off = 2 * np.abs(lse).max() * (43 + 4 * np.abs(lse).max()) * U * z_coef
    assert abs(float(o["loss"][1]) - loss[1]) <= off + (T / 1024 + 60) * U * loss[1]

    d_loss, add = torch.full((1,), 37.0, device=DEV), rng.standard_normal((T, E)).astype(np.float32)
    ref, size = ao.balance_loss_backward(x, counts, tokens, k, score, 0.3, z_coef, 37.0, offsets, mask, S)
    bound = (4 * r + 140) * U * size + (43 * U * 37 * 2 * z_coef / max(1, tokens[-1])) + 1e-38
    d = torch.full((T, E), float("nan"), device=DEV)
    ctx.moe_balance_loss_backward(xd, o["counts"], o["tokens"], d, d_loss=d_loss, **how)
    assert (np.abs(d.cpu().numpy() - ref) <= bound).all()
    into = dev(add)
    ctx.moe_balance_loss_backward(xd, o["counts"], o["tokens"], into, d_loss=d_loss, add=into, **how)
    assert (np.abs(into.cpu().numpy() - (ref + add)) <= bound + 2 * U * (np.abs(add) + np.abs(ref))).all()
    seq = ao.sequence_of(T, offsets, mask)
    assert torch.equal(into.cpu()[torch.from_numpy(seq < 0)], torch.from_numpy(add)[torch.from_numpy(seq < 0)])
    # without d_loss: 1
    ctx.moe_balance_loss_backward(xd, o["counts"], o["tokens"], into, **how)
    one, size = ao.balance_loss_backward(x, counts, tokens, k, score, 0.3, z_coef, 1.0, offsets, mask, S)
    assert (np.abs(into.cpu().numpy() - one) <= bound / 37 + 1e-38).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_far_logits(score):
    """Logits of +-80 and rows far below zero: probabilities keep their digits, element by element."""
    rng = np.random.default_rng(3)
    T, E, k = 200, 64, 4
    x = rng.uniform(-80, 80, (T, E)).astype(np.float32)
    x[:50] = rng.uniform(-180, -100, (50, E))
    x[50:80] = rng.uniform(-45, -35, (30, E))
    ids = choose(rng, T, E, k)
    ctx = binding.Context(T, 64, 64, E, k)
    o = run_loss(ctx, dev(x), dev(ids), score=score)
    counts, tokens, mean, loss = ao.balance_loss(x, ids, score, 1.0, 0.0)
    assert (np.abs(o["mean"].cpu().numpy() - mean) <= (2 * 180 + 130) * U * mean + 1e-38).all()
    d = torch.empty(T, E, device=DEV)
    ctx.moe_balance_loss_backward(dev(x), o["counts"], o["tokens"], d, score=score)
    ref, size = ao.balance_loss_backward(x, counts, tokens, k, score, 1.0, 0.0)
    # (an exponential below 2^-126 has fewer digits: 2^-149 of the largest)
    assert (np.abs(d.cpu().numpy() - ref) <= (4 * 180 + 140) * U * size + 2.0 ** -120).all()


def masked_logits(T, E, rng):
    x = rng.standard_normal((T, E)).astype(np.float32)
    x[rng.random((T, E)) < 0.3] = -np.inf
    x[2] = -np.inf
    x[3] = np.finfo(np.float32).min                          # a mask of the type's lowest value: all alike
    x[4, 1:] = np.finfo(np.float32).min
    return x


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_masked_experts(score):
    rng = np.random.default_rng(4)
    T, E, k = 70, 40, 3
    x, ids = masked_logits(T, E, rng), choose(rng, T, E, k)
    ctx = binding.Context(T, 64, 64, E, k)
    o = run_loss(ctx, dev(x), dev(ids), score=score, coef=0.5)
    counts, tokens, mean, loss = ao.balance_loss(x, ids, score, 0.5, 0.0)
    assert np.array_equal(o["counts"].cpu().numpy(), counts) and o["tokens"][-1] == T
    assert (np.abs(o["mean"].cpu().numpy() - mean) <= 150 * U * mean + 1e-38).all()
    d = torch.full((T, E), float("nan"), device=DEV)
    ctx.moe_balance_loss_backward(dev(x), o["counts"], o["tokens"], d, score=score, coef=0.5)
    ref, size = ao.balance_loss_backward(x, counts, tokens, k, score, 0.5, 0.0)
    d = d.cpu().numpy()
    assert (np.abs(d - ref) <= 170 * U * size + 1e-38).all()
    assert (d[np.isneginf(x)] == 0).all() and (d[2] == 0).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_nan_spoils_its_row_and_the_losses_only_when_it_counts(score):
    rng = np.random.default_rng(5)
    T, E, k = 64, 32, 2
    x, ids = rng.standard_normal((T, E)).astype(np.float32), choose(rng, T, E, k)
    x[9, 3] = np.nan
    ctx = binding.Context(T, 64, 64, E, k)
    o = run_loss(ctx, dev(x), dev(ids), score=score, z_coef=1.0)
    assert o["loss"].isnan().all() and int(o["counts"].sum()) == T * k
    d = torch.zeros(T, E, device=DEV)
    ctx.moe_balance_loss_backward(dev(x), o["counts"], o["tokens"], d, score=score)
    assert d[9].isnan().all() and d[:9].isfinite().all() and d[10:].isfinite().all()
    mask = np.ones(T, np.uint8)
    mask[9] = 0
    o = run_loss(ctx, dev(x), dev(ids), score=score, z_coef=1.0, token_mask=dev(mask))
    assert o["loss"].isfinite().all() and int(o["tokens"][0]) == T - 1
    ctx.moe_balance_loss_backward(dev(x), o["counts"], o["tokens"], d, score=score, token_mask=dev(mask))
    assert (d[9] == 0).all() and d.isfinite().all()


def test_nothing_counts_and_no_tokens():
    T, E, k = 40, 16, 2
    ctx = binding.Context(T, 64, 64, E, k)
    x, ids = torch.randn(T, E, device=DEV), dev(choose(np.random.default_rng(0), T, E, k))
    none = torch.zeros(T, dtype=torch.uint8, device=DEV)
    for how in (dict(token_mask=none, z_coef=1.0), dict(seq_offsets=torch.zeros(4, dtype=torch.int32, device=DEV), sequences=3)):
        o = run_loss(ctx, x, ids, **how)
        assert (o["loss"] == 0).all() and (o["counts"] == 0).all() and (o["tokens"] == 0).all() and (o["mean"] == 0).all()
        d = torch.full((T, E), float("nan"), device=DEV)
        ctx.moe_balance_loss_backward(x, o["counts"], o["tokens"], d, **how)
        assert (d == 0).all()
    ctx.moe_set_active_tokens(0)
    o = run_loss(ctx, x, ids)
    assert (o["loss"] == 0).all() and (o["counts"] == 0).all() and (o["tokens"] == 0).all()


def test_bad_ids_are_reported_and_not_counted():
    T, E, k = 50, 24, 3
    rng = np.random.default_rng(6)
    ids = choose(rng, T, E, k)
    x = rng.standard_normal((T, E)).astype(np.float32)
    ctx = binding.Context(T, 64, 64, E, k)
    for bad in (-1, E, 2 ** 31 - 1):
        spoiled = ids.copy()
        spoiled[17, 1] = bad
        o = run_loss(ctx, dev(x), dev(spoiled))
        assert ctx.moe_last_device_status() == (4, 17 * k + 1)
        assert int(o["counts"].sum()) == T * k - 1 and int(o["tokens"][0]) == T
    assert ctx.moe_last_device_status() == (0, 0)


def test_same_bits_every_time_on_any_stream_and_from_graphs():
    T, E, k, S = 2000, 64, 4, 9
    rng = np.random.default_rng(7)
    x, ids, offsets, mask = case(rng, T, E, k, S, True)
    ctx = binding.Context(T, 64, 64, E, k)
    xd, idd = dev(x), dev(ids)
    how = dict(score="sigmoid", coef=0.1, z_coef=0.01, sequences=S, seq_offsets=dev(offsets), token_mask=dev(mask))
    want = run_loss(ctx, xd, idd, **how)
    grad = torch.empty(T, E, device=DEV)
    ctx.moe_balance_loss_backward(xd, want["counts"], want["tokens"], grad, **how)
    torch.cuda.synchronize()
    # two graphs with a scratch each, replayed beside one another
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    graphs, outs = [], []
    for s in side:
        scratch = torch.empty(ctx.balance_scratch_bytes(S), dtype=torch.uint8, device=DEV)
        o = {n: torch.empty_like(t) for n, t in want.items()}
        d = torch.empty_like(grad)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            ctx.moe_balance_loss(xd, idd, o["counts"], o["tokens"], o["mean"], o["loss"], scratch, **how)
            ctx.moe_balance_loss_backward(xd, o["counts"], o["tokens"], d, **how)
        graphs.append((g, scratch))
        outs.append((o, d))
    for _ in range(5):
        for (g, _), s in zip(graphs, side):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for o, d in outs:
            assert all(torch.equal(o[n], want[n]) for n in o) and torch.equal(d, grad)
            for t in (*o.values(), d):
                t.zero_()
        torch.cuda.synchronize()


def test_gradient_beside_the_weights_gradient():
    """The router's whole gradient: moe_routing_backward, then the loss's added to it; against differences of the oracle."""
    T, E, k = 24, 16, 3
    rng = np.random.default_rng(8)
    x, dw = rng.standard_normal((T, E)).astype(np.float32), rng.standard_normal((T, k)).astype(np.float32)
    ids = choose(rng, T, E, k)
    rule = sro.Rule("sigmoid", 1, 1, 1, True, 1.0)
    ctx = binding.Context(T, 64, 64, E, k)
    d = torch.empty(T, E, device=DEV)
    xd, idd = dev(x), dev(ids)
    ctx.moe_routing_backward(xd, idd, dev(dw), binding.make_route_rule("sigmoid"), d)
    o = run_loss(ctx, xd, idd, score="sigmoid", coef=0.4)
    ctx.moe_balance_loss_backward(xd, o["counts"], o["tokens"], d, add=d, score="sigmoid", coef=0.4)

    def value(v):
        w = np.stack([sro.weights(v[t], ids[t], rule) for t in range(T)])
        return (w * dw).sum() + ao.balance_loss(v, ids, "sigmoid", 0.4, 0.0)[3][0]

    d, v = d.cpu().numpy(), x.astype(np.float64)
    for at in [(0, 0), (3, int(ids[3, 1])), (23, 15), (11, int(ids[11, 0]))]:
        up, down = v.copy(), v.copy()
        up[at] += 1e-5
        down[at] -= 1e-5
        assert abs((value(up) - value(down)) / 2e-5 - d[at]) < 1e-6


def test_many_sequences_of_one_token():
    T, E, k = 5000, 8, 2
    rng = np.random.default_rng(9)
    x, ids = rng.standard_normal((T, E)).astype(np.float32), choose(rng, T, E, k)
    offsets = np.arange(T + 1, dtype=np.int32)
    ctx = binding.Context(T, 64, 64, E, k)
    o = run_loss(ctx, dev(x), dev(ids), sequences=T, seq_offsets=dev(offsets))
    counts, tokens, mean, loss = ao.balance_loss(x, ids, "softmax", 1.0, 0.0, offsets, None, T)
    assert np.array_equal(o["counts"].cpu().numpy(), counts) and np.array_equal(o["tokens"].cpu().numpy(), tokens)
    assert (np.abs(o["mean"].cpu().numpy() - mean) <= 150 * U * mean).all()
    assert abs(float(o["loss"][0]) - loss[0]) <= 200 * U * loss[0]


def test_refusals():
    T, E, k = 8, 16, 2
    ctx = binding.Context(T, 64, 64, E, k)
    x, ids = torch.zeros(T, E, device=DEV), torch.zeros(T, k, dtype=torch.int32, device=DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    c, n, m, l = torch.zeros(2, E, **i32), torch.zeros(4, **i32), torch.zeros(2, E, device=DEV), torch.zeros(2, device=DEV)
    scratch = torch.zeros(ctx.balance_scratch_bytes(2), dtype=torch.uint8, device=DEV)
    off = torch.zeros(4, **i32)
    good = dict(logits=x, topk_ids=ids, counts=c, tokens=n, mean=m, loss=l, scratch=scratch)
    for change, code in [(dict(logits=None), 1), (dict(topk_ids=None), 1), (dict(counts=None), 1), (dict(tokens=None), 1),
                         (dict(mean=None), 1), (dict(loss=None), 1), (dict(scratch=None), 1), (dict(coef=float("nan")), 1),
                         (dict(z_coef=float("inf")), 1), (dict(sequences=0), 2), (dict(sequences=2), 1),
                         (dict(sequences=(1 << 20) + 1, seq_offsets=off), 2), (dict(scratch=scratch[:64]), 3),
                         (dict(seq_offsets=off[1:3]), 1), (dict(token_mask=scratch[1:T + 1]), 1)]:
        with pytest.raises(binding.MoeError) as err:
            ctx.moe_balance_loss(**{**good, **change})
        assert err.value.code == code, change
    for change in (dict(counts=None), dict(tokens=None), dict(d_logits=None), dict(logits=None), dict(d_loss=l[1:])):
        with pytest.raises(binding.MoeError) as err:
            ctx.moe_balance_loss_backward(**{**dict(logits=x, counts=c, tokens=n, d_logits=x), **change})
        assert err.value.code == 1
    with pytest.raises(ValueError, match="score"):
        ctx.moe_balance_loss(**good, score="relu")
    assert ctx.balance_scratch_bytes(0) == 0
