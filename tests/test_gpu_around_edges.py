"""The operators around the layer where their own files do not look: infinite logits, gradients of rows between 8192 and 16384
columns, rows beyond fp32's squares, and captured graphs replayed on other inputs (sequences, masks, choices and segments
are found on the device, so a graph has to follow them).  Bounds are those of test_gpu_norm and test_gpu_balance; a replay gives
the bits of a fresh call on the same inputs."""
import numpy as np
import pytest
import torch

from moe_testlib import DEV, dev_bf16_to_f64
from oracle import around_oracle as ao
from paper_2607_23264_b200 import binding
from test_gpu_adapter_edges import context
from test_gpu_balance import case, choose, dev, run_loss
from test_gpu_norm import EPS, U, bf16, make, outputs, run_backward
import test_gpu_adapters as ga

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(1, 64, 64, 1, 1)


# -------------------------------------------------------------------------------------------------------------- norm
@pytest.mark.parametrize("rows,cols", [(333, 8200), (149, 9216), (40, 10248), (301, 12288), (7, 12296), (160, 15352), (450, 11272)])
@pytest.mark.parametrize("with_sum,gain,offset", [(True, "bf16", 0.0), (False, "fp32", 1.0)])
def test_gradients_of_rows_of_nine_to_fifteen_warps(ctx, rows, cols, with_sum, gain, offset):
    rng = np.random.default_rng(rows + cols)
    s, sv, e, ev, g, gv = make(rng, rows, cols, gain)
    d, dv = bf16(rng.standard_normal((rows, cols)) * np.exp(rng.uniform(-3, 3, (rows, 1))))
    dx, dg = run_backward(ctx, s, g, d, e if with_sum else None, rows, cols, offset=offset)
    rx, rg, size_x, size_g = ao.rms_norm_backward(sv, gv, dv, ev if with_sum else None, EPS, offset)
    assert (np.abs(dev_bf16_to_f64(dx) - rx) <= 2.0 ** -8 * np.abs(rx) + 80 * U * size_x + 2.0 ** -134).all()
    ctas = ctx.rms_norm_scratch_bytes(rows, cols) // (4 * cols)
    assert (np.abs(dg.cpu().numpy() - rg) <= (-(-rows // ctas) + ctas / 8 + 50) * U * size_g + 1e-38).all()
    again, _ = run_backward(ctx, s, g, d, e if with_sum else None, rows, cols, offset=offset, want=("dx",))
    assert torch.equal(again, dx)


def test_gradient_of_rows_beyond_fp32s_squares(ctx):
    """Such a row is normalised to zeros, so it passes d_sum on and adds nothing to the gain's gradient."""
    rng = np.random.default_rng(0)
    rows, cols = 6, 512
    s, sv, e, ev, g, gv = make(rng, rows, cols)
    d, dv = bf16(rng.standard_normal((rows, cols)))
    s[2] = 1e25
    dx, dg = run_backward(ctx, s, g, d, e, rows, cols)
    keep = [0, 1, 3, 4, 5]
    want_x, want_g = run_backward(ctx, s[keep], g, d[keep], e[keep], 5, cols)
    assert torch.equal(dx[2], e[2]) and torch.equal(dx[keep], want_x)
    _, rg, _, size_g = ao.rms_norm_backward(sv[keep], gv, dv[keep], ev[keep], EPS)
    assert (np.abs(dg.cpu().numpy() - rg) <= 80 * U * size_g + 1e-38).all()


@pytest.mark.parametrize("rows,cols,form,with_residual", [(70, 1024, "blk", True), (2000, 512, "rows", False), (513, 1152, "mx", True),
                                                          (3000, 2048, "none", False)])
def test_norm_replayed_on_other_inputs(ctx, rows, cols, form, with_residual):
    rng = np.random.default_rng(rows)
    sets = [make(rng, rows, cols)[::2] for _ in range(3)]                # x, residual, gain
    sets[2][0][rows // 2] = 0
    sets[2][0][1, 5] = float("inf")
    x, r, g = (t.clone() for t in sets[0])
    d, _ = bf16(rng.standard_normal((rows, cols)))
    o, dx, dg = outputs(rows, cols, form), torch.empty_like(x), torch.empty(cols, device=DEV)
    scratch = torch.empty(ctx.rms_norm_scratch_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        ctx.moe_add_rms_norm(x, r if with_residual else None, g, rows, cols, form=form, **o)
        ctx.moe_rms_norm_backward(o["sum_out"], g, d, rows, cols, dx, dg, scratch, d_sum=r)
    for new in sets:
        for to, source in zip((x, r, g), new):
            to.copy_(source)
        graph.replay()
        torch.cuda.synchronize()
        want = outputs(rows, cols, form)
        ctx.moe_add_rms_norm(new[0], new[1] if with_residual else None, new[2], rows, cols, form=form, **want)
        wx, wg = run_backward(ctx, want["sum_out"], new[2], d, new[1], rows, cols)
        assert all(torch.equal(o[n].view(torch.uint8), want[n].view(torch.uint8)) for n in o)
        assert torch.equal(dx.view(torch.int16), wx.view(torch.int16)) and torch.equal(dg.view(torch.int32), wg.view(torch.int32))


# ------------------------------------------------------------------------------------------------------------- balance
@pytest.mark.parametrize("E", [16, 128, 200, 384])
@pytest.mark.parametrize("z_coef", [0.0, 0.5])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_infinite_logits(score, z_coef, E):
    """+inf is NaN to a softmax and to the logarithm of the sum, and 1 to a sigmoid."""
    rng = np.random.default_rng(11)
    T, k = 90, 2
    x, ids = rng.standard_normal((T, E)).astype(np.float32), choose(rng, T, E, k)
    x[9, 3], x[9, 5] = np.inf, -np.inf
    ctx = binding.Context(T, 64, 64, E, k)
    how = dict(score=score, coef=0.5, z_coef=z_coef)
    o = run_loss(ctx, dev(x), dev(ids), **how)
    d = torch.full((T, E), float("nan"), device=DEV)
    ctx.moe_balance_loss_backward(dev(x), o["counts"], o["tokens"], d, **how)
    d = d.cpu().numpy()
    rest = np.arange(T) != 9
    finite = x.copy()
    finite[9, 3] = 90                                             # sigma is 1 to 2^-129 there
    counts, tokens, mean, loss = ao.balance_loss(finite, ids, score, 0.5, z_coef)
    ref, size = ao.balance_loss_backward(finite, counts, tokens, k, score, 0.5, z_coef)
    # the logarithm of a sum enters with its size, below 10 (4 + 43 / |log| roundings of |log|)
    bound = (4 * 90 + 140) * U * size + (43 + 40) * U * 2 * z_coef / T + 1e-38
    assert np.array_equal(o["counts"].cpu().numpy(), counts)
    assert (np.abs(d - ref) <= bound)[rest].all()
    if score == "sigmoid":
        assert (np.abs(o["mean"].cpu().numpy() - mean) <= (2 * 90 + 130) * U * mean + 1e-38).all()
        assert abs(float(o["loss"][0]) - loss[0]) <= 400 * U * loss[0]
    else:
        assert o["loss"][0].isnan() and o["mean"].isnan().all()
    if score == "softmax" or z_coef:
        assert np.isnan(d[9]).all() and (z_coef == 0 or o["loss"][1].isnan())
    else:
        assert (np.abs(d[9] - ref[9]) <= bound[9]).all() and o["loss"][1] == 0


@pytest.mark.parametrize("T,E,k,S", [(700, 64, 4, 9), (3000, 256, 8, 3), (513, 200, 3, 40)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_balance_replayed_on_other_sequences(score, T, E, k, S):
    rng = np.random.default_rng(T)
    ctx = binding.Context(T, 64, 64, E, k)
    sets = []
    for spread in (3.0, 60.0, 0.1):
        x, ids, offsets, mask = case(rng, T, E, k, S, True, spread)
        sets.append([x, ids, np.asarray(offsets, np.int32), mask])
    sets[1][2] = np.array([0] * (S - 1) + [T // 2, T], np.int32)         # all in the last two sequences
    sets[2][2] = np.array([0] + [1] * (S - 1) + [T - 3], np.int32)       # the first has one token, some come behind the last
    sets[2][3] = np.zeros(T, np.uint8)
    sets[2][3][[0, T // 3]] = 1
    sets.append([sets[0][0], np.zeros((T, k), np.int32) + np.arange(k, dtype=np.int32), sets[0][2], np.ones(T, np.uint8)])
    x, ids, offsets, mask = (dev(v) for v in sets[0])
    how = dict(score=score, coef=0.2, z_coef=0.01, sequences=S)
    scratch = torch.empty(ctx.balance_scratch_bytes(S), dtype=torch.uint8, device=DEV)
    o = dict(counts=torch.empty(S, E, dtype=torch.int32, device=DEV), tokens=torch.empty(S + 1, dtype=torch.int32, device=DEV),
             mean=torch.empty(S, E, device=DEV), loss=torch.empty(2, device=DEV))
    d, graph = torch.empty(T, E, device=DEV), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        ctx.moe_balance_loss(x, ids, o["counts"], o["tokens"], o["mean"], o["loss"], scratch, seq_offsets=offsets, token_mask=mask,
                             **how)
        ctx.moe_balance_loss_backward(x, o["counts"], o["tokens"], d, seq_offsets=offsets, token_mask=mask, **how)
    for new in sets + sets[::-1]:
        for to, v in zip((x, ids, offsets, mask), new):
            to.copy_(dev(v))
        graph.replay()
        torch.cuda.synchronize()
        want = run_loss(ctx, dev(new[0]), dev(new[1]), seq_offsets=dev(new[2]), token_mask=dev(new[3]), **how)
        grad = torch.empty(T, E, device=DEV)
        ctx.moe_balance_loss_backward(dev(new[0]), want["counts"], want["tokens"], grad, seq_offsets=dev(new[2]),
                                      token_mask=dev(new[3]), **how)
        assert all(torch.equal(o[n], want[n]) for n in o) and torch.equal(d, grad)
        counts, tokens, _, loss = ao.balance_loss(new[0], new[1], score, 0.2, 0.01, new[2], new[3], S)
        assert np.array_equal(o["counts"].cpu().numpy(), counts) and np.array_equal(o["tokens"].cpu().numpy(), tokens)
    assert ctx.moe_last_device_status() == (0, 0)


# ------------------------------------------------------------------------------------------------------------ adapters
@pytest.mark.parametrize("kernel,rows,segments", [("rows", 60, 60), ("rows", 900, 12), ("tiles", 900, 12)])
def test_adapters_replayed_on_other_segments(kernel, rows, segments):
    ctx, adapters = context(kernel), 12
    p, rng = ga.make(rows, rows, 520, 776, 24, adapters)
    single = segments == rows
    splits = [None] * 4 if single else [ga.cut(rng, rows, segments), [0] * 11 + [rows - 5, rows],
                                        [0, 850] + list(range(851, 862)), list(range(12)) + [rows]]
    picks = [rng.integers(-1, adapters, segments), np.full(segments, 3), np.arange(segments) % adapters, np.full(segments, -1)]
    idd, off = ga.i32(picks[0]), ga.i32(splits[0])
    x, y, out = p["x"].clone(), p["y"].clone(), torch.empty_like(p["y"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        ctx.moe_add_adapters(x, p["a"], p["b"], idd, y, out, None, rows, 520, 776, 24, adapters, segments, offsets=off,
                             scale=p["scale"])
    for i, (bounds, ids) in enumerate(zip(splits + splits[::-1], picks + picks[::-1])):
        p["x"], p["xv"] = bf16(rng.standard_normal((rows, 776)))
        x.copy_(p["x"])
        idd.copy_(ga.i32(ids))
        if not single:
            off.copy_(ga.i32(bounds))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        ga.check(p, ids, bounds, out)
        assert torch.equal(out.view(torch.int16), ga.run(ctx, p, ids, bounds).view(torch.int16))
    assert ctx.moe_last_device_status() == (0, 0)
