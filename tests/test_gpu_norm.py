"""Residual addition, RMS norm and its 8-bit outputs on the GPU against the oracle, and the norm's gradients.

Bounds, counted in roundings of 2^-24: a row's sum of squares adds 32 values per lane, five levels in a warp and five over
warps (positive terms: at most 45 of its value), the root halves that, and the mean, the root, the two products and the gain's
offset add one each: n is within 30 of its value.  A bf16 output adds half a step, 2^-8 of the value.  A scale is n's largest
magnitude over 448 (one more).  A code is within half an E4M3 step, 2^-4 of the value or 2^-10 of the scale, and the fp32
errors of n and of the scale (64 together) decide ties.  Gradients: the sum of g h adds another 45 of the magnitudes in it, and the
formula ten: 80 of rstd (|g| + |h| mean|g h|) + |d_sum|.  d_gain adds rows in order: (rows per CTA + CTAs / 8 + 50) of sum|d h|."""
import numpy as np
import pytest
import torch

from oracle import around_oracle as ao
from oracle import blk_oracle as blk
from oracle import fp8_oracle as f8
from oracle import mx_oracle as mx
from paper_2607_23264_b200 import binding, inputs as gen
from moe_testlib import DEV, bits_to_dev, dev_bf16_to_f64

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-6


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(1, 64, 64, 1, 1)


def bf16(v):
    """A bf16 tensor and its values."""
    bits = gen.f32_to_bf16_bits(np.asarray(v, np.float32))
    return bits_to_dev(bits), gen.bf16_bits_to_f32(bits).astype(np.float64)


def make(rng, rows, cols, gain="bf16"):
    x, xv = bf16(rng.standard_normal((rows, cols)) * np.exp(rng.uniform(-6, 6, (rows, 1))))
    r, rv = bf16(rng.standard_normal((rows, cols)) * np.exp(rng.uniform(-6, 6, (rows, 1))))
    gv = 1 + 0.3 * rng.standard_normal(cols)
    if gain == "bf16":
        g, gv = bf16(gv)
    else:
        gv = gv.astype(np.float32)
        g = torch.from_numpy(gv).to(DEV)
    return x, xv, r, rv, g, gv.astype(np.float64)


def outputs(rows, cols, form, extra=0):
    """Poisoned outputs, `extra` rows longer than needed."""
    o = {n: torch.full((rows + extra, cols), float("nan"), dtype=torch.bfloat16, device=DEV) for n in ("sum_out", "out")}
    if form != "none":
        o["codes"] = torch.full((rows + extra, cols), 0x7F, dtype=torch.uint8, device=DEV)
        shape = {"rows": (rows,), "blk": (-(-cols // 128), rows), "mx": (cols // 128, rows)}[form]
        o["scales"] = torch.full(shape, -1, dtype=torch.int32, device=DEV)
        if form != "mx":
            o["scales"] = o["scales"].view(torch.float32)
    return o


def check_codes(o, n, form):
    rows, cols = n.shape
    codes = o["codes"][:rows].cpu().numpy()
    if form == "mx":
        bytes_ = o["scales"].cpu().numpy().view(np.uint8).reshape(cols // 128, rows, 4).transpose(1, 0, 2).reshape(rows, cols // 32)
        amax = np.abs(n).reshape(rows, cols // 32, 32).max(2)
        for edge in (1 - 64 * U, 1 + 64 * U):                  # the fp32 amax lies between
            e = mx.block_exponents(np.repeat((amax * edge).astype(np.float32), 32, axis=1)) + 127
            assert (bytes_ <= e).all() if edge > 1 else (bytes_ >= e).all()
        scale = np.repeat(2.0 ** (bytes_.astype(np.float64) - 127), 32, axis=1)
    elif form == "rows":
        s = o["scales"].cpu().numpy().astype(np.float64)
        want = np.abs(n).max(1) / 448
        assert (np.abs(s - np.where(want > 0, want, 1)) <= 64 * U * s).all()
        scale = s[:, None]
    else:
        s = o["scales"].cpu().numpy().astype(np.float64)
        want = np.stack([np.abs(n[:, lo:lo + 128]).max(1) for lo in range(0, cols, 128)]) / 448
        assert (np.abs(s - np.where(want > 0, want, 1)) <= 64 * U * s).all()
        scale = np.repeat(s, 128, axis=0)[:cols].T
    err = np.abs(f8.e4m3_decode(codes) * scale - n)
    assert (err <= np.maximum(2.0 ** -4 * np.abs(n), 2.0 ** -10 * scale) * (1 + 2.0 ** -17) + 64 * U * np.abs(n)).all()


SIZES = [(1, 8, "none"), (1, 16, "blk"), (3, 24, "rows"), (3, 128, "mx"), (37, 144, "blk"), (1, 7168, "blk"), (64, 7168, "blk"),
         (65, 7168, "rows"), (300, 1040, "blk"), (1001, 2048, "mx"), (9, 4096, "mx"), (7, 8200, "none"), (130, 4104, "rows"),
         (513, 1024, "mx"), (700, 528, "blk"), (2, 32768, "rows"), (3, 32768, "mx"), (5, 16400, "blk"), (2000, 256, "rows")]


@pytest.mark.parametrize("rows,cols,form", SIZES)
@pytest.mark.parametrize("residual,gain,offset", [(True, "bf16", 0.0), (False, "fp32", 1.0)])
def test_norm_against_oracle(ctx, rows, cols, form, residual, gain, offset):
    rng = np.random.default_rng(rows * 7 + cols)
    x, xv, r, rv, g, gv = make(rng, rows, cols, gain)
    if rows > 2:
        x[1] = 0
        r[1] = 0
        xv[1] = rv[1] = 0
    o = outputs(rows, cols, form, extra=2)
    ctx.moe_add_rms_norm(x, r if residual else None, g, rows, cols, form=form, eps=EPS, gain_offset=offset, **o)
    torch.cuda.synchronize()
    assert ctx.moe_last_launch_count() == 1
    s = ao.residual_sum(xv, rv if residual else None)
    n = ao.rms_norm(s, gv, EPS, offset)
    assert np.array_equal(dev_bf16_to_f64(o["sum_out"][:rows]), s)
    got = dev_bf16_to_f64(o["out"][:rows])
    assert (np.abs(got - n) <= (2.0 ** -8 + 30 * U) * np.abs(n) + 2.0 ** -134).all()
    if form != "none":
        check_codes(o, n, form)
        assert (o["codes"][rows:] == 0x7F).all()
    assert o["out"][rows:].isnan().all() and o["sum_out"][rows:].isnan().all()


@pytest.mark.parametrize("form", ["rows", "mx", "blk"])
def test_each_output_alone_and_in_place(ctx, form):
    rng = np.random.default_rng(5)
    rows, cols = 41, 1152
    x, _, r, _, g, _ = make(rng, rows, cols)
    whole = outputs(rows, cols, form)
    ctx.moe_add_rms_norm(x, r, g, rows, cols, form=form, **whole)
    for keep in (("sum_out",), ("out",), ("codes", "scales")):
        o = {n: t for n, t in outputs(rows, cols, form).items() if n in keep}
        ctx.moe_add_rms_norm(x, r, g, rows, cols, form=form if "codes" in keep else "none", **o)
        for n in keep:
            assert torch.equal(o[n].view(torch.uint8), whole[n].view(torch.uint8)), n
    # the stream replaces the residual, the normalised rows replace x
    x2, r2 = x.clone(), r.clone()
    o = outputs(rows, cols, form)
    ctx.moe_add_rms_norm(x2, r2, g, rows, cols, sum_out=r2, out=x2, codes=o["codes"], scales=o["scales"], form=form)
    assert torch.equal(r2, whole["sum_out"]) and torch.equal(x2, whole["out"]) and torch.equal(o["codes"], whole["codes"])


def test_codes_agree_with_the_quantisation_calls_where_bf16_holds_the_norm(ctx):
    """Rows whose norm is exact in bf16: the fused codes and scales are those of the separate calls, bit for bit."""
    rng = np.random.default_rng(6)
    rows, cols = 33, 512
    s = rng.choice([-1.0, 1.0], (rows, cols))
    x, _ = bf16(s)
    g, gv = bf16(rng.standard_normal(cols))
    n = torch.from_numpy(s * gv).to(torch.bfloat16).to(DEV)
    for form, call in (("rows", ctx.moe_quantize_rows), ("mx", ctx.moe_quantize_rows_mx), ("blk", ctx.moe_quantize_rows_blk)):
        a, b = outputs(rows, cols, form), outputs(rows, cols, form)
        ctx.moe_add_rms_norm(x, None, g, rows, cols, form=form, eps=1e-12, **a)      # mean 1: rstd is exactly 1
        call(n, rows, cols, b["codes"], b["scales"])
        torch.cuda.synchronize()
        assert torch.equal(a["out"], n)
        assert torch.equal(a["codes"], b["codes"]) and torch.equal(a["scales"].view(torch.int32), b["scales"].view(torch.int32))


def test_values_that_are_not_numbers_stay_in_their_row(ctx):
    rows, cols = 6, 256
    rng = np.random.default_rng(7)
    x, _, _, _, g, _ = make(rng, rows, cols)
    x[1, 3], x[2, 200], x[3, 0] = float("nan"), float("inf"), -float("inf")
    x[4] = 1e30                                                # sum of squares beyond fp32
    clean = x.clone()
    clean[1:5] = 1
    a, b = outputs(rows, cols, "blk"), outputs(rows, cols, "blk")
    ctx.moe_add_rms_norm(x, None, g, rows, cols, form="blk", **a)
    ctx.moe_add_rms_norm(clean, None, g, rows, cols, form="blk", **b)
    torch.cuda.synchronize()
    assert a["out"][1].isnan().all() and a["out"][2, 200].isnan() and a["out"][3, 0].isnan() and (a["out"][4] == 0).all()
    for r in (0, 5):
        assert torch.equal(a["out"][r], b["out"][r]) and torch.equal(a["codes"][r], b["codes"][r])
    assert (a["codes"][1] & 0x7F == 0x7F).all() and (a["codes"][4] & 0x7F == 0).all()


def test_rows_behind_the_32nd_bit(ctx):
    """2^32 bytes lie between the first and the last rows."""
    rows, cols = 300_000, 8192
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    g, gv = bf16(np.linspace(0.5, 2, cols))
    last, lv = bf16(np.random.default_rng(8).standard_normal((2, cols)))
    x[-2:] = last
    codes, scales = torch.empty(rows, cols, dtype=torch.uint8, device=DEV), torch.empty(64, rows, device=DEV)
    ctx.moe_add_rms_norm(x, None, g, rows, cols, out=x, codes=codes, scales=scales, form="blk")
    n = ao.rms_norm(lv, gv, EPS)
    assert (np.abs(dev_bf16_to_f64(x[-2:]) - n) <= (2.0 ** -8 + 30 * U) * np.abs(n)).all()
    check_codes({"codes": codes[-2:], "scales": scales[:, -2:].contiguous()}, n, "blk")
    assert (x[:-2] == 0).all() and (scales[:, :-2] == 1).all()


def run_backward(ctx, s, g, d, e, rows, cols, eps=EPS, offset=0.0, stream=None, want=("dx", "dg")):
    dx = torch.full((rows, cols), float("nan"), dtype=torch.bfloat16, device=DEV) if "dx" in want else None
    dg = torch.full((cols,), float("nan"), device=DEV) if "dg" in want else None
    scratch = torch.full((max(16, ctx.rms_norm_scratch_bytes(rows, cols)),), 0xFF, dtype=torch.uint8, device=DEV)
    ctx.moe_rms_norm_backward(s, g, d, rows, cols, dx, dg, scratch if dg is not None else None, d_sum=e, eps=eps,
                              gain_offset=offset, stream=stream)
    return dx, dg


@pytest.mark.parametrize("rows,cols", [(1, 8), (1, 7168), (3, 24), (37, 144), (301, 7168), (2500, 1024), (1000, 2056), (777, 4096),
                                       (64, 520), (5, 32768), (700, 16384), (4001, 256)])
@pytest.mark.parametrize("with_sum,gain,offset", [(True, "bf16", 0.0), (False, "fp32", 1.0)])
def test_gradients_against_oracle(ctx, rows, cols, with_sum, gain, offset):
    rng = np.random.default_rng(rows + cols)
    s, sv, e, ev, g, gv = make(rng, rows, cols, gain)
    d, dv = bf16(rng.standard_normal((rows, cols)) * np.exp(rng.uniform(-3, 3, (rows, 1))))
    if rows > 2:
        s[1], sv[1] = 0, 0
    dx, dg = run_backward(ctx, s, g, d, e if with_sum else None, rows, cols, offset=offset)
    rx, rg, size_x, size_g = ao.rms_norm_backward(sv, gv, dv, ev if with_sum else None, EPS, offset)
    assert (np.abs(dev_bf16_to_f64(dx) - rx) <= 2.0 ** -8 * np.abs(rx) + 80 * U * size_x + 2.0 ** -134).all()
    ctas = ctx.rms_norm_scratch_bytes(rows, cols) // (4 * cols)
    steps = -(-rows // ctas) + ctas / 8 + 50
    assert (np.abs(dg.cpu().numpy() - rg) <= steps * U * size_g + 1e-38).all()


def test_gradients_one_at_a_time_in_place_and_repeated(ctx):
    rng = np.random.default_rng(9)
    rows, cols = 401, 1544
    s, _, e, _, g, _ = make(rng, rows, cols)
    d, _ = bf16(rng.standard_normal((rows, cols)))
    dx, dg = run_backward(ctx, s, g, d, e, rows, cols)
    for _ in range(3):
        x2, g2 = run_backward(ctx, s, g, d, e, rows, cols)
        assert torch.equal(x2, dx) and torch.equal(g2, dg)
    assert torch.equal(run_backward(ctx, s, g, d, e, rows, cols, want=("dx",))[0], dx)
    assert torch.equal(run_backward(ctx, s, g, d, e, rows, cols, want=("dg",))[1], dg)
    for into in ("d", "e"):
        d2, e2 = d.clone(), e.clone()
        ctx.moe_rms_norm_backward(s, g, d2, rows, cols, d2 if into == "d" else e2, None, d_sum=e2)
        assert torch.equal(d2 if into == "d" else e2, dx)
    zero = torch.full((cols,), float("nan"), device=DEV)
    ctx.moe_rms_norm_backward(None, g, None, 0, cols, None, zero)
    assert (zero == 0).all()


def test_gradient_of_the_call_against_differences(ctx):
    """The forward's own outputs: d_x against the change of sum(out * d) for a step in x that bf16 holds."""
    rng = np.random.default_rng(10)
    rows, cols = 4, 64
    xv = rng.choice([-1.5, -1.0, -0.5, 0.5, 1.0, 1.5], (rows, cols))
    g = torch.ones(cols, device=DEV)
    d, dv = bf16(rng.standard_normal((rows, cols)))
    x, _ = bf16(xv)
    dx, _ = run_backward(ctx, x, g, d, None, rows, cols)
    for c in (0, 17, 63):
        n = []
        for step in (0.125, -0.125):
            v = xv.copy()
            v[:, c] += step
            y, _ = bf16(v)
            o = outputs(rows, cols, "none")
            ctx.moe_add_rms_norm(y, None, g, rows, cols, out=o["out"])
            n.append((dev_bf16_to_f64(o["out"]) * dv).sum(1))
        # bf16 outputs: each product is off by 2^-8 of itself; the third derivative of n along one of 64 columns is below 1
        size = 2.0 ** -8 * np.abs(dv * 2.5).sum(1) * 2 / 0.25 + 0.125 ** 2 * np.abs(dv).sum(1)
        assert (np.abs((n[0] - n[1]) / 0.25 - dev_bf16_to_f64(dx)[:, c]) <= size).all()


def test_other_stream_and_graph_replay(ctx):
    rng = np.random.default_rng(11)
    rows, cols = 96, 1024
    x, _, r, _, g, _ = make(rng, rows, cols)
    d, _ = bf16(rng.standard_normal((rows, cols)))
    want = outputs(rows, cols, "blk")
    ctx.moe_add_rms_norm(x, r, g, rows, cols, form="blk", **want)
    wx, wg = run_backward(ctx, want["sum_out"], g, d, r, rows, cols)
    torch.cuda.synchronize()
    o, dx, dg = outputs(rows, cols, "blk"), torch.empty_like(wx), torch.empty_like(wg)
    scratch = torch.empty(ctx.rms_norm_scratch_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ctx.moe_add_rms_norm(x, r, g, rows, cols, form="blk", **o)
        ctx.moe_rms_norm_backward(o["sum_out"], g, d, rows, cols, dx, dg, scratch, d_sum=r)
    for _ in range(3):
        for t in (*o.values(), dx, dg):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o[n].view(torch.uint8), want[n].view(torch.uint8)) for n in o)
        assert torch.equal(dx, wx) and torch.equal(dg, wg)


@pytest.mark.parametrize("change,code", [
    (dict(cols=12), 2), (dict(cols=0), 2), (dict(cols=32776), 2), (dict(rows=-1), 2), (dict(rows=1 << 30), 2),
    (dict(cols=136, form="mx"), 2), (dict(cols=136, form="blk"), 2), (dict(eps=0.0), 1), (dict(eps=float("inf")), 1),
    (dict(eps=float("nan")), 1), (dict(gain_offset=float("nan")), 1), (dict(x=None), 1), (dict(codes=None), 1),
    (dict(scales=None), 1), (dict(form="none"), 1), (dict(same=True), 1), (dict(odd="x"), 1), (dict(odd="out"), 1),
    (dict(nothing=True), 1)])
def test_refusals_of_the_norm(ctx, change, code):
    rows, cols = 4, 256
    buf = torch.zeros(rows * cols + 64, dtype=torch.bfloat16, device=DEV)
    a = dict(x=buf[:rows * cols].view(rows, cols), residual=None, gain=torch.ones(cols, device=DEV), rows=rows, cols=cols,
             eps=1e-6, gain_offset=0.0, **outputs(rows, cols, "blk"), form="blk")
    change = dict(change)
    if change.pop("same", False):
        a["sum_out"] = a["out"]
    if change.pop("nothing", False):
        a.update(sum_out=None, out=None, codes=None, scales=None, form="none")
    odd = change.pop("odd", None)
    if odd:
        a[odd] = buf[1:rows * cols + 1].view(rows, cols)
    a.update(change)
    with pytest.raises(binding.MoeError) as err:
        ctx.moe_add_rms_norm(**a)
    assert err.value.code == code and ctx.moe_last_launch_count() == 0


def test_refusals_of_the_gradient(ctx):
    rows, cols = 4, 256
    t = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    g, dg = torch.ones(cols, device=DEV), torch.zeros(cols, device=DEV)
    scratch = torch.zeros(ctx.rms_norm_scratch_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    for args, kw, code in [((None, g, t, rows, cols, t, dg, scratch), {}, 1), ((t, g, None, rows, cols, t, dg, scratch), {}, 1),
                           ((t, g, t, rows, cols, None, None, scratch), {}, 1), ((t, g, t, rows, cols, t, dg, None), {}, 1),
                           ((t, g, t, rows, cols, t, dg, scratch[:-16]), {}, 3), ((t, g, t, rows, 12, t, dg, scratch), {}, 2),
                           ((t, g, t, rows, cols, t, dg, scratch), dict(eps=0.0), 1)]:
        with pytest.raises(binding.MoeError) as err:
            ctx.moe_rms_norm_backward(*args, **kw)
        assert err.value.code == code
    with pytest.raises(ValueError):
        ctx.moe_add_rms_norm(t[:, ::2], None, g, rows, cols // 2, out=t)
    assert ctx.rms_norm_scratch_bytes(1, 4) == 0 and ctx.rms_norm_scratch_bytes(-1, 8) == 0


@pytest.mark.parametrize("rows,cols", [(2500, 1032), (450, 7168), (20011, 128), (1203, 4104), (445, 6152), (1300, 2048)])
@pytest.mark.parametrize("gain,offset", [("bf16", 0.0), ("fp32", 1.0)])
def test_more_rows_than_are_resident_without_residual_and_codes(ctx, rows, cols, gain, offset):
    rng = np.random.default_rng(rows + cols)
    x, xv, _, _, g, gv = make(rng, rows, cols, gain)
    x[1], xv[1] = 0, 0
    x[rows // 2, 3] = float("nan")                             # spoils its own row, and none that the CTA takes before or after
    o = outputs(rows, cols, "none", extra=2)
    ctx.moe_add_rms_norm(x, None, g, rows, cols, eps=EPS, gain_offset=offset, **o)
    torch.cuda.synchronize()
    assert ctx.moe_last_launch_count() == 1
    n = ao.rms_norm(xv, gv, EPS, offset)
    keep = np.arange(rows) != rows // 2
    got = dev_bf16_to_f64(o["out"][:rows])
    assert np.isnan(got[~keep]).all()
    assert (np.abs(got - n) <= (2.0 ** -8 + 30 * U) * np.abs(n) + 2.0 ** -134)[keep].all()
    assert torch.equal(o["sum_out"][:rows].view(torch.int16), x.view(torch.int16))
    assert o["out"][rows:].isnan().all() and o["sum_out"][rows:].isnan().all()
    again = x.clone()                                          # in place, the same bits
    ctx.moe_add_rms_norm(again, None, g, rows, cols, out=again, eps=EPS, gain_offset=offset)
    assert torch.equal(again.view(torch.int16), o["out"][:rows].view(torch.int16))
