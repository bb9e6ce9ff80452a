"""FP8 in blocks of 128 on the GPU against the oracle.

Codes and scales are fp32 decisions on both sides: compared bit for bit.  Products are compared on identical operands:
the bf16 rounding (2^-8 of the value at most) and fp32 sums (one rounding per 32-deep instruction, one for aligning its
products, one per block: (K/16 + K/128 + 8) 2^-23 of the sum of magnitudes).  The layer is compared element by element
on the GPU's own h codes, and in norm against the independent oracle, where a last-bit difference in h can move a code."""
import numpy as np
import pytest
import torch

from oracle import blk_oracle as blk
from oracle import moe_oracle as orc
from oracle import scored_router_oracle as sro
from oracle.scored_router_oracle import Rule
from paper_2607_23264_b200 import binding, inputs as gen
from moe_testlib import DEV, TOL_FRO, Layer, assert_out_close, bits_to_dev, dev_bf16_to_f64, rel_fro

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(1, 64, 64, 1, 1)


def spread(rng, rows, cols):
    return (rng.standard_normal((rows, cols)) * np.exp(rng.uniform(-8, 8, (rows, 1)))).astype(np.float32)


@pytest.mark.parametrize("rows,cols", [(1, 16), (1, 128), (7, 144), (37, 256), (300, 1040), (5, 7168), (1001, 112)])
def test_quantize_rows_bits(ctx, rows, cols):
    rng = np.random.default_rng(rows + cols)
    v = spread(rng, rows, cols)
    v[0, :128] = 0.0
    if rows > 2:
        v[2, :16] = 448.0 * 2.0 ** rng.integers(-5, 5, 16)
    bits = gen.f32_to_bf16_bits(v)
    nb = -(-cols // 128)
    codes = torch.full((rows, cols), 0x7F, dtype=torch.uint8, device=DEV)
    scales = torch.full((nb, rows), float("nan"), device=DEV)
    ctx.moe_quantize_rows_blk(bits_to_dev(bits), rows, cols, codes, scales)
    torch.cuda.synchronize()
    ref_c, ref_s = blk.quantize_rows(gen.bf16_bits_to_f32(bits))
    assert np.array_equal(scales.cpu().numpy(), ref_s)
    assert np.array_equal(codes.cpu().numpy(), ref_c)


@pytest.mark.parametrize("mats,rows,cols", [(1, 1, 16), (2, 128, 128), (3, 136, 272), (1, 1000, 1040), (5, 64, 384)])
def test_quantize_weights_bits(ctx, mats, rows, cols):
    rng = np.random.default_rng(rows + cols)
    v = np.stack([spread(rng, rows, cols) for _ in range(mats)])
    v[0, :128, :128] = 0.0
    bits = gen.f32_to_bf16_bits(v)
    codes = torch.full((mats, rows, cols), 0x7F, dtype=torch.uint8, device=DEV)
    scales = torch.full((mats, -(-rows // 128), -(-cols // 128)), float("nan"), device=DEV)
    ctx.moe_quantize_weights_blk(bits_to_dev(bits), mats, rows, cols, codes, scales)
    torch.cuda.synchronize()
    for m in range(mats):
        ref_c, ref_s = blk.quantize_weights(gen.bf16_bits_to_f32(bits[m]))
        assert np.array_equal(scales[m].cpu().numpy(), ref_s)
        assert np.array_equal(codes[m].cpu().numpy(), ref_c)


def test_quantize_keeps_the_sign_of_zero(ctx):
    v = np.tile(np.array([-0.0, 0.0, 1.0, -1e-30], dtype=np.float32), (128, 32))
    codes = torch.full((128, 128), 0x7F, dtype=torch.uint8, device=DEV)
    scales = torch.zeros(1, 128, device=DEV)
    x = bits_to_dev(gen.f32_to_bf16_bits(v))
    ctx.moe_quantize_rows_blk(x, 128, 128, codes, scales)
    torch.cuda.synchronize()
    assert np.array_equal(codes.cpu().numpy(), blk.quantize_rows(v)[0])
    ctx.moe_quantize_weights_blk(x, 1, 128, 128, codes, scales)
    torch.cuda.synchronize()
    assert np.array_equal(codes.cpu().numpy(), blk.quantize_weights(v)[0])


def test_quantize_keeps_nan_and_infinity_visible(ctx):
    v = np.ones((2, 256), dtype=np.float32)
    v[0, 3], v[0, 130], v[1, 255] = np.nan, np.inf, -np.inf
    x = torch.from_numpy(v).to(torch.bfloat16).to(DEV)
    codes = torch.zeros(2, 256, dtype=torch.uint8, device=DEV)
    scales = torch.zeros(2, 2, device=DEV)
    ctx.moe_quantize_rows_blk(x, 2, 256, codes, scales)
    torch.cuda.synchronize()
    back = codes.view(torch.float8_e4m3fn).float().cpu() * scales.t().cpu().repeat_interleave(128, 1)
    assert bool(back[0, 3].isnan()) and torch.equal(back[0, :3], torch.ones(3)) and torch.equal(back[1, :128], torch.ones(128))
    assert not back[0, 128:].isfinite().any() and not back[1, 128:].isfinite().any()


def make_product(rng, counts, N, K, tail=0):
    """Random operands of a grouped product: (a codes, sa, offsets, [b codes], [sb])."""
    rows = int(sum(counts)) + tail
    a, sa = blk.quantize_rows(spread(rng, max(rows, 1), K))
    b = [blk.quantize_weights((rng.standard_normal((N, K)) * np.exp(rng.uniform(-2, 2))).astype(np.float32)) for _ in counts]
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    return a, sa, offsets, b


def run_product(ctx, a, sa, offsets, b, N, K, use_offsets=True, stream=None):
    rows, G = a.shape[0], len(b)
    y = torch.full((rows, N), float("nan"), dtype=torch.bfloat16, device=DEV)
    args = (dev(a), dev(sa), dev(np.stack([c for c, _ in b])), dev(np.stack([s for _, s in b])))
    off = dev(offsets)
    torch.cuda.synchronize()
    ctx.moe_gemm_blk(*args, y, rows, N, K, groups=G, offsets=off if use_offsets else None, stream=stream)
    torch.cuda.synchronize()
    assert ctx.moe_last_device_status()[0] == 0
    return y


def check_product(y, a, sa, offsets, b, N, K):
    got = dev_bf16_to_f64(y)
    assert np.isnan(got[offsets[-1]:]).all(), "rows outside every group were written"
    for g, (bc, bs) in enumerate(b):
        lo, hi = offsets[g], offsets[g + 1]
        if hi == lo:
            continue
        ref = blk.gemm(a[lo:hi], sa[:, lo:hi], bc, bs)
        mag = blk.magnitude(a[lo:hi], sa[:, lo:hi], bc, bs)
        bound = 2.0 ** -8 * np.abs(ref) + (K / 16 + K / 128 + 8) * 2.0 ** -23 * mag
        err = np.abs(got[lo:hi] - ref)
        assert (err <= bound).all(), (g, np.nanmax(err / bound))


@pytest.mark.parametrize("counts,N,K", [
    ([1], 8, 16), ([1], 128, 128), ([17], 136, 144), ([64], 256, 256), ([65], 264, 272), ([128], 1024, 384),
    ([129], 520, 1040), ([200], 384, 640), ([257], 256, 2048), ([700], 512, 512), ([1], 4096, 7168), ([33], 2104, 4112),
    ([0, 1, 0, 5, 16], 136, 256), ([3, 0, 40, 130, 0, 64], 264, 400), ([17, 15, 48, 49, 96, 97, 112, 113], 128, 128),
    ([300, 2, 0, 270], 640, 1152), ([1] * 200, 64, 128), ([0] * 9 + [2] + [0] * 1000, 72, 128),
    ([20] * 700, 8, 16), ([193] * 660, 8, 16), ([128, 140, 64, 65, 66, 129], 520, 784), ([1025, 900, 1], 264, 272),
    ([1025, 1300], 264, 272), ([2000], 520, 1040),
])
def test_product(ctx, counts, N, K):
    rng = np.random.default_rng(N + K + len(counts))
    a, sa, offsets, b = make_product(rng, counts, N, K, tail=3 if len(counts) > 1 else 0)
    y = run_product(ctx, a, sa, offsets, b, N, K)
    check_product(y, a, sa, offsets, b, N, K)
    if len(counts) == 1:
        assert torch.equal(run_product(ctx, a, sa, offsets, b, N, K, use_offsets=False).view(torch.int16), y.view(torch.int16))
    again = run_product(ctx, a, sa, offsets, b, N, K, stream=torch.cuda.Stream())
    assert torch.equal(again.view(torch.int16), y.view(torch.int16)), "not the same bits on another stream"


@pytest.mark.parametrize("knobs", ["x.blk_pair_rows=0", "x.blk_pair_rows=1073741824,x.blk_few_rows=0",
                                   "x.blk_pair_rows=1073741824,x.blk_few_rows=1073741824"])
@pytest.mark.parametrize("counts,N,K", [
    ([1, 0, 31, 33, 64, 65], 136, 144), ([127, 128, 129, 255, 256, 257], 264, 1040), ([513], 1032, 2064),
    ([1300, 1100], 520, 400),
])
def test_product_by_every_kind_of_tile(monkeypatch, knobs, counts, N, K):
    """The tile is chosen by the average rows per group; each kind has to be right for every group all the same."""
    monkeypatch.setenv("MOE_TUNING", knobs)
    forced = binding.Context(1, 64, 64, 1, 1)
    rng = np.random.default_rng(N + K)
    a, sa, offsets, b = make_product(rng, counts, N, K, tail=2)
    check_product(run_product(forced, a, sa, offsets, b, N, K), a, sa, offsets, b, N, K)


def test_product_random_shapes(ctx):
    rng = np.random.default_rng(21)
    for trial in range(24):
        G = int(rng.integers(1, 9)) if trial % 2 else 1
        counts = [int(rng.integers(0, 2) * np.exp(rng.uniform(0, 6))) for _ in range(G)]
        if not sum(counts):
            counts[0] = 1 + trial
        N, K = 8 * int(np.exp(rng.uniform(0, 5))), 16 * int(np.exp(rng.uniform(0, 5)))
        a, sa, offsets, b = make_product(rng, counts, N, K)
        check_product(run_product(ctx, a, sa, offsets, b, N, K), a, sa, offsets, b, N, K)


def test_product_scales_of_all_sizes(ctx):
    """Scales far apart between blocks: the running sum must not lose the small ones to a common exponent."""
    rng = np.random.default_rng(8)
    N, K, M = 128, 512, 40
    a, sa, offsets, b = make_product(rng, [M], N, K)
    sa *= np.array([2.0 ** -60, 1.0, 2.0 ** 40, 2.0 ** -20], dtype=np.float32)[:, None]
    sb = b[0][1] * np.array([2.0 ** 50, 1.0, 2.0 ** -50, 2.0 ** 10], dtype=np.float32)
    b = [(b[0][0], sb)]
    check_product(run_product(ctx, a, sa, offsets, b, N, K), a, sa, offsets, b, N, K)


def test_nan_rows_stay_in_their_rows(ctx):
    rng = np.random.default_rng(12)
    a, sa, offsets, b = make_product(rng, [20, 30], 128, 256)
    a[7, 5], a[25, 200] = 0x7F, 0xFF
    y = dev_bf16_to_f64(run_product(ctx, a, sa, offsets, b, 128, 256))
    bad = np.isnan(y).all(axis=1)
    assert list(np.flatnonzero(bad)) == [7, 25] and np.isfinite(np.delete(y, [7, 25], axis=0)).all()


def test_input_gradient_is_the_product_with_transposed_weights(ctx):
    """d_a = d_y . b is the same call on the transposed codes and scales; against differences of the fp64 product."""
    rng = np.random.default_rng(30)
    N, K, M = 256, 384, 20
    (bc, bs) = blk.quantize_weights(rng.standard_normal((N, K)).astype(np.float32))
    g, sg = blk.quantize_rows(rng.standard_normal((M, N)).astype(np.float32))
    off = np.array([0, M], dtype=np.int32)
    bt = [(np.ascontiguousarray(bc.T), np.ascontiguousarray(bs.T))]
    y = run_product(ctx, g, sg, off, bt, K, N)
    check_product(y, g, sg, off, bt, K, N)
    w, gv = blk.dequantize_weights(bc, bs), blk.dequantize_rows(g, sg)
    x = rng.standard_normal((M, K))
    got = dev_bf16_to_f64(y)
    for r, c in ((0, 0), (3, 200), (19, 383)):
        e = np.zeros((M, K))
        e[r, c] = 1e-3
        diff = (((x + e) @ w.T * gv).sum() - ((x - e) @ w.T * gv).sum()) / 2e-3
        assert abs(diff - got[r, c]) <= 2.0 ** -8 * abs(diff) + 1e-3


def test_product_refusals(ctx):
    t8, t4 = torch.zeros(4096, dtype=torch.uint8, device=DEV), torch.zeros(64, device=DEV)
    y = torch.zeros(256, dtype=torch.bfloat16, device=DEV)
    off = torch.zeros(8, dtype=torch.int32, device=DEV)

    def call(a=t8, sa=t4, b=t8, sb=t4, y=y, rows=2, N=16, K=32, groups=1, offsets=None):
        ctx.moe_gemm_blk(a, sa, b, sb, y, rows, N, K, groups=groups, offsets=offsets)

    call()
    call(rows=0)
    for bad, code in ((dict(N=12), 2), (dict(K=24), 2), (dict(N=0), 2), (dict(K=0), 2), (dict(rows=-1), 2),
                      (dict(groups=0), 2), (dict(groups=1025, offsets=off), 2), (dict(rows=1 << 30), 2),
                      (dict(groups=2), 1), (dict(a=None), 1), (dict(sb=None), 1), (dict(y=None), 1),
                      (dict(a=t8[1:2049]), 1), (dict(sa=t4[1:33]), 1), (dict(offsets=off[1:3], groups=1), 1)):
        with pytest.raises(binding.MoeError) as e:
            call(**bad)
        assert e.value.code == code, bad
    for f in (lambda: ctx.moe_quantize_rows_blk(y, 1, 24, t8, t4), lambda: ctx.moe_quantize_rows_blk(y, -1, 16, t8, t4),
              lambda: ctx.moe_quantize_rows_blk(None, 1, 16, t8, t4), lambda: ctx.moe_quantize_weights_blk(y, 1, 1, 8, t8, t4),
              lambda: ctx.moe_quantize_weights_blk(y, -1, 1, 16, t8, t4)):
        with pytest.raises(binding.MoeError) as e:
            f()
        assert e.value.code == 1
    odd = binding.Context(4, 192, 128, 2, 1)                 # H is not a multiple of 128
    with pytest.raises(binding.MoeError) as e:
        odd.workspace_layout_blk()
    assert e.value.code == 2
    for f in (lambda: odd.moe_dispatch_blk(t8, t4, off, t8, t4),
              lambda: odd.moe_expert_ffn_blk(*[t8] * 12),
              lambda: odd.moe_fused_forward_blk(t8, t4, None, binding.make_route_rule(), *[t8] * 6, y, t8)):
        with pytest.raises(binding.MoeError) as e:
            f()
        assert e.value.code == 2
    small = binding.Context(4, 128, 128, 2, 1)
    with pytest.raises(binding.MoeError) as e:
        small.moe_fused_forward_blk(t8, t4, None, binding.make_route_rule(), *[t8] * 6, y, t8[:256])
    assert e.value.code == 3
    with pytest.raises(binding.MoeError) as e:
        small.moe_fused_forward_blk(t8, t4, None, binding.make_route_rule(n_group=3), *[t8] * 6, y, t8)
    assert e.value.code == 1


class BlkLayer:
    """A layer whose weights are quantised on the GPU, with the oracle's own quantisation beside it."""

    def __init__(self, cfg, x_bits=None):
        self.cfg = cfg
        self.L = Layer(cfg, x_bits=x_bits)
        L, E, F, H = self.L, cfg.E, cfg.F, cfg.H
        self.q = {}
        for name, t, rows, cols in (("gate", L.w_gate, F, H), ("up", L.w_up, F, H), ("down", L.w_down, H, F)):
            codes = torch.full((E, rows, cols), 0x7F, dtype=torch.uint8, device=DEV)
            scales = torch.full((E, rows // 128, cols // 128), float("nan"), device=DEV)
            L.ctx.moe_quantize_weights_blk(t, E, rows, cols, codes, scales)
            self.q[name] = (codes, scales)
        torch.cuda.synchronize()
        self._wq = {}

    def weights(self):
        return [t for n in ("gate", "up", "down") for t in self.q[n]]

    def oracle_weights(self, e):
        if e not in self._wq:
            self._wq[e] = [blk.quantize_weights(gen.bf16_bits_to_f32(w)) for w in self.L.weights(e)]
        return self._wq[e]


def cfg_of(T, H, F, E, k, seed, router="xWr"):
    return gen.MoEConfig(name="blk", T=T, H=H, F=F, E=E, k=k, seed=seed, router=router)


@pytest.mark.parametrize("T,H,F,E,k,router", [
    (64, 128, 128, 4, 2, "xWr"),
    (300, 512, 384, 8, 2, "xWr"),
    (129, 256, 640, 16, 4, "xWr_zipf"),
    (5, 384, 256, 6, 6, "xWr"),
    (1, 256, 128, 3, 1, "xWr"),
    (70, 128, 128, 1024, 32, "xWr"),
    (700, 256, 384, 2, 2, "xWr"),
    (600, 384, 256, 8, 2, "xWr"),
    (256, 256, 384, 3, 2, "xWr"),
    (1900, 256, 384, 2, 2, "xWr"),
    (2300, 128, 256, 4, 2, "xWr"),
])
def test_expert_ffn_parity(T, H, F, E, k, router):
    cfg = cfg_of(T, H, F, E, k, seed=T + H, router=router)
    M = BlkLayer(cfg)
    L, ctx = M.L, M.L.ctx
    L.plan()
    R = cfg.R
    xq = torch.full((T, H), 0x7F, dtype=torch.uint8, device=DEV)
    sx = torch.full((H // 128, T), float("nan"), device=DEV)
    ctx.moe_quantize_rows_blk(L.x, T, H, xq, sx)
    xq_perm = torch.full((R, H), 0x7F, dtype=torch.uint8, device=DEV)
    sx_perm = torch.full((H // 128, R), float("nan"), device=DEV)
    ctx.moe_dispatch_blk(xq, sx, L.inv_perm, xq_perm, sx_perm)
    torch.cuda.synchronize()
    ref_c, ref_s = blk.quantize_rows(gen.bf16_bits_to_f32(L.x_bits))
    tok = L.perm.cpu().numpy().astype(np.int64) // k
    assert np.array_equal(xq_perm.cpu().numpy(), ref_c[tok]) and np.array_equal(sx_perm.cpu().numpy(), ref_s[:, tok])
    for e in (0, E - 1):
        for (c, s), name in zip(M.oracle_weights(e), ("gate", "up", "down")):
            assert np.array_equal(M.q[name][0][e].cpu().numpy(), c) and np.array_equal(M.q[name][1][e].cpu().numpy(), s)
    hq = torch.full((R, F), 0x7F, dtype=torch.uint8, device=DEV)
    sh = torch.full((F // 128, R), float("nan"), device=DEV)
    y = L.nan_bf16(R, H)
    h_dbg = torch.full((R, F), float("nan"), device=DEV)
    ctx.moe_expert_ffn_blk(xq_perm, sx_perm, L.offsets, *M.weights(), hq, sh, y, h_dbg)
    torch.cuda.synchronize()
    L.check_device_status()
    offsets = L.offsets.cpu().numpy()
    xc, xs = ref_c[tok], ref_s[:, tok]
    h_gpu = h_dbg.cpu().numpy()
    assert np.isfinite(h_gpu).all()
    # h's codes and scales are the oracle's quantisation of the GPU's own fp32 h
    req_c, req_s = blk.quantize_rows(h_gpu)
    assert np.array_equal(hq.cpu().numpy(), req_c) and np.array_equal(sh.cpu().numpy(), req_s)
    y_gpu = dev_bf16_to_f64(y)
    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        if hi == lo:
            continue
        gate, up, down = M.oracle_weights(e)
        h_ref = blk.expert_rows(xc[lo:hi], xs[:, lo:hi], gate, up)
        assert rel_fro(h_gpu[lo:hi].astype(np.float64), h_ref) <= TOL_FRO / 50, e
        ref = blk.gemm(req_c[lo:hi], req_s[:, lo:hi], *down)
        mag = blk.magnitude(req_c[lo:hi], req_s[:, lo:hi], *down)
        assert (np.abs(y_gpu[lo:hi] - ref) <= 2.0 ** -8 * np.abs(ref) + (F / 16 + F / 128 + 8) * 2.0 ** -23 * mag).all(), e


def check_fused(M, rule, bias, ws, out, tokens, samples=40):
    """out of a fused call against the oracle on the GPU's own h codes, and in norm against the independent oracle."""
    cfg, L, ctx = M.cfg, M.L, M.L.ctx
    H, F, E, k = cfg.H, cfg.F, cfg.E, cfg.k
    lay = ctx.workspace_layout_blk()
    R = tokens * k
    part = lambda n, count, kind: ws[lay[n]:lay[n] + 4 * count].view(kind).cpu().numpy()  # noqa: E731
    ids, w = part("topk_ids", R, torch.int32).reshape(tokens, k), part("topk_w", R, torch.float32).reshape(tokens, k)
    inv = part("inv_perm", R, torch.int32)
    ref_ids, _ = sro.route(L.logits[:tokens], bias, rule, k)
    assert (ids == ref_ids).all(1).mean() >= 0.97
    counts, offsets, perm, inv_ref = orc.plan_permutation(ids, E)
    assert np.array_equal(inv, inv_ref)
    hq = ws[lay["hq"]:lay["hq"] + R * F].view(R, F).cpu().numpy()
    sh = part("sh", F // 128 * R, torch.float32).reshape(F // 128, R)
    toks = np.unique(np.linspace(0, tokens - 1, min(tokens, samples)).astype(int))
    xc, xs = blk.quantize_rows(gen.bf16_bits_to_f32(L.x_bits[toks]))
    own, free = np.zeros((len(toks), H)), np.zeros((len(toks), H))
    for i, t in enumerate(toks):
        for j in range(k):
            gate, up, down = M.oracle_weights(int(ids[t, j]))
            row = int(inv[t * k + j])
            own[i] += w[t, j] * blk.gemm(hq[row:row + 1], sh[:, row:row + 1], *down)[0]
            hc, hs = blk.quantize_rows(blk.expert_rows(xc[i:i + 1], xs[:, i:i + 1], gate, up))
            free[i] += w[t, j] * blk.gemm(hc, hs, *down)[0]
    got = dev_bf16_to_f64(out)[toks]
    assert np.isfinite(got).all()
    assert_out_close(got, own, f"out, {tokens} tokens, on the GPU's h codes")
    if tokens >= 33:
        assert rel_fro(got, free) <= 2e-2


def test_fused_forward_and_smaller_batches():
    cfg = cfg_of(300, 384, 256, 16, 4, seed=31)
    M = BlkLayer(cfg)
    L, ctx = M.L, M.L.ctx
    rule = Rule("sigmoid", 4, 2, 2, True, 2.5)
    r = binding.make_route_rule("sigmoid", 4, 2, 2, True, 2.5)
    bias = (np.arange(cfg.E) % 5 / 32).astype(np.float32)
    d_bias = dev(bias)
    ws = torch.empty(ctx.workspace_layout_blk()["total"], dtype=torch.uint8, device=DEV)
    for tokens in (300, 33, 1, 0):
        ctx.moe_set_active_tokens(tokens)
        out = L.nan_bf16(max(tokens, 1), cfg.H)
        x, logits = L.x[:max(tokens, 1)].contiguous(), L.d_logits[:max(tokens, 1)].contiguous()
        ctx.moe_fused_forward_blk(x, logits, d_bias, r, *M.weights(), out, ws)
        torch.cuda.synchronize()
        L.check_device_status()
        if tokens == 0:
            assert ctx.moe_last_launch_count() == 0
            continue
        check_fused(M, rule, bias, ws, out, tokens)
        again = L.nan_bf16(tokens, cfg.H)
        ctx.moe_fused_forward_blk(x, logits, d_bias, r, *M.weights(), again, ws, stream=torch.cuda.Stream())
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), again.view(torch.int16))


def test_fused_forward_long_k_loops():
    # K loops of 32 and 11 blocks, 11 column tiles of Linear-1, hundreds of rows per expert
    cfg = cfg_of(1024, 4096, 1408, 2, 2, seed=9)
    M = BlkLayer(cfg)
    L, ctx = M.L, M.L.ctx
    ws = torch.empty(ctx.workspace_layout_blk()["total"], dtype=torch.uint8, device=DEV)
    out = L.nan_bf16(cfg.T, cfg.H)
    ctx.moe_fused_forward_blk(L.x, L.d_logits, None, binding.make_route_rule(), *M.weights(), out, ws)
    torch.cuda.synchronize()
    L.check_device_status()
    check_fused(M, Rule(), None, ws, out, cfg.T, samples=16)


def test_fused_forward_of_a_token_with_every_expert_masked_is_zero():
    cfg = cfg_of(40, 128, 128, 8, 2, seed=3)
    M = BlkLayer(cfg)
    L, ctx = M.L, M.L.ctx
    logits = L.d_logits.clone()
    logits[7] = -float("inf")
    ws = torch.empty(ctx.workspace_layout_blk()["total"], dtype=torch.uint8, device=DEV)
    out, ref = L.nan_bf16(cfg.T, cfg.H), L.nan_bf16(cfg.T, cfg.H)
    rule = binding.make_route_rule("sigmoid")
    ctx.moe_fused_forward_blk(L.x, L.d_logits, None, rule, *M.weights(), ref, ws)
    ctx.moe_fused_forward_blk(L.x, logits, None, rule, *M.weights(), out, ws)
    torch.cuda.synchronize()
    L.check_device_status()
    assert out[7].eq(0).all()
    keep = [t for t in range(cfg.T) if t != 7]
    assert torch.equal(out[keep].view(torch.int16), ref[keep].view(torch.int16))


def test_router_tuning_example_learns():
    """The example runs every new call as a training loop would: 20 steps take the loss clearly down."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tune_router.py")
    spec = importlib.util.spec_from_file_location("tune_router", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.main(["--steps", "20"])
    assert losses[-1] < 0.9 * losses[0]


def test_layer_equals_its_separate_calls():
    """moe_fused_forward_blk gives the bits of plan, quantise, dispatch, experts and combine called one by one."""
    cfg = cfg_of(200, 512, 256, 16, 3, seed=44)
    M = BlkLayer(cfg)
    L, ctx = M.L, M.L.ctx
    T, H, F, R = cfg.T, cfg.H, cfg.F, cfg.R
    rule = binding.make_route_rule("sigmoid", 4, 3, 1, True, 1.5)
    bias = dev((np.arange(cfg.E) % 3 / 16).astype(np.float32))
    ws = torch.empty(ctx.workspace_layout_blk()["total"], dtype=torch.uint8, device=DEV)
    fused, apart = L.nan_bf16(T, H), L.nan_bf16(T, H)
    ctx.moe_fused_forward_blk(L.x, L.d_logits, bias, rule, *M.weights(), fused, ws)
    assert ctx.moe_last_launch_count() in (5, 7)
    ctx.moe_plan_routing_scored(L.d_logits, bias, rule, L.topk_ids, L.topk_w, L.counts, L.offsets, L.perm, L.inv_perm)
    u8 = dict(dtype=torch.uint8, device=DEV)
    xq, sx, xp, sxp = torch.empty(T, H, **u8), torch.empty(H // 128, T, device=DEV), torch.empty(R, H, **u8), torch.empty(H // 128, R, device=DEV)
    hq, sh, y = torch.empty(R, F, **u8), torch.empty(F // 128, R, device=DEV), L.nan_bf16(R, H)
    ctx.moe_quantize_rows_blk(L.x, T, H, xq, sx)
    ctx.moe_dispatch_blk(xq, sx, L.inv_perm, xp, sxp)
    ctx.moe_expert_ffn_blk(xp, sxp, L.offsets, *M.weights(), hq, sh, y)
    ctx.moe_combine(y, L.inv_perm, L.topk_w, apart)
    torch.cuda.synchronize()
    L.check_device_status()
    assert torch.equal(fused.view(torch.int16), apart.view(torch.int16))
    lay = ctx.workspace_layout_blk()
    assert torch.equal(ws[lay["xq_perm"]:lay["xq_perm"] + R * H], xp.view(-1))
    assert torch.equal(ws[lay["sx_perm"]:lay["sx_perm"] + 4 * R * (H // 128)].view(torch.float32), sxp.view(-1))


def test_calls_can_be_captured_in_a_graph():
    cfg = cfg_of(48, 256, 128, 8, 2, seed=45)
    M = BlkLayer(cfg)
    L, ctx = M.L, M.L.ctx
    rule = binding.make_route_rule("softmax")
    ws = torch.empty(ctx.workspace_layout_blk()["total"], dtype=torch.uint8, device=DEV)
    eager, out = L.nan_bf16(cfg.T, cfg.H), L.nan_bf16(cfg.T, cfg.H)
    ctx.moe_fused_forward_blk(L.x, L.d_logits, None, rule, *M.weights(), eager, ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            ctx.moe_fused_forward_blk(L.x, L.d_logits, None, rule, *M.weights(), out, ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), eager.view(torch.int16))


@pytest.mark.parametrize("N,K", [(128, 16), (128, 128), (264, 256), (520, 272), (136, 240), (384, 144)])
def test_product_of_mixed_tiles_with_few_blocks_of_k(ctx, N, K):
    """Hundreds of groups of 1 to 128 rows: every CTA goes from tiles with the rows on the M side (65 to 128 rows) to tiles
    with swapped operands and back, and with one or two blocks of K its warps may be a tile apart."""
    rng = np.random.default_rng(N + K)
    counts = [int(c) for c in rng.integers(1, 129, 600)]
    a, sa, offsets, b = make_product(rng, counts, N, K)
    y = run_product(ctx, a, sa, offsets, b, N, K)
    check_product(y, a, sa, offsets, b, N, K)
    for _ in range(5):
        again = run_product(ctx, a, sa, offsets, b, N, K)
        assert torch.equal(again.view(torch.int16), y.view(torch.int16)), "not the same bits every time"


@pytest.mark.parametrize("H,F", [(128, 256), (256, 128), (256, 256)])
def test_experts_of_mixed_tiles_with_few_blocks_of_k(H, F):
    """The same through both GEMMs of a layer: 400 experts with loads from about 12 to 130 rows."""
    cfg = cfg_of(6000, H, F, 400, 4, seed=H + F)
    M = BlkLayer(cfg)
    L, ctx = M.L, M.L.ctx
    L.plan()
    R = cfg.R
    xq, sx = torch.empty(cfg.T, H, dtype=torch.uint8, device=DEV), torch.empty(H // 128, cfg.T, device=DEV)
    xp, sxp = torch.empty(R, H, dtype=torch.uint8, device=DEV), torch.empty(H // 128, R, device=DEV)
    ctx.moe_quantize_rows_blk(L.x, cfg.T, H, xq, sx)
    ctx.moe_dispatch_blk(xq, sx, L.inv_perm, xp, sxp)
    counts = L.counts.cpu().numpy()
    assert ((counts > 0) & (counts <= 64)).sum() > 100 and (counts > 64).sum() > 100     # both kinds of tile
    hq = torch.full((R, F), 0x7F, dtype=torch.uint8, device=DEV)
    sh = torch.full((F // 128, R), float("nan"), device=DEV)
    y, h = L.nan_bf16(R, H), torch.full((R, F), float("nan"), device=DEV)
    ctx.moe_expert_ffn_blk(xp, sxp, L.offsets, *M.weights(), hq, sh, y, h)
    torch.cuda.synchronize()
    L.check_device_status()
    offsets, xc, xs = L.offsets.cpu().numpy(), xp.cpu().numpy(), sxp.cpu().numpy()
    h_gpu, hc, hs, y_gpu = h.cpu().numpy(), hq.cpu().numpy(), sh.cpu().numpy(), dev_bf16_to_f64(y)
    req_c, req_s = blk.quantize_rows(h_gpu)
    assert np.array_equal(hc, req_c) and np.array_equal(hs, req_s)
    for e in range(cfg.E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        if hi == lo:
            continue
        gate, up, down = M.oracle_weights(e)
        assert rel_fro(h_gpu[lo:hi].astype(np.float64), blk.expert_rows(xc[lo:hi], xs[:, lo:hi], gate, up)) <= TOL_FRO / 50, e
        ref, mag = blk.gemm(hc[lo:hi], hs[:, lo:hi], *down), blk.magnitude(hc[lo:hi], hs[:, lo:hi], *down)
        assert (np.abs(y_gpu[lo:hi] - ref) <= 2.0 ** -8 * np.abs(ref) + (F / 16 + F / 128 + 8) * 2.0 ** -23 * mag).all(), e


LONGEST = 2 ** 31 - 16               # the last multiple of 16 an int32 holds


def test_quantize_the_longest_row(ctx):
    """One row of 2^31 - 16 values: a period of 2^20 over and over, so that the codes are those of one short call."""
    period = 1 << 20
    g = torch.Generator(device=DEV).manual_seed(3)
    part = torch.randn(period, generator=g, device=DEV).to(torch.bfloat16)
    x = part.repeat(LONGEST // period + 1)[:LONGEST]
    codes, scales = torch.empty(LONGEST, dtype=torch.uint8, device=DEV), torch.empty(1 << 24, device=DEV)
    small_c, small_s = torch.empty(period, dtype=torch.uint8, device=DEV), torch.empty(period // 128, device=DEV)
    ctx.moe_quantize_rows_blk(part, 1, period, small_c, small_s)
    whole = LONGEST // period * period
    tail_c, tail_s = torch.empty(LONGEST - whole, dtype=torch.uint8, device=DEV), torch.empty(period // 128, device=DEV)
    ctx.moe_quantize_rows_blk(part, 1, LONGEST - whole, tail_c, tail_s)
    # as a matrix of one row too: its blocks of 128 x 128 are the same 128 values
    for call in (lambda: ctx.moe_quantize_rows_blk(x, 1, LONGEST, codes, scales),
                 lambda: ctx.moe_quantize_weights_blk(x, 1, 1, LONGEST, codes, scales)):
        codes.fill_(0x7F)
        scales.fill_(float("nan"))
        call()
        torch.cuda.synchronize()
        assert bool((codes[:whole].view(-1, period) == small_c).all()) and torch.equal(codes[whole:], tail_c)
        assert bool((scales[:whole // 128].view(-1, period // 128) == small_s).all())
        assert torch.equal(scales[whole // 128:], tail_s)
    del x, codes, scales
    torch.cuda.empty_cache()


def test_product_with_the_longest_k(ctx):
    """K = 2^31 - 16: ones in a few places of a against small whole numbers in b, first block, middle and short last one."""
    N = 8
    a = torch.zeros(1, LONGEST, dtype=torch.uint8, device=DEV)
    b = torch.full((N, LONGEST), 0x38, dtype=torch.uint8, device=DEV)                       # 1.0
    where = torch.tensor([0, 5, 127, 128, 2 ** 30 + 1, 2 ** 31 - 129, 2 ** 31 - 128, LONGEST - 1], device=DEV)
    a[0, where] = 0x38
    b[:, LONGEST - 1] = torch.arange(N, device=DEV).float().to(torch.float8_e4m3fn).view(torch.uint8)
    y = torch.full((1, N), float("nan"), dtype=torch.bfloat16, device=DEV)
    ones = torch.ones(1 << 24, device=DEV)
    ctx.moe_gemm_blk(a, ones, b, ones, y, 1, N, LONGEST)
    torch.cuda.synchronize()
    assert ctx.moe_last_device_status()[0] == 0
    assert y[0].tolist() == [7.0 + n for n in range(N)]
    del a, b, ones
    torch.cuda.empty_cache()


def test_more_blocks_than_a_grid_holds_are_refused(ctx):
    t8, t4 = torch.zeros(4096, dtype=torch.uint8, device=DEV), torch.zeros(64, device=DEV)
    for mats, rows, cols in ((1 << 29, 2 ** 31 - 1, LONGEST), (1 << 29, 2 ** 30, 2 ** 24), (1, 2 ** 31 - 1, LONGEST)):
        with pytest.raises(binding.MoeError) as e:
            ctx.moe_quantize_weights_blk(t8, mats, rows, cols, t8, t4)
        assert e.value.code == 5, (mats, rows, cols)


def product_and_kernel(ctx, *args):
    """y of run_product, and the name of the kernel that it launched (None where no launch can be recorded here)."""
    from torch.profiler import ProfilerActivity, profile
    with profile(activities=[ProfilerActivity.CUDA], acc_events=True) as seen:
        y = run_product(ctx, *args)
    names = [e.name for e in seen.events()]
    mine = [n for n in names if "gemm_blk" in n]
    assert len(mine) == 1 or not names, names
    return y, mine[0] if mine else None


def assert_pair_kernel(name):
    if name is None:
        pytest.skip("the result is right; which kernel computed it could not be recorded")
    assert "<false, 2, 128>" in name.replace("(bool)0", "false").replace("(int)", ""), name


# ragged and empty groups; second weight boxes beyond N and beyond the last group, K that ends inside a block, last tiles of
# 1 to 128 rows (the peer CTA has none) and of 129 to 255
PAIR_SHAPES = [([1, 0, 31, 33, 64, 65], 136, 144), ([127, 128, 129, 255, 256, 257, 0], 264, 1040), ([513], 1032, 2064),
               ([1300, 1100], 520, 400), ([0, 385, 0, 0, 640, 2], 904, 1168), ([1], 8, 16), ([300], 136, 4112),
               ([5] * 300, 264, 272), ([200] * 150, 392, 144), ([0, 0, 769], 2056, 528)]


@pytest.mark.parametrize("counts,N,K", PAIR_SHAPES)
def test_product_by_pairs_of_ctas(monkeypatch, counts, N, K):
    """The pair kernel on shapes that the rule gives to other kernels as well as on its own."""
    monkeypatch.setenv("MOE_TUNING", "x.blk_pair_rows=0")
    forced = binding.Context(1, 64, 64, 1, 1)
    rng = np.random.default_rng(N + K + len(counts))
    a, sa, offsets, b = make_product(rng, counts, N, K, tail=2)
    y, kernel = product_and_kernel(forced, a, sa, offsets, b, N, K)
    check_product(y, a, sa, offsets, b, N, K)
    assert_pair_kernel(kernel)


@pytest.mark.parametrize("counts,N,K", [([1100, 901, 0, 1700], 136, 112), ([3333], 264, 128), ([2000, 2100, 1, 1900], 5128, 272)])
def test_product_by_pairs_without_being_forced(ctx, counts, N, K):
    """More than 900 rows a group on average, and K that a split cannot shorten or more tiles than SMs."""
    rng = np.random.default_rng(N + K)
    a, sa, offsets, b = make_product(rng, counts, N, K)
    y, kernel = product_and_kernel(ctx, a, sa, offsets, b, N, K)
    check_product(y, a, sa, offsets, b, N, K)
    assert_pair_kernel(kernel)


@pytest.mark.parametrize("T,H,F,E,k", [(300, 384, 256, 6, 2), (513, 256, 384, 2, 1), (40, 512, 128, 12, 3)])
def test_experts_by_pairs_of_ctas(monkeypatch, T, H, F, E, k):
    """Both GEMMs of a layer by the pair kernel: the bits of h's codes, and y on them."""
    monkeypatch.setenv("MOE_TUNING", "x.blk_pair_rows=0")
    test_expert_ffn_parity(T, H, F, E, k, "xWr")


@pytest.mark.parametrize("E", [1, 20])
def test_silu_in_the_epilogue_to_a_few_ulp(E):
    """h = silu(g) u with g = u = the row's scale (codes of 1 in one place), so that h is the epilogue's arithmetic alone.
    expf 2 ulp, reciprocal 1, a sum and two products half each: 4.5 ulp of 2^-23 at most."""
    T, H, F = 640, 128, 128
    ctx = binding.Context(T, H, F, E, 1)
    sx = np.concatenate([np.linspace(-86, 86, T - 2), [0.0, 300.0]]).astype(np.float32)
    one = 0x38
    xq = torch.zeros(T, H, dtype=torch.uint8, device=DEV)
    xq[:, 0] = one
    w = torch.zeros(E, F, H, dtype=torch.uint8, device=DEV)
    w[:, :, 0] = one
    ws = torch.ones(E, 1, 1, device=DEV)
    offsets = torch.tensor([T * e // E for e in range(E + 1)], dtype=torch.int32, device=DEV)
    hq, sh = torch.empty(T, F, dtype=torch.uint8, device=DEV), torch.empty(1, T, device=DEV)
    y, h = torch.empty(T, H, dtype=torch.bfloat16, device=DEV), torch.full((T, F), float("nan"), device=DEV)
    ctx.moe_expert_ffn_blk(xq, dev(sx[None]), offsets, w, ws, w, ws, w, ws, hq, sh, y, h)
    torch.cuda.synchronize()
    assert ctx.moe_last_device_status()[0] == 0
    g = sx.astype(np.float64)
    ref = (g * g / (1 + np.exp(-g)))[:, None]
    err = np.abs(h.cpu().numpy() - ref)
    assert (err <= 4.5 * 2.0 ** -23 * np.abs(ref)).all(), np.max(err[ref[:, 0] != 0] / np.abs(ref[ref[:, 0] != 0]) * 2 ** 23)
