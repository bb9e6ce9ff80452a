"""The operators around the expert layer run together, as a block of a model would: norm, projection with adapters, norm, router,
experts, and back: balance loss, gradients of gate and norm.

Each step is held to the oracle on the values that the step before left on the device (its own file has the bounds); the
gradient of the whole is held to autograd in 64 bits, the choice of experts held fixed."""
import numpy as np
import pytest
import torch

from oracle import around_oracle as ao
from oracle import blk_oracle as blk
from paper_2607_23264_b200 import binding, inputs as gen
from moe_testlib import DEV, bits_to_dev, dev_bf16_to_f64

pytestmark = pytest.mark.gpu
T, H, F, E, K, RANK, ADAPTERS = 200, 256, 128, 16, 4, 16, 3
U = 2.0 ** -24


class Block:
    def __init__(self):
        self.ctx = binding.Context(T, H, F, E, K)
        rng = np.random.default_rng(0)
        bf = lambda v: bits_to_dev(gen.f32_to_bf16_bits(np.asarray(v, np.float32)))  # noqa: E731
        bt = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
        i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device=DEV)  # noqa: E731
        self.x, self.res = bf(rng.standard_normal((T, H))), bf(2 * rng.standard_normal((T, H)))
        self.g1, self.g2 = bf(1 + 0.2 * rng.standard_normal(H)), torch.from_numpy((1 + 0.2 * rng.standard_normal(H)).astype(np.float32)).to(DEV)
        self.a, self.b = bf(rng.standard_normal((ADAPTERS, RANK, H)) / 16), bf(rng.standard_normal((ADAPTERS, H, RANK)) / 8)
        self.offsets = torch.tensor([0, 90, 91, 92, 170, 200], dtype=torch.int32, device=DEV)
        self.who = torch.tensor([0, 2, -1, 1, 0], dtype=torch.int32, device=DEV)
        self.router = torch.from_numpy((rng.standard_normal((H, E)) / 16).astype(np.float32)).to(DEV)
        self.rule = binding.make_route_rule("sigmoid", n_group=4, topk_group=2, group_top=2, weight_scale=2.0)
        self.weights = []
        for mats, rows, cols in ((1, H, H), (E, F, H), (E, F, H), (E, H, F)):
            w = bf(rng.standard_normal((mats, rows, cols)) / np.sqrt(cols))
            codes = torch.empty(mats, rows, cols, dtype=torch.uint8, device=DEV)
            scales = torch.empty(mats, rows // 128, cols // 128, device=DEV)
            self.ctx.moe_quantize_weights_blk(w, mats, rows, cols, codes, scales)
            self.weights += [codes, scales]
        R, u8, f32 = T * K, dict(dtype=torch.uint8, device=DEV), dict(device=DEV)
        self.s1, self.n1, self.y, self.s2, self.n2, self.out = (bt(T, H) for _ in range(6))
        self.c1, self.c2 = torch.empty(T, H, **u8), torch.empty(T, H, **u8)
        self.f1, self.f2 = torch.empty(H // 128, T, **f32), torch.empty(H // 128, T, **f32)
        self.scratch = torch.empty(max(16, self.ctx.adapter_scratch_bytes(T, H, RANK)), **u8)
        self.ids, self.w, self.counts, self.off = i32(T, K), torch.empty(T, K, **f32), i32(E), i32(E + 1)
        self.perm, self.inv = i32(R), i32(R)
        self.xp, self.sxp = torch.empty(R, H, **u8), torch.empty(H // 128, R, **f32)
        self.hq, self.sh, self.yp = torch.empty(R, F, **u8), torch.empty(F // 128, R, **f32), bt(R, H)
        self.bc, self.tok, self.mean, self.loss = i32(1, E), i32(2), torch.empty(1, E, **f32), torch.empty(2, **f32)
        self.bscratch = torch.empty(self.ctx.balance_scratch_bytes(1), **u8)
        self.d_out = bf(rng.standard_normal((T, H)) / 16)
        self.d_w, self.d_logits = torch.empty(T, K, **f32), torch.empty(T, E, **f32)
        self.d_s2, self.d_g2 = bt(T, H), torch.empty(H, **f32)
        self.nscratch = torch.empty(self.ctx.rms_norm_scratch_bytes(T, H), **u8)

    def forward(self):
        c = self.ctx
        c.moe_add_rms_norm(self.x, self.res, self.g1, T, H, sum_out=self.s1, out=self.n1, codes=self.c1, scales=self.f1, form="blk")
        c.moe_gemm_blk(self.c1, self.f1, self.weights[0], self.weights[1], self.y, T, H, H)
        self.projected = self.y.clone()
        c.moe_add_adapters(self.n1, self.a, self.b, self.who, self.y, self.y, self.scratch, T, H, H, RANK, ADAPTERS, 5,
                           offsets=self.offsets)
        c.moe_add_rms_norm(self.y, self.s1, self.g2, T, H, sum_out=self.s2, out=self.n2, codes=self.c2, scales=self.f2, form="blk")
        self.logits = self.n2.float() @ self.router
        c.moe_plan_routing_scored(self.logits, None, self.rule, self.ids, self.w, self.counts, self.off, self.perm, self.inv)
        c.moe_dispatch_blk(self.c2, self.f2, self.inv, self.xp, self.sxp)
        c.moe_expert_ffn_blk(self.xp, self.sxp, self.off, *self.weights[2:], self.hq, self.sh, self.yp)
        c.moe_combine(self.yp, self.inv, self.w, self.out)

    def backward(self):
        c = self.ctx
        c.moe_balance_loss(self.logits, self.ids, self.bc, self.tok, self.mean, self.loss, self.bscratch, score="sigmoid", coef=0.5,
                           z_coef=0.01)
        c.moe_combine_backward(self.d_out, self.yp, self.inv, self.w, None, self.d_w)
        c.moe_routing_backward(self.logits, self.ids, self.d_w, self.rule, self.d_logits)
        c.moe_balance_loss_backward(self.logits, self.bc, self.tok, self.d_logits, add=self.d_logits, score="sigmoid", coef=0.5,
                                    z_coef=0.01)
        self.d_n2 = (self.d_logits @ self.router.t()).to(torch.bfloat16)
        c.moe_rms_norm_backward(self.s2, self.g2, self.d_n2, T, H, self.d_s2, self.d_g2, self.nscratch)

    def results(self):
        return [self.out, self.w, self.loss, self.d_logits, self.d_s2, self.d_g2]


def test_each_step_against_the_oracle():
    b = Block()
    b.forward()
    b.backward()
    torch.cuda.synchronize()
    assert b.ctx.moe_last_device_status() == (0, 0)
    f64 = lambda t: dev_bf16_to_f64(t) if t.dtype == torch.bfloat16 else t.cpu().numpy().astype(np.float64)  # noqa: E731
    s1 = ao.residual_sum(f64(b.x), f64(b.res))
    n1 = ao.rms_norm(s1, f64(b.g1), 1e-6)
    assert np.array_equal(f64(b.s1), s1) and (np.abs(f64(b.n1) - n1) <= (2.0 ** -8 + 30 * U) * np.abs(n1)).all()
    codes, scales = b.c1.cpu().numpy(), b.f1.cpu().numpy()
    wc, ws = b.weights[0][0].cpu().numpy(), b.weights[1][0].cpu().numpy()
    y = blk.gemm(codes, scales, wc, ws)
    size = blk.magnitude(codes, scales, wc, ws)
    assert (np.abs(f64(b.projected) - y) <= 2.0 ** -8 * np.abs(y) + (H / 16 + 10) * 2 * U * size).all()
    y, st, sy = ao.add_adapters(f64(b.n1), f64(b.a), f64(b.b), None, b.who.tolist(), f64(b.projected), b.offsets.tolist())
    assert (np.abs(f64(b.y) - y) <= 2.0 ** -8 * np.abs(y) + (H / 16 + 64) * U * st + (2.0 ** -16 + 24 * U) * sy).all()
    s2 = ao.residual_sum(f64(b.y), f64(b.s1))
    assert np.array_equal(f64(b.s2), s2)
    counts, tokens, mean, loss = ao.balance_loss(f64(b.logits), b.ids.cpu().numpy(), "sigmoid", 0.5, 0.01)
    assert np.array_equal(b.bc.cpu().numpy(), counts) and np.array_equal(b.bc[0].cpu().numpy(), b.counts.cpu().numpy())
    assert np.abs(f64(b.loss) - loss).max() <= 1e-5 * np.abs(loss).max()
    # the whole gradient of the last norm's input: through logits, weights and losses, by autograd in 64 bits
    s = torch.from_numpy(s2).requires_grad_(True)
    gain = b.g2.cpu().double().requires_grad_(True)
    n = s / torch.sqrt(s.square().mean(1, keepdim=True) + 1e-6) * gain
    logits = n @ b.router.cpu().double()
    ids = b.ids.cpu().long()
    p = torch.sigmoid(logits)
    w = p.gather(1, ids)
    w = 2.0 * w / w.sum(1, keepdim=True)
    rows = b.yp.cpu().double()[b.inv.cpu().long()].view(T, K, H)
    value = (torch.einsum("tk,tkh->th", w, rows) * b.d_out.cpu().double()).sum()
    q = p / p.sum(1, keepdim=True)
    value = value + 0.5 * (E * torch.from_numpy(counts[0]).double() / (K * T) * q.mean(0)).sum()
    value = value + 0.01 * torch.logsumexp(logits, 1).square().mean()
    want_s, want_g = torch.autograd.grad(value, (s, gain))
    # bf16 roundings on the way: n2 (2^-9 a value, on average of both signs) into the logits, d_n2 and d_s2
    for got, want in ((b.d_s2, want_s), (b.d_g2, want_g)):
        assert np.linalg.norm(f64(got) - want.numpy()) <= 1e-2 * np.linalg.norm(want.numpy())


def test_the_fused_layer_answers_like_the_separate_calls():
    """The layer's one call on the bf16 rows against the steps from the norm's own codes (quantised from fp32, not from bf16): both
    are within the 8-bit form's error of the same layer."""
    b = Block()
    b.forward()
    ws = torch.empty(b.ctx.workspace_layout_blk()["total"], dtype=torch.uint8, device=DEV)
    out = torch.empty_like(b.out)
    b.ctx.moe_fused_forward_blk(b.n2, b.logits, None, b.rule, *b.weights[2:], out, ws)
    torch.cuda.synchronize()
    a, c = dev_bf16_to_f64(out), dev_bf16_to_f64(b.out)
    assert np.linalg.norm(a - c) <= 2.0 ** -4 * np.linalg.norm(a)


def test_captured_and_replayed():
    b = Block()
    b.forward()
    b.backward()
    torch.cuda.synchronize()
    want = [t.clone() for t in b.results()]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        b.forward()
        b.backward()
    for _ in range(3):
        for t in b.results():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(b.results(), want))
