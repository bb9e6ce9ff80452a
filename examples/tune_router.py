"""Tunes the router of a fine-grained MoE layer whose experts are frozen in FP8 blocks of 128.

The layer's inputs come from a frozen dense projection in the same form.  A teacher router defines the target outputs; a
student router starts from another matrix and is trained on the mean squared error, step by step with the library's calls:
scored plan, quantise, dispatch, experts, combine, then the gradient of the combine (to the weights) and of the scores (to
the logits).  The router matrix itself, its product with x and the update are plain torch.  The balance bias moves towards
even loads, as it does in training.  The tuned router then answers through the fused layer, as it would be served.

    python examples/tune_router.py [--steps 40]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_23264_b200 import binding  # noqa: E402


def frozen_matrix(ctx, mats, rows, cols, g):
    """Random matrices in blocks of 128: codes and scales."""
    w = (torch.randn(mats, rows, cols, generator=g, device="cuda") / cols ** 0.5).to(torch.bfloat16)
    codes = torch.empty(mats, rows, cols, dtype=torch.uint8, device="cuda")
    scales = torch.empty(mats, rows // 128, cols // 128, device="cuda")
    ctx.moe_quantize_weights_blk(w, mats, rows, cols, codes, scales)
    return codes, scales


class FrozenLayer:
    """The experts, quantised once, and the buffers that a training loop keeps."""

    def __init__(self, T, H, F, E, k, seed=0):
        self.ctx = binding.Context(T, H, F, E, k)
        self.T, self.H, self.F, self.E, self.k = T, H, F, E, k
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.weights = []
        for rows, cols in ((F, H), (F, H), (H, F)):                     # gate, up, down
            self.weights += frozen_matrix(self.ctx, E, rows, cols, g)
        self.projection = frozen_matrix(self.ctx, 1, H, H, g)
        R, i32 = T * k, dict(dtype=torch.int32, device="cuda")
        self.ids, self.w = torch.empty(T, k, **i32), torch.empty(T, k, device="cuda")
        self.counts, self.offsets = torch.empty(E, **i32), torch.empty(E + 1, **i32)
        self.perm, self.inv = torch.empty(R, **i32), torch.empty(R, **i32)
        u8 = dict(dtype=torch.uint8, device="cuda")
        self.xq, self.sx = torch.empty(T, H, **u8), torch.empty(H // 128, T, device="cuda")
        self.xp, self.sxp = torch.empty(R, H, **u8), torch.empty(H // 128, R, device="cuda")
        self.hq, self.sh = torch.empty(R, F, **u8), torch.empty(F // 128, R, device="cuda")
        self.y = torch.empty(R, H, dtype=torch.bfloat16, device="cuda")
        self.d_w, self.d_logits = torch.empty(T, k, device="cuda"), torch.empty(T, E, device="cuda")
        self.workspace = torch.empty(self.ctx.workspace_layout_blk()["total"], **u8)

    def project(self, x):
        """The frozen dense projection in front of the layer."""
        out = torch.empty_like(x)
        self.ctx.moe_quantize_rows_blk(x, self.T, self.H, self.xq, self.sx)
        self.ctx.moe_gemm_blk(self.xq, self.sx, *self.projection, out, self.T, self.H, self.H)
        return out

    def forward(self, x, logits, bias, rule):
        c, out = self.ctx, torch.empty_like(x)
        c.moe_plan_routing_scored(logits, bias, rule, self.ids, self.w, self.counts, self.offsets, self.perm, self.inv)
        c.moe_quantize_rows_blk(x, self.T, self.H, self.xq, self.sx)
        c.moe_dispatch_blk(self.xq, self.sx, self.inv, self.xp, self.sxp)
        c.moe_expert_ffn_blk(self.xp, self.sxp, self.offsets, *self.weights, self.hq, self.sh, self.y)
        c.moe_combine(self.y, self.inv, self.w, out)
        return out

    def serve(self, x, logits, bias, rule):
        """The same output by one call."""
        out = torch.empty_like(x)
        self.ctx.moe_fused_forward_blk(x, logits, bias, rule, *self.weights, out, self.workspace)
        return out

    def backward_to_logits(self, logits, rule, d_out):
        """Gradient of the last forward's output with respect to its logits; the experts are frozen, so their rows' own
        gradient is not asked for."""
        self.ctx.moe_combine_backward(d_out, self.y, self.inv, self.w, None, self.d_w)
        self.ctx.moe_routing_backward(logits, self.ids, self.d_w, rule, self.d_logits)
        return self.d_logits


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=40)
    args = ap.parse_args(argv)
    T, H, F, E, k = 1024, 512, 256, 32, 4
    layer = FrozenLayer(T, H, F, E, k)
    rule = binding.make_route_rule("sigmoid", n_group=4, topk_group=2, group_top=2, renormalise=True, weight_scale=2.0)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = layer.project(torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16))
    xf = x.float()
    teacher = 2 * torch.randn(H, E, generator=g, device="cuda") / H ** 0.5
    router = teacher + 0.5 * torch.randn(H, E, generator=g, device="cuda") / H ** 0.5
    bias = torch.zeros(E, device="cuda")
    target = layer.forward(x, xf @ teacher, bias, rule).float()
    losses = []
    m, v = torch.zeros_like(router), torch.zeros_like(router)
    for step in range(1, args.steps + 1):
        logits = xf @ router
        diff = layer.forward(x, logits, bias, rule).float() - target
        losses.append(float(diff.square().mean()))
        d_out = (diff * (2 / diff.numel()) * 1024).to(torch.bfloat16)          # a loss scale: the gradient is bf16
        grad = xf.t() @ layer.backward_to_logits(logits, rule, d_out) / 1024
        m.lerp_(grad, 0.1)
        v.lerp_(grad.square(), 0.01)
        router -= 0.01 * (m / (1 - 0.9 ** step)) / ((v / (1 - 0.99 ** step)).sqrt() + 1e-12)
        bias -= 1e-4 * torch.sign(layer.counts.float() - T * k / E)            # towards even loads
        if step % 10 == 0 or step == 1:
            spread = layer.counts.float().std() / (T * k / E)
            print(f"step {step:4d}  loss {losses[-1]:.5f}  load spread {float(spread):.3f}", flush=True)
    tuned = layer.serve(x, xf @ router, bias, rule)
    losses.append(float((tuned.float() - target).square().mean()))
    print(f"the tuned router, served: loss {losses[-1]:.5f}", flush=True)
    code, _ = layer.ctx.moe_last_device_status()
    assert code == 0, code
    return losses


if __name__ == "__main__":
    found = main()
    assert found[-1] < 0.8 * found[0], "the loss did not fall"
