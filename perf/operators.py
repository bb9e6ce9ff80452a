"""Measured cases of the fine-grained layer's operators: scored routing, its gradient through the combine, quantisation
in blocks of 128, the block-scaled FP8 product, and the layer that runs them together.

Each case can be run in two ways on the same inputs: with `own` false as a chain of elementary torch operations in fp32,
rounded once at the end; with `own` true through the library's entry points, as a user calls them.  `exact` computes
the same outputs in fp64, written apart from both.

Layouts (those of include/moe.h): E4M3 codes row-major; scales of row operands [ceil(K/128)][rows] fp32, scales of
weights [groups][ceil(N/128)][ceil(K/128)] fp32; value = code * scale.
"""
import functools
import math
import random

import torch

own = False

DEV = "cuda"
FP8 = torch.float8_e4m3fn


# ------------------------------------------------------------------------------------------------------------- cases
def _rule(score, n_group, topk_group, group_top, renormalise, weight_scale, bias):
    return {"score": score, "n_group": n_group, "topk_group": topk_group, "group_top": group_top,
            "renormalise": renormalise, "weight_scale": weight_scale, "bias": bias}


def listed():
    grouped = _rule("sigmoid", 8, 4, 2, True, 2.5, True)
    return [
        # one decode step of a 64-token batch over the 256 experts of the DeepSeek-V3-like layer: launch latency counts
        {"name": "route_decode", "op": "route", "T": 64, "E": 256, "k": 8, **grouped},
        # a long prefill chunk through the same router
        {"name": "route_prefill", "op": "route", "T": 16384, "E": 256, "k": 8, **grouped},
        # an odd number of tokens, softmax scores, six groups ranked by their best expert, weights not renormalised
        {"name": "route_softmax", "op": "route", "T": 4099, "E": 96, "k": 6,
         **_rule("softmax", 6, 3, 1, False, 16.0, False)},
        # router tuning with frozen experts: a small batch of the fine-grained layer ...
        {"name": "gate_grad_small", "op": "gate_grad", "T": 301, "H": 7168, "E": 256, "k": 8, **grouped},
        # ... and a full batch of the Mixtral-like layer (softmax over all experts, two of eight)
        {"name": "gate_grad_large", "op": "gate_grad", "T": 8192, "H": 4096, "E": 8, "k": 2,
         **_rule("softmax", 1, 1, 1, False, 1.0, False)},
        # the tokens of a mid-size batch, an odd number of rows
        {"name": "quant_rows", "op": "quant", "kind": "rows", "mats": 1, "rows": 1001, "cols": 7168},
        # loading time: one projection of the Mixtral-like layer's eight experts
        {"name": "quant_weights", "op": "quant", "kind": "weights", "mats": 8, "rows": 14336, "cols": 4096},
        # a dense projection at decode: few rows, the weights are the work
        {"name": "product_decode", "op": "product", "groups": 1, "rows": 17, "N": 4096, "K": 7168},
        # a dense projection at prefill: the tensor cores are the work
        {"name": "product_dense", "op": "product", "groups": 1, "rows": 8192, "N": 4096, "K": 7168},
        # one projection of 32 experts with uneven loads, some of them empty, neither N nor K whole blocks
        {"name": "product_ragged", "op": "product", "groups": 32, "rows": 3001, "N": 2104, "K": 4112},
        # the whole layer at decode: 64 tokens, weight streaming
        {"name": "layer_decode", "op": "layer", "T": 64, "H": 7168, "F": 2048, "E": 256, "k": 8, **grouped},
        # the whole layer at prefill: about 128 rows for each expert
        {"name": "layer_prefill", "op": "layer", "T": 4096, "H": 7168, "F": 2048, "E": 256, "k": 8, **grouped},
    ]


def _log_int(rng, lo, hi, step=1):
    """A multiple of step between lo and hi, spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)))
    v = min(hi, max(lo, int(v / step + 0.5) * step)) // step * step
    return v if v != 3072 else v + step                     # (a size that no layer of this library has)


def _draw_rule(rng, most_experts):
    n_group = rng.choice([1, 1, 2, 4, 8])
    while n_group > most_experts:
        n_group //= 2
    size = _log_int(rng, max(1, 8 // n_group), max(1, most_experts // n_group))
    E = n_group * size
    topk_group = rng.randint(1, n_group)
    k = rng.randint(1, min(12, topk_group * size))
    score = rng.choice(["softmax", "sigmoid", "sigmoid"])
    rule = _rule(score, n_group, topk_group, rng.choice([1, 2]) if size > 1 else 1, rng.random() < 0.6,
                 rng.choice([1.0, 2.5, 16.0]), score == "sigmoid" and rng.random() < 0.7)
    return E, k, rule


def draw(rng):
    op = rng.choice(["route", "gate_grad", "quant", "product", "product", "layer", "layer"])
    if op == "route":
        E, k, rule = _draw_rule(rng, 512)
        return {"op": op, "T": _log_int(rng, 1, 16384), "E": E, "k": k, **rule}
    if op == "gate_grad":
        E, k, rule = _draw_rule(rng, 256)
        return {"op": op, "T": _log_int(rng, 1, 8192), "H": _log_int(rng, 128, 7168, 64), "E": E, "k": k, **rule}
    if op == "quant":
        cols = _log_int(rng, 128, 14336, 16)
        if rng.random() < 0.5:
            return {"op": op, "kind": "rows", "mats": 1, "rows": _log_int(rng, 1, 32768), "cols": cols}
        return {"op": op, "kind": "weights", "mats": rng.randint(1, 8), "rows": _log_int(rng, 64, 14336, 8), "cols": cols}
    if op == "product":
        groups = rng.choice([1, _log_int(rng, 2, 64)])
        N, K = _log_int(rng, 128, 8192, 8), _log_int(rng, 128, 8192, 16)
        rows = _log_int(rng, 1, 16384)
        return {"op": op, "groups": groups, "rows": rows, "N": N, "K": K}
    E, k, rule = _draw_rule(rng, 128)
    H, F = _log_int(rng, 256, 7168, 128), _log_int(rng, 128, 4096, 128)
    most = min(32768 // k, int(4.8e11 / (k * H * F)))       # rows and multiply-adds of the largest listed layer
    return {"op": op, "T": _log_int(rng, 1, most), "H": H, "F": F, "E": E, "k": k, **rule}


def work(case):
    op = case["op"]
    if op == "route":
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": 4 * T * E + 16 * T * k + 8 * E, "flops": 4 * T * E}
    if op == "gate_grad":
        T, H, E, k = case["T"], case["H"], case["E"], case["k"]
        return {"bytes": 2 * H * T + 4 * H * T * k + 16 * T * k + 8 * T * E, "flops": 3 * T * k * H}
    if op == "quant":
        n = case["mats"] * case["rows"] * case["cols"]
        blocks = n // 128 if case["kind"] == "rows" else n // 16384
        return {"bytes": 3 * n + 4 * blocks, "flops": 2 * n}
    if op == "product":
        G, R, N, K = case["groups"], case["rows"], case["N"], case["K"]
        read = min(G, R)                                    # a group without rows need not be read
        return {"bytes": R * K + read * N * K + 2 * R * N + R * K // 32 + read * N * K // 4096, "flops": 2 * R * N * K}
    T, H, F, E, k = (case[n] for n in ("T", "H", "F", "E", "k"))
    used = E * (1.0 - (1.0 - k / E) ** T)                   # experts that a batch with even loads reaches
    return {"bytes": 4 * T * H + 4 * T * E + 3 * used * H * F * (1 + 1 / 4096), "flops": 6 * T * k * H * F}


# ------------------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


def _activations(g, rows, cols):
    """bf16 hidden states: unit variance with a few channels an order of magnitude larger, as hidden states have them."""
    x = _randn(g, rows, cols)
    loud = (torch.rand(cols, generator=g, device=DEV) < 0.005).float()
    return (x * (1 + 9 * loud)).to(torch.bfloat16)


def _quantised_weights(g, mats, N, K):
    """E4M3 codes and block scales of mats random matrices N(0, 1/sqrt(K)), made a few at a time."""
    nb, kb = -(-N // 128), -(-K // 128)
    codes = torch.empty(mats, N, K, dtype=torch.uint8, device=DEV)
    scales = torch.empty(mats, nb, kb, dtype=torch.float32, device=DEV)
    at_once = max(1, (1 << 28) // (N * K))
    for m in range(0, mats, at_once):
        n = min(at_once, mats - m)
        w = (_randn(g, n, N, K) / math.sqrt(K)).to(torch.bfloat16)
        c, s = plain_quantise_weights(w)
        codes[m:m + n] = c.view(torch.uint8)
        scales[m:m + n] = s
    return codes, scales


def _logits(g, T, E):
    """Router logits of unit variance over tokens, some experts more popular than others."""
    return _randn(g, T, E) + 0.3 * _randn(g, 1, E)


def _spread_rows(seed, groups, rows):
    """Rows of each group: uneven shares, about one group in eight without any."""
    if groups == 1:
        return [rows]
    r = random.Random(seed)
    share = [0.0 if r.random() < 0.125 else math.exp(r.gauss(0, 0.7)) for _ in range(groups)]
    if not any(share):
        share[r.randrange(groups)] = 1.0
    total, counts = sum(share), []
    for s in share:
        counts.append(int(rows * s / total))
    counts[max(range(groups), key=lambda i: share[i])] += rows - sum(counts)
    return counts


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    state = {"case": case}
    if op in ("route", "layer"):
        state["logits"] = _logits(g, case["T"], case["E"])
        state["bias"] = 0.05 * _randn(g, case["E"]) if case["bias"] else None
    if op == "layer":
        T, H, F, E = (case[n] for n in ("T", "H", "F", "E"))
        state["x"] = _activations(g, T, H)
        state["gate"] = _quantised_weights(g, E, F, H)
        state["up"] = _quantised_weights(g, E, F, H)
        state["down"] = _quantised_weights(g, E, H, F)
    elif op == "gate_grad":
        T, H, E, k = (case[n] for n in ("T", "H", "E", "k"))
        # what the forward pass of such a step has left behind
        state["logits"] = _logits(g, T, E)
        bias = 0.05 * _randn(g, E) if case["bias"] else None
        ids, w = plain_route(state["logits"], bias, case)
        state["ids"], state["w"] = ids, w
        state["inv"] = plain_plan(ids, E)[3]
        state["y"] = _randn(g, T * k, H).to(torch.bfloat16)
        state["d_out"] = (_randn(g, T, H) / math.sqrt(H)).to(torch.bfloat16)
    elif op == "quant":
        if case["kind"] == "rows":
            state["v"] = _activations(g, case["rows"], case["cols"])
        else:
            state["v"] = torch.empty(case["mats"], case["rows"], case["cols"], dtype=torch.bfloat16, device=DEV)
            for m in range(case["mats"]):
                state["v"][m] = _randn(g, case["rows"], case["cols"]) / math.sqrt(case["cols"])
    elif op == "product":
        G, R, N, K = (case[n] for n in ("groups", "rows", "N", "K"))
        a, sa = plain_quantise_rows(_activations(g, R, K))
        state["a"], state["sa"] = a.view(torch.uint8), sa
        state["b"], state["sb"] = _quantised_weights(g, G, N, K)
        counts = _spread_rows(seed, G, R)
        state["offsets"] = torch.tensor([sum(counts[:i]) for i in range(G + 1)], dtype=torch.int32, device=DEV)
    return state


# -------------------------------------------------------------------------------------------------------- plain form
def plain_scores(logits, rule):
    if rule["score"] == "sigmoid":
        return 1 / (1 + torch.exp(-logits))
    e = torch.exp(logits - logits.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def plain_route(logits, bias, rule):
    """Expert ids [T,k] int32 and weights [T,k] fp32: the k best choices of the best groups, ties to the lower index."""
    T, E = logits.shape
    s = plain_scores(logits, rule)
    choice = logits if bias is None else s + bias           # without a bias scores rank as the logits do
    groups = rule["n_group"]
    if groups > 1:
        ranked = choice
        if bias is None and rule["group_top"] == 2:         # sums of scores; softmax's common divisor ranks nothing
            ranked = s if rule["score"] == "sigmoid" else torch.exp(logits - logits.amax(-1, keepdim=True))
        best = ranked.view(T, groups, E // groups).sort(dim=-1, descending=True).values[..., :rule["group_top"]].sum(-1)
        kept = best.sort(dim=-1, descending=True, stable=True).indices[:, :rule["topk_group"]]
        open_ = torch.zeros(T, groups, dtype=torch.bool, device=logits.device).scatter(1, kept, True)
        choice = choice.masked_fill(~open_.repeat_interleave(E // groups, 1), -math.inf)
    ids = choice.sort(dim=-1, descending=True, stable=True).indices[:, :rule["k"]]
    w = s.gather(1, ids)
    if rule["renormalise"]:
        if rule["score"] == "softmax":
            x = logits.gather(1, ids)
            w = torch.exp(x - x.amax(-1, keepdim=True))
        w = w / w.sum(-1, keepdim=True)
    return ids.to(torch.int32), w * rule["weight_scale"]


def plain_plan(ids, E):
    """counts, offsets, perm, inv_perm: the slots in expert order, stable."""
    flat = ids.reshape(-1).long()
    perm = flat.sort(stable=True).indices
    slots = torch.arange(flat.numel(), device=flat.device)
    inv = torch.empty_like(slots).scatter(0, perm, slots)
    counts = torch.zeros(E, dtype=torch.long, device=flat.device).scatter_add(0, flat, torch.ones_like(flat))
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return tuple(t.to(torch.int32) for t in (counts, offsets, perm, inv))


def plain_gate_grad(s, rule):
    T, k = s["ids"].shape
    d_out, inv, ids = s["d_out"].float(), s["inv"].long(), s["ids"].long()
    dy = torch.empty_like(s["y"])
    dy[inv] = (s["w"].unsqueeze(-1) * d_out.unsqueeze(1)).reshape(T * k, -1).to(torch.bfloat16)
    dw = (s["y"].float()[inv].view(T, k, -1) * d_out.unsqueeze(1)).sum(-1)
    p = plain_scores(s["logits"], rule)
    sel, g = p.gather(1, ids), dw * rule["weight_scale"]
    if rule["score"] == "sigmoid":
        if rule["renormalise"]:
            total = sel.sum(-1, keepdim=True)
            g = (g - (g * sel / total).sum(-1, keepdim=True)) / total
        dx = torch.zeros_like(p).scatter(1, ids, g * sel * (1 - sel))
    elif rule["renormalise"]:
        x = s["logits"].gather(1, ids)
        q = torch.exp(x - x.amax(-1, keepdim=True))
        q = q / q.sum(-1, keepdim=True)
        dx = torch.zeros_like(p).scatter(1, ids, q * (g - (g * q).sum(-1, keepdim=True)))
    else:
        dx = p * (torch.zeros_like(p).scatter(1, ids, g) - (g * sel).sum(-1, keepdim=True))
    return {"d_y": dy, "d_w": dw, "d_logits": dx}


def _scale_of(amax):
    top = torch.full((), 448.0, device=amax.device, dtype=amax.dtype)   # (a tensor: a true division, not a product)
    return torch.where(amax > 0, amax / top, torch.ones_like(amax))


def plain_quantise_rows(v):
    """codes [rows,cols] E4M3, scales [ceil(cols/128)][rows] of the row's blocks of 128."""
    rows, cols = v.shape
    v = v.float()
    padded = torch.nn.functional.pad(v, (0, -cols % 128)).view(rows, -1, 128)
    scale = _scale_of(padded.abs().amax(-1))
    codes = (padded / scale.unsqueeze(-1)).reshape(rows, -1)[:, :cols].to(FP8).contiguous()
    return codes, scale.t().contiguous()


def plain_quantise_weights(w):
    """codes [mats,N,K] E4M3, scales [mats][ceil(N/128)][ceil(K/128)] of blocks of 128 x 128."""
    m, N, K = w.shape
    w = w.float()
    padded = torch.nn.functional.pad(w, (0, -K % 128, 0, -N % 128))
    blocks = padded.view(m, padded.shape[1] // 128, 128, padded.shape[2] // 128, 128)
    scale = _scale_of(blocks.abs().amax((2, 4)))
    codes = (blocks / scale[:, :, None, :, None]).reshape(padded.shape)[:, :N, :K].to(FP8).contiguous()
    return codes, scale


def plain_rows(codes, scales, dtype=torch.float32):
    """The values of quantised rows."""
    K = codes.shape[1]
    return codes.view(FP8).to(dtype) * scales.to(dtype).repeat_interleave(128, 0)[:K].t()


def plain_weights(codes, scales):
    """The values of quantised weights, fp32."""
    _, N, K = codes.shape
    w = codes.view(FP8).float()
    w *= scales.repeat_interleave(128, 1)[:, :N].repeat_interleave(128, 2)[:, :, :K]
    return w


def plain_grouped(a, offsets, w):
    """a [R,K] in group order times each group's w[g] [N,K], transposed: [R,N]."""
    G = w.shape[0]
    if G == 1:
        return a @ w[0].t()
    rows = torch.arange(a.shape[0], device=a.device)
    ends = offsets[1:].long()
    group = torch.searchsorted(ends, rows, right=True)
    place = rows - offsets.long()[group]
    most = int((offsets[1:] - offsets[:-1]).max())          # a chain of torch operations has to know its sizes
    padded = a.new_zeros(G, most, a.shape[1])
    padded[group, place] = a
    return torch.bmm(padded, w.transpose(1, 2))[group, place]


def plain_layer(s, rule):
    T, H = s["x"].shape
    E, k = rule["E"], rule["k"]
    ids, w = plain_route(s["logits"], s["bias"], rule)
    _, offsets, perm, inv = plain_plan(ids, E)
    x = plain_rows(*plain_quantise_rows(s["x"]))[perm.long() // k]
    gate = plain_grouped(x, offsets, plain_weights(*s["gate"]))
    up = plain_grouped(x, offsets, plain_weights(*s["up"]))
    h = gate / (1 + torch.exp(-gate)) * up
    y = plain_grouped(plain_rows(*plain_quantise_rows(h)), offsets, plain_weights(*s["down"]))
    out = (y[inv.long()].view(T, k, H) * w.unsqueeze(-1)).sum(1)
    return {"out": out.to(torch.bfloat16), "ids": ids, "w": w}


def _run_plain(state):
    case, op = state["case"], state["case"]["op"]
    if op == "route":
        ids, w = plain_route(state["logits"], state["bias"], case)
        counts, offsets, perm, inv = plain_plan(ids, case["E"])
        return {"ids": ids, "w": w, "counts": counts, "offsets": offsets, "perm": perm, "inv": inv}
    if op == "gate_grad":
        return plain_gate_grad(state, case)
    if op == "quant":
        codes, scales = plain_quantise_rows(state["v"]) if case["kind"] == "rows" else plain_quantise_weights(state["v"])
        return {"codes": codes, "scales": scales}
    if op == "product":
        a = plain_rows(state["a"], state["sa"])
        return {"y": plain_grouped(a, state["offsets"], plain_weights(state["b"], state["sb"])).to(torch.bfloat16)}
    return plain_layer(state, case)


# ----------------------------------------------------------------------------------------------------- the library
@functools.lru_cache(maxsize=8)
def _context(T, H, F, E, k):
    """The handle a program creates once for a layer's shape and keeps."""
    from paper_2607_23264_b200 import binding
    return binding.Context(T, H, F, E, k, device=torch.cuda.current_device())


@functools.lru_cache(maxsize=32)
def _library_rule(score, n_group, topk_group, group_top, renormalise, weight_scale):
    from paper_2607_23264_b200 import binding
    return binding.make_route_rule(score=score, n_group=n_group, topk_group=topk_group, group_top=group_top,
                                   renormalise=renormalise, weight_scale=weight_scale)


def _rule_of(case):
    return _library_rule(case["score"], case["n_group"], case["topk_group"], case["group_top"], case["renormalise"],
                         case["weight_scale"])


def _int32(*shape):
    return torch.empty(shape, dtype=torch.int32, device=DEV)


def _run_own(state):
    case, op = state["case"], state["case"]["op"]
    if op == "route":
        T, E, k = case["T"], case["E"], case["k"]
        ctx = _context(T, 64, 64, E, k)
        o = {"ids": _int32(T, k), "w": torch.empty(T, k, device=DEV), "counts": _int32(E), "offsets": _int32(E + 1),
             "perm": _int32(T * k), "inv": _int32(T * k)}
        ctx.moe_plan_routing_scored(state["logits"], state["bias"], _rule_of(case), o["ids"], o["w"], o["counts"],
                                    o["offsets"], o["perm"], o["inv"])
        return o
    if op == "gate_grad":
        T, H, E, k = (case[n] for n in ("T", "H", "E", "k"))
        ctx = _context(T, H, 64, E, k)
        o = {"d_y": torch.empty_like(state["y"]), "d_w": torch.empty(T, k, device=DEV),
             "d_logits": torch.empty(T, E, device=DEV)}
        ctx.moe_combine_backward(state["d_out"], state["y"], state["inv"], state["w"], o["d_y"], o["d_w"])
        ctx.moe_routing_backward(state["logits"], state["ids"], o["d_w"], _rule_of(case), o["d_logits"])
        return o
    if op == "quant":
        mats, rows, cols = case["mats"], case["rows"], case["cols"]
        ctx, v, kb = _context(1, 64, 64, 1, 1), state["v"], -(-cols // 128)
        codes = torch.empty(v.shape, dtype=torch.uint8, device=DEV)
        if case["kind"] == "rows":
            scales = torch.empty(kb, rows, device=DEV)
            ctx.moe_quantize_rows_blk(v, rows, cols, codes, scales)
        else:
            scales = torch.empty(mats, -(-rows // 128), kb, device=DEV)
            ctx.moe_quantize_weights_blk(v, mats, rows, cols, codes, scales)
        return {"codes": codes.view(FP8), "scales": scales}
    if op == "product":
        G, R, N, K = (case[n] for n in ("groups", "rows", "N", "K"))
        ctx = _context(1, 64, 64, 1, 1)
        y = torch.empty(R, N, dtype=torch.bfloat16, device=DEV)
        ctx.moe_gemm_blk(state["a"], state["sa"], state["b"], state["sb"], y, R, N, K, groups=G,
                         offsets=state["offsets"] if G > 1 else None)
        return {"y": y}
    T, H, F, E, k = (case[n] for n in ("T", "H", "F", "E", "k"))
    ctx = _context(T, H, F, E, k)
    if "workspace" not in state:                            # kept from step to step, as a serving program does
        state["layout"] = ctx.workspace_layout_blk()
        state["workspace"] = torch.empty(state["layout"]["total"], dtype=torch.uint8, device=DEV)
    out, ws, at = torch.empty_like(state["x"]), state["workspace"], state["layout"]
    ctx.moe_fused_forward_blk(state["x"], state["logits"], state["bias"], _rule_of(case), *state["gate"], *state["up"],
                              *state["down"], out, ws)
    slots = lambda name, kind: ws[at[name]:at[name] + 4 * T * k].view(kind).view(T, k)  # noqa: E731
    return {"out": out, "ids": slots("topk_ids", torch.int32), "w": slots("topk_w", torch.float32)}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------- exact, in 64 bits
def _exact_route(logits, bias, case):
    x = logits.double()
    if case["score"] == "sigmoid":
        s = torch.special.expit(x)
    else:
        s = torch.softmax(x, -1)
    c = s if bias is None else s + bias.double()
    T, E = x.shape
    G = case["n_group"]
    best = torch.topk(c.view(T, G, E // G), case["group_top"], -1).values.sum(-1)
    floor = torch.topk(best, case["topk_group"], -1).values[:, -1:]
    c = torch.where((best >= floor).repeat_interleave(E // G, 1), c, torch.full_like(c, -1e9))
    ids = torch.topk(c, case["k"], -1).indices
    w = torch.gather(s, 1, ids)
    if case["renormalise"]:
        w = w / w.sum(-1, keepdim=True)
    return ids, w * case["weight_scale"]


def _exact_values(v, dims):
    """v (fp64) and the scale of each block: blocks of 128 along the last axis, or of 128 x 128."""
    scale = torch.empty([-(-n // 128) if d >= v.dim() - dims else n for d, n in enumerate(v.shape)], dtype=v.dtype,
                        device=v.device)
    for j in range(scale.shape[-1]):
        if dims == 1:
            scale[..., j] = v[..., 128 * j:128 * (j + 1)].abs().amax(-1)
        else:
            for i in range(scale.shape[-2]):
                scale[..., i, j] = v[..., 128 * i:128 * (i + 1), 128 * j:128 * (j + 1)].abs().amax((-1, -2))
    scale = torch.where(scale == 0, torch.ones_like(scale), scale / 448)
    full = scale.repeat_interleave(128, -1)[..., :v.shape[-1]]
    if dims == 2:
        full = full.repeat_interleave(128, -2)[..., :v.shape[-2], :]
    return (v / full).to(FP8).double(), scale, full


def _exact_matrix(codes, scales):
    N, K = codes.shape
    rows = torch.arange(N, device=codes.device) // 128
    cols = torch.arange(K, device=codes.device) // 128
    return codes.view(FP8).double() * scales.double()[rows][:, cols]


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "route":
        _, w = _exact_route(s["logits"], s["bias"], case)
        return {"ids": None, "w": w, "counts": None, "offsets": None, "perm": None, "inv": None}
    if op == "gate_grad":
        T, k, scale = case["T"], case["k"], case["weight_scale"]
        d_out, inv = s["d_out"].double(), s["inv"].long().view(T, k)
        dy = torch.empty(s["y"].shape, dtype=torch.float64, device=DEV)
        dw = torch.empty(T, k, dtype=torch.float64, device=DEV)
        for j in range(k):
            dy[inv[:, j]] = s["w"].double()[:, j:j + 1] * d_out
            dw[:, j] = torch.einsum("th,th->t", d_out, s["y"][inv[:, j]].double())
        # the weights as a function of the logits, differentiated
        x = s["logits"].double().requires_grad_(True)
        score = torch.special.expit(x) if case["score"] == "sigmoid" else torch.softmax(x, -1)
        w = torch.gather(score, 1, s["ids"].long())
        if case["renormalise"]:
            w = w / w.sum(-1, keepdim=True)
        (scale * w * dw).sum().backward()
        return {"d_y": dy, "d_w": dw, "d_logits": x.grad}
    if op == "quant":
        if case["kind"] == "rows":
            codes, scales, _ = _exact_values(s["v"].double(), 1)
            return {"codes": codes, "scales": scales.t().contiguous()}
        each = [_exact_values(s["v"][m].double(), 2)[:2] for m in range(case["mats"])]
        return {"codes": torch.stack([c for c, _ in each]), "scales": torch.stack([c for _, c in each])}
    if op == "product":
        a = plain_rows(s["a"], s["sa"], torch.float64)
        y = torch.empty(case["rows"], case["N"], dtype=torch.float64, device=DEV)
        at = s["offsets"].tolist()
        for g in range(case["groups"]):
            if at[g + 1] > at[g]:
                y[at[g]:at[g + 1]] = a[at[g]:at[g + 1]] @ _exact_matrix(s["b"][g], s["sb"][g]).t()
        return {"y": y}
    ids, w = _exact_route(s["logits"], s["bias"], case)
    codes, _, full = _exact_values(s["x"].double(), 1)
    x = codes * full
    out = torch.zeros(s["x"].shape, dtype=torch.float64, device=DEV)
    for e in range(case["E"]):
        token, slot = torch.nonzero(ids == e, as_tuple=True)
        if token.numel() == 0:
            continue
        gate = x[token] @ _exact_matrix(s["gate"][0][e], s["gate"][1][e]).t()
        up = x[token] @ _exact_matrix(s["up"][0][e], s["up"][1][e]).t()
        codes, _, full = _exact_values(gate * torch.special.expit(gate) * up, 1)
        y = (codes * full) @ _exact_matrix(s["down"][0][e], s["down"][1][e]).t()
        out.index_add_(0, token, y * w[token, slot].unsqueeze(-1))
    return {"out": out, "ids": None, "w": w}
