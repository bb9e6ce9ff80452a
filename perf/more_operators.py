"""Measured cases of the operators around the expert layer: the residual's addition with the RMS norm and its 8-bit output,
that norm's gradient, the router's balance loss with its gradient, and low-rank adapters beside a shared projection.

Each case can be run in two ways on the same inputs: with `own` false as a chain of elementary torch operations in fp32,
rounded once at the end; with `own` true through the library's entry points, as a user calls them.  `exact` computes
the same outputs in fp64, written apart from both.

Layouts (those of include/moe.h): E4M3 codes row-major; scales of rows [rows] fp32 (form "rows"), [ceil(cols/128)][rows]
fp32 (form "blk") or, as exponent bytes, [cols/128][rows][4] (form "mx"); value = code * scale.
"""
import functools
import math
import random

import torch

own = False

DEV = "cuda"
FP8 = torch.float8_e4m3fn
E8M0 = torch.float8_e8m0fnu
EPS = 1e-6


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decode step of a 64-token batch in front of the fine-grained layer: the router reads the bf16 rows, the experts
        # the codes in blocks of 128; launch latency counts
        {"name": "norm_decode", "op": "norm", "rows": 64, "cols": 7168, "residual": True, "out": True, "form": "blk",
         "gain": "bf16"},
        # a prefill batch in front of the same layer
        {"name": "norm_prefill", "op": "norm", "rows": 8192, "cols": 7168, "residual": True, "out": True, "form": "blk",
         "gain": "bf16"},
        # an odd number of tokens in front of experts with one scale per row, nothing to add, the codes alone
        {"name": "norm_rows", "op": "norm", "rows": 1001, "cols": 4096, "residual": False, "out": False, "form": "rows",
         "gain": "fp32"},
        # tokens in front of MXFP8 experts
        {"name": "norm_mx", "op": "norm", "rows": 4099, "cols": 2048, "residual": True, "out": True, "form": "mx",
         "gain": "bf16"},
        # the norm's gradients while a router is tuned: a small batch of the fine-grained layer ...
        {"name": "norm_grad_small", "op": "norm_grad", "rows": 301, "cols": 7168, "residual": False, "gain": "bf16"},
        # ... and a full batch of the Mixtral-like layer, with the gradient that comes along the residual
        {"name": "norm_grad_large", "op": "norm_grad", "rows": 8192, "cols": 4096, "residual": True, "gain": "fp32"},
        # a training batch of one long sequence over the 256 experts of the fine-grained layer: loss, counts, gradient
        {"name": "balance_long", "op": "balance", "T": 16384, "E": 256, "k": 8, "score": "sigmoid", "sequences": 1,
         "mask": False, "z": False},
        # packed sequences of uneven lengths with padded tokens, softmax scores, the logits' own penalty with it
        {"name": "balance_packed", "op": "balance", "T": 4099, "E": 64, "k": 6, "score": "softmax", "sequences": 13,
         "mask": True, "z": True},
        # decode: 64 requests of one token each, 32 adapters of rank 16 beside one projection
        {"name": "adapters_decode", "op": "adapters", "rows": 64, "N": 4096, "K": 7168, "rank": 16, "adapters": 32,
         "segments": 64},
        # prefill: four requests of about two thousand tokens, adapters of rank 64
        {"name": "adapters_prefill", "op": "adapters", "rows": 8192, "N": 4096, "K": 7168, "rank": 64, "adapters": 4,
         "segments": 4},
        # long and short requests in one batch, some without an adapter, neither N nor K whole tiles
        {"name": "adapters_mixed", "op": "adapters", "rows": 1501, "N": 2104, "K": 4112, "rank": 24, "adapters": 9,
         "segments": 40},
    ]


def _log_int(rng, lo, hi, step=1):
    """A multiple of step between lo and hi, spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)))
    return min(hi // step * step, max(-(-lo // step) * step, int(v / step + 0.5) * step))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "balance", "balance", "adapters", "adapters", "adapters"])
    if op in ("norm", "norm_grad"):
        form = rng.choice(["none", "rows", "mx", "blk", "blk"])
        cols = _log_int(rng, 128, 8192, 128 if form == "mx" else 16 if form == "blk" else 8)
        rows = _log_int(rng, 1, min(16384, 8192 * 7168 // cols))
        case = {"op": op, "rows": rows, "cols": cols, "residual": rng.random() < 0.7, "gain": rng.choice(["bf16", "fp32"])}
        return case if op == "norm_grad" else {**case, "form": form, "out": form == "none" or rng.random() < 0.6}
    if op == "balance":
        E = _log_int(rng, 4, 512)
        T = _log_int(rng, 1, 16384)
        return {"op": op, "T": T, "E": E, "k": rng.randint(1, min(8, E)), "score": rng.choice(["softmax", "sigmoid"]),
                "sequences": rng.choice([1, 1, _log_int(rng, 2, 64)]), "mask": rng.random() < 0.4, "z": rng.random() < 0.5}
    N, K = _log_int(rng, 256, 7168, 8), _log_int(rng, 256, 7168, 8)
    rows = _log_int(rng, 1, min(8192, 8192 * (7168 + 2 * 4096) // (K + 2 * N)))        # no more bytes than the largest listed
    segments = rows if rng.random() < 0.3 and rows <= 512 else _log_int(rng, 1, min(rows, 256))
    return {"op": op, "rows": rows, "N": N, "K": K, "rank": _log_int(rng, 8, 64, 8), "adapters": _log_int(rng, 1, 32),
            "segments": segments}


def work(case):
    op = case["op"]
    if op == "norm":
        n = case["rows"] * case["cols"]
        moved = 2 + (4 if case["residual"] else 0) + (2 if case["out"] else 0) + (0 if case["form"] == "none" else 1)
        per_row = {"none": 0, "rows": 4, "mx": case["cols"] // 32, "blk": 4 * -(-case["cols"] // 128)}[case["form"]]
        return {"bytes": n * moved + case["rows"] * per_row + case["cols"] * 4, "flops": 8 * n}
    if op == "norm_grad":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (8 if case["residual"] else 6) + 8 * case["cols"], "flops": 12 * n}
    if op == "balance":
        T, E, k, S = (case[n] for n in ("T", "E", "k", "sequences"))
        return {"bytes": 12 * T * E + 4 * T * k + 8 * S * E, "flops": 20 * T * E}
    R, N, K, rank = (case[n] for n in ("rows", "N", "K", "rank"))
    used = min(case["adapters"], case["segments"])
    return {"bytes": 2 * R * K + 4 * R * N + 2 * used * rank * (N + K), "flops": 2 * R * rank * (N + K)}


# ------------------------------------------------------------------------------------------------------------ inputs
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


def _activations(g, rows, cols):
    """bf16 hidden states: unit variance with a few channels an order of magnitude larger, as hidden states have them."""
    loud = (torch.rand(cols, generator=g, device=DEV) < 0.005).float()
    return (_randn(g, rows, cols) * (1 + 9 * loud)).to(torch.bfloat16)


def _spread(r, parts, total, empty):
    """`total` split into `parts` uneven counts, a share of them zero."""
    weight = [0.0 if r.random() < empty else math.exp(r.gauss(0, 1)) for _ in range(parts)]
    if not any(weight):
        weight[r.randrange(parts)] = 1.0
    whole = sum(weight)
    counts = [int(total * w / whole) for w in weight]
    counts[max(range(parts), key=lambda i: weight[i])] += total - sum(counts)
    return counts


def _offsets(counts):
    return torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g, r, op = torch.Generator(device=DEV).manual_seed(seed), random.Random(seed), case["op"]
    state = {"case": case}
    if op in ("norm", "norm_grad"):
        rows, cols = case["rows"], case["cols"]
        state["x"] = _activations(g, rows, cols)
        state["gain"] = (1 + 0.2 * _randn(g, cols)).to(torch.bfloat16 if case["gain"] == "bf16" else torch.float32)
        if op == "norm":
            state["residual"] = (4 * _randn(g, rows, cols)).to(torch.bfloat16) if case["residual"] else None
        else:
            state["d_out"] = (_randn(g, rows, cols) / math.sqrt(cols)).to(torch.bfloat16)
            state["d_sum"] = (_randn(g, rows, cols) / math.sqrt(cols)).to(torch.bfloat16) if case["residual"] else None
    elif op == "balance":
        T, E, k, S = (case[n] for n in ("T", "E", "k", "sequences"))
        state["logits"] = _randn(g, T, E) + 0.5 * _randn(g, 1, E)
        # the choice of the layer's plan, moved by a balance bias
        noisy = state["logits"] + 0.3 * _randn(g, 1, E)
        state["ids"] = noisy.sort(dim=-1, descending=True).indices[:, :k].to(torch.int32).contiguous()
        state["offsets"] = _offsets(_spread(r, S, T, 0.1)) if S > 1 else None
        state["mask"] = (torch.rand(T, generator=g, device=DEV) < 0.8).to(torch.uint8) if case["mask"] else None
        state["d_loss"] = torch.full((1,), 1024.0, device=DEV)               # a loss scale
        state["add"] = _randn(g, T, E) * 0.01                                # what the weights' gradient left behind
    else:
        R, N, K, rank, A, S = (case[n] for n in ("rows", "N", "K", "rank", "adapters", "segments"))
        state["x"] = _activations(g, R, K)
        state["a"] = (_randn(g, A, rank, K) / math.sqrt(K)).to(torch.bfloat16)
        state["b"] = (0.5 * _randn(g, A, N, rank) / math.sqrt(rank)).to(torch.bfloat16)
        state["scale"] = 0.5 + torch.rand(A, generator=g, device=DEV)
        state["y"] = _randn(g, R, N).to(torch.bfloat16)                      # the shared projection's output
        if S == R:
            state["offsets"] = None                                          # every row a request of its own
        else:
            counts = _spread(r, S, R, 0.05)
            if S >= 16:                                                      # long prompts beside single tokens
                counts = [1] * (S // 2) + _spread(r, S - S // 2, R - S // 2, 0.05)
                r.shuffle(counts)
            state["offsets"] = _offsets(counts)
        none = 0.1 if S >= 8 else 0.0
        ids = [-1 if r.random() < none else r.randrange(A) for _ in range(S)]
        state["ids"] = torch.tensor(ids, dtype=torch.int32, device=DEV)
    return state


# -------------------------------------------------------------------------------------------------------- plain form
def _scale_of(amax):
    top = torch.full((), 448.0, device=amax.device)                          # (a tensor: a true division, not a product)
    return torch.where(amax > 0, amax / top, torch.ones_like(amax))


def _plain_mx(n):
    """Codes, and the exponent bytes [cols/128][rows][4]: the smallest power of two that brings a block below 448."""
    rows, cols = n.shape
    blocks = n.view(rows, cols // 32, 32)
    m, e = torch.frexp(blocks.abs().amax(-1))                                # amax = m 2^e, 0.5 <= m < 1
    e = torch.where(m > 0.875, e - 8, e - 9).clamp_min(-127)                 # 448 = 0.875 2^9
    codes = torch.ldexp(blocks, -e.unsqueeze(-1)).reshape(rows, cols).to(FP8)
    return codes, (e + 127).to(torch.uint8).view(rows, cols // 128, 4).transpose(0, 1).contiguous()


def _plain_norm(s, case):
    x, result = s["x"], {}
    if case["residual"]:
        x = (x.float() + s["residual"].float()).to(torch.bfloat16)           # the stream as the next layer reads it
        result["sum"] = x
    x = x.float()
    n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["gain"].float()
    if case["out"]:
        result["out"] = n.to(torch.bfloat16)
    if case["form"] == "rows":
        scale = _scale_of(n.abs().amax(-1))
        result["codes"], result["scales"] = (n / scale.unsqueeze(-1)).to(FP8), scale
    elif case["form"] == "blk":
        rows, cols = n.shape
        blocks = torch.nn.functional.pad(n, (0, -cols % 128)).view(rows, -1, 128)
        scale = _scale_of(blocks.abs().amax(-1))
        result["codes"] = (blocks / scale.unsqueeze(-1)).reshape(rows, -1)[:, :cols].to(FP8).contiguous()
        result["scales"] = scale.t().contiguous()
    elif case["form"] == "mx":
        codes, bytes_ = _plain_mx(n)
        result["codes"], result["scales"] = codes, bytes_.view(E8M0)
    return result


def _plain_norm_grad(s):
    x, d = s["x"].float(), s["d_out"].float()
    rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    hat, dg = x * rstd, d * s["gain"].float()
    dx = rstd * (dg - hat * (dg * hat).mean(-1, keepdim=True))
    if s["d_sum"] is not None:
        dx = dx + s["d_sum"].float()
    return {"d_x": dx.to(torch.bfloat16), "d_gain": (d * hat).sum(0)}


def _coefs(case):
    return 0.01, 1e-3 if case["z"] else 0.0


def _plain_balance(s, case):
    T, E, k, S = (case[n] for n in ("T", "E", "k", "sequences"))
    coef, z_coef = _coefs(case)
    x, ids = s["logits"], s["ids"].long()
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    soft = e / total
    score = soft if case["score"] == "softmax" else 1 / (1 + torch.exp(-x))
    p = score if case["score"] == "softmax" else score / score.sum(-1, keepdim=True)
    lse = (torch.log(total) + top)[:, 0]
    tokens = torch.arange(T, device=x.device)
    counted = torch.ones(T, device=x.device) if s["mask"] is None else (s["mask"] != 0).float()
    seq = torch.zeros_like(tokens) if S == 1 else torch.searchsorted(s["offsets"][1:].long(), tokens, right=True)
    member = (seq == torch.arange(S, device=x.device).unsqueeze(1)).float() * counted              # [S, T]
    n = member.sum(-1)
    one = (counted > 0).long().unsqueeze(1).expand(T, k).reshape(-1)
    counts = torch.zeros(S * E, dtype=torch.long, device=x.device).scatter_add(0, (seq.unsqueeze(1) * E + ids).reshape(-1), one)
    counts = counts.view(S, E)
    some = n.clamp_min(1).unsqueeze(1)
    mean = member @ p / some
    load = counts.float() * E / (k * some)
    all_ = n.sum().clamp_min(1)
    loss = torch.stack([coef / S * (load * mean).sum(), z_coef / all_ * (counted * lse * lse).sum()])
    up = s["d_loss"] * coef / S * (load / some)[seq] * counted.unsqueeze(1)
    dx = p * (up - (up * p).sum(-1, keepdim=True))
    if case["score"] == "sigmoid":
        dx = dx / (1 + torch.exp(x))
    if case["z"]:
        dx = dx + s["d_loss"] * (2 * z_coef / all_) * (counted * lse).unsqueeze(1) * soft
    return {"counts": counts.to(torch.int32), "mean": mean, "loss": loss, "d_logits": s["add"] + dx}


def _plain_adapters(s, case):
    R, A, rank = case["rows"], case["adapters"], case["rank"]
    rows = torch.arange(R, device=s["x"].device)
    segment = rows if s["offsets"] is None else torch.searchsorted(s["offsets"][1:].long(), rows, right=True)
    ids = s["ids"].long()[segment]
    group = torch.where(ids < 0, A, ids)                                     # rows without an adapter: a group of their own
    order = group.sort(stable=True).indices
    sizes = torch.zeros(A + 1, dtype=torch.long, device=rows.device).scatter_add(0, group, torch.ones_like(group))
    place = torch.empty_like(rows).scatter(0, order, rows) - (sizes.cumsum(0) - sizes)[group]
    has = ids >= 0
    at = (group[has], place[has])
    x = torch.zeros(A, int(sizes[:A].max()), case["K"], device=rows.device)  # a chain of torch operations has to know its sizes
    x[at] = s["x"].float()[has]
    t = torch.bmm(x, s["a"].float().transpose(1, 2)) * s["scale"].view(A, 1, 1)
    y = s["y"].float()
    y[has] += torch.bmm(t, s["b"].float().transpose(1, 2))[at]
    return {"y": y.to(torch.bfloat16)}


def _run_plain(state):
    case, op = state["case"], state["case"]["op"]
    if op == "norm":
        return _plain_norm(state, case)
    if op == "norm_grad":
        return _plain_norm_grad(state)
    return _plain_balance(state, case) if op == "balance" else _plain_adapters(state, case)


# ----------------------------------------------------------------------------------------------------- the library
@functools.lru_cache(maxsize=8)
def _context(T, E, k):
    """The handle a program creates once for a layer's shape and keeps."""
    from paper_2607_23264_b200 import binding
    return binding.Context(T, 64, 64, E, k, device=torch.cuda.current_device())


def _scratch(state, size):
    """Kept from step to step, as a program does."""
    if "scratch" not in state:
        state["scratch"] = torch.empty(max(16, size()), dtype=torch.uint8, device=DEV)
    return state["scratch"]


def _run_own(state):
    case, op = state["case"], state["case"]["op"]
    if op == "norm":
        ctx, x, form = _context(1, 1, 1), state["x"], case["form"]
        rows, cols = x.shape
        o = {}
        if case["residual"]:
            o["sum"] = torch.empty_like(x)
        if case["out"]:
            o["out"] = torch.empty_like(x)
        if form != "none":
            o["codes"] = torch.empty(rows, cols, dtype=FP8, device=DEV)
            if form == "mx":
                o["scales"] = torch.empty(cols // 128, rows, 4, dtype=E8M0, device=DEV)
            else:
                o["scales"] = torch.empty(rows if form == "rows" else (-(-cols // 128), rows), device=DEV)
        ctx.moe_add_rms_norm(x, state["residual"], state["gain"], rows, cols, sum_out=o.get("sum"), out=o.get("out"),
                             codes=o.get("codes"), scales=o.get("scales"), form=form, eps=EPS)
        return o
    if op == "norm_grad":
        ctx, x = _context(1, 1, 1), state["x"]
        rows, cols = x.shape
        scratch = _scratch(state, lambda: ctx.rms_norm_scratch_bytes(rows, cols))
        o = {"d_x": torch.empty_like(x), "d_gain": torch.empty(cols, device=DEV)}
        ctx.moe_rms_norm_backward(x, state["gain"], state["d_out"], rows, cols, o["d_x"], o["d_gain"], scratch,
                                  d_sum=state["d_sum"], eps=EPS)
        return o
    if op == "balance":
        T, E, k, S = (case[n] for n in ("T", "E", "k", "sequences"))
        ctx, (coef, z_coef) = _context(T, E, k), _coefs(case)
        scratch = _scratch(state, lambda: ctx.balance_scratch_bytes(S))
        o = {"counts": torch.empty(S, E, dtype=torch.int32, device=DEV), "mean": torch.empty(S, E, device=DEV),
             "loss": torch.empty(2, device=DEV), "d_logits": torch.empty(T, E, device=DEV)}
        tokens = torch.empty(S + 1, dtype=torch.int32, device=DEV)
        how = dict(score=case["score"], coef=coef, z_coef=z_coef, sequences=S, seq_offsets=state["offsets"],
                   token_mask=state["mask"])
        ctx.moe_balance_loss(state["logits"], state["ids"], o["counts"], tokens, o["mean"], o["loss"], scratch, **how)
        ctx.moe_balance_loss_backward(state["logits"], o["counts"], tokens, o["d_logits"], d_loss=state["d_loss"],
                                      add=state["add"], **how)
        return o
    R, N, K, rank, A, S = (case[n] for n in ("rows", "N", "K", "rank", "adapters", "segments"))
    ctx = _context(1, 1, 1)
    scratch = _scratch(state, lambda: ctx.adapter_scratch_bytes(R, K, rank))
    y = torch.empty_like(state["y"])
    ctx.moe_add_adapters(state["x"], state["a"], state["b"], state["ids"], state["y"], y, scratch, R, N, K, rank, A, S,
                         offsets=state["offsets"], scale=state["scale"])
    return {"y": y}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------- exact, in 64 bits
def _exact_codes(n, form):
    """Codes (as values) and scales of n, a block at a time."""
    rows, cols = n.shape
    width = {"rows": cols, "blk": 128, "mx": 32}[form]
    codes, scales = torch.empty_like(n), []
    for lo in range(0, cols, width):
        part = n[:, lo:lo + width]
        amax = part.abs().amax(-1)
        if form == "mx":
            scale = torch.exp2(torch.ceil(torch.log2(amax.clamp_min(2.0 ** -140) / 448)).clamp(-127, 127))
        else:
            scale = torch.where(amax == 0, torch.ones_like(amax), amax / 448)
        codes[:, lo:lo + width] = (part / scale.unsqueeze(-1)).to(FP8).double()
        scales.append(scale)
    if form == "rows":
        return codes, scales[0]
    if form == "blk":
        return codes, torch.stack(scales)
    return codes, torch.stack(scales).view(cols // 128, 4, rows).transpose(1, 2).contiguous()


def _exact_balance(s, case):
    T, E, k, S = (case[n] for n in ("T", "E", "k", "sequences"))
    coef, z_coef = _coefs(case)
    bounds = [0, T] if s["offsets"] is None else s["offsets"].tolist()
    use = torch.ones(T, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"] != 0
    x = s["logits"].double().requires_grad_(True)
    total, mean, z_sum, z_n = 0.0, torch.zeros(S, E, dtype=torch.float64, device=DEV), 0.0, 0
    for i in range(S):
        keep = torch.nonzero(use[bounds[i]:bounds[i + 1]])[:, 0] + bounds[i]
        if keep.numel() == 0:
            continue
        part = x[keep]
        q = torch.softmax(part, -1) if case["score"] == "softmax" else torch.special.expit(part)
        q = q / q.sum(-1, keepdim=True)
        load = torch.bincount(s["ids"][keep].reshape(-1).long(), minlength=E).double() * E / (k * keep.numel())
        total = total + coef / S * (load * q.mean(0)).sum()
        mean[i] = q.mean(0).detach()
        z_sum, z_n = z_sum + torch.logsumexp(part, -1).square().sum(), z_n + keep.numel()
    z = z_coef * z_sum / max(1, z_n)
    loss = torch.stack([torch.as_tensor(v, dtype=torch.float64, device=DEV).detach() for v in (total, z)])
    grad = torch.zeros(T, E, dtype=torch.float64, device=DEV)
    if z_n:
        grad = torch.autograd.grad(total + z, x)[0]
    return {"counts": None, "mean": mean, "loss": loss, "d_logits": s["add"].double() + s["d_loss"].double() * grad}


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "norm":
        result, x = {}, s["x"].double()
        if case["residual"]:
            result["sum"] = x = (x + s["residual"].double()).to(torch.bfloat16).double()
        n = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["cols"] + EPS) * s["gain"].double()
        if case["out"]:
            result["out"] = n
        if case["form"] != "none":
            result["codes"], result["scales"] = _exact_codes(n, case["form"])
        return result
    if op == "norm_grad":
        x, gain = s["x"].double().requires_grad_(True), s["gain"].double().requires_grad_(True)
        n = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["cols"] + EPS) * gain
        dx, d_gain = torch.autograd.grad(n, (x, gain), s["d_out"].double())
        return {"d_x": dx if s["d_sum"] is None else dx + s["d_sum"].double(), "d_gain": d_gain}
    if op == "balance":
        return _exact_balance(s, case)
    y = s["y"].double()
    bounds = range(case["rows"] + 1) if s["offsets"] is None else s["offsets"].tolist()
    for i, adapter in enumerate(s["ids"].tolist()):
        lo, hi = bounds[i], bounds[i + 1]
        if adapter >= 0 and hi > lo:
            t = s["x"][lo:hi].double() @ s["a"][adapter].double().t()
            y[lo:hi] += s["scale"][adapter].double() * (t @ s["b"][adapter].double().t())
    return {"y": y}
