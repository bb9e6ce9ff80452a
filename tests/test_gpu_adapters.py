"""Low-rank adapters added to a projection's output, on the GPU against the oracle.

Bound of an element: half a bf16 step of y (2^-8), and in fp32 roundings of 2^-24: t sums K exact products in pieces of 16
((K / 16 + 64) of the magnitudes |x||a|, carried through |b|); the second product adds the rank's terms (rank + 8 of |t||b|), and t
enters it as two bf16 terms (2^-16 of |t||b|)."""
import os

import numpy as np
import pytest
import torch

from oracle import around_oracle as ao
from paper_2607_23264_b200 import binding, inputs as gen
from moe_testlib import DEV, bits_to_dev, dev_bf16_to_f64

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module", params=["rule", "rows", "tiles"])
def ctx(request):
    """Every test runs three times: with the kernel that the sizes choose, and with either of them (calls without offsets have
    one kernel)."""
    before = os.environ.get("MOE_TUNING")
    if request.param != "rule":
        os.environ["MOE_TUNING"] = f"x.adapter_tiles={int(request.param == 'tiles')}"
    try:
        made = binding.Context(1, 64, 64, 1, 1)
    finally:
        if before is None:
            os.environ.pop("MOE_TUNING", None)
        else:
            os.environ["MOE_TUNING"] = before
    return made


def bf16(v):
    bits = gen.f32_to_bf16_bits(np.asarray(v, np.float32))
    return bits_to_dev(bits), gen.bf16_bits_to_f32(bits).astype(np.float64)


def i32(v):
    return None if v is None else torch.tensor(np.asarray(v, np.int32), device=DEV)


def make(seed, rows, N, K, rank, adapters, scaled=True):
    rng = np.random.default_rng(seed)
    p = dict(rows=rows, N=N, K=K, rank=rank, adapters=adapters)
    for name, v in (("x", rng.standard_normal((rows, K))), ("a", rng.standard_normal((adapters, rank, K)) / np.sqrt(K)),
                    ("b", rng.standard_normal((adapters, N, rank)) / np.sqrt(rank)), ("y", rng.standard_normal((rows, N)))):
        p[name], p[name + "v"] = bf16(v)
    p["scalev"] = (0.5 + rng.random(adapters)).astype(np.float32) if scaled else None
    p["scale"] = torch.from_numpy(p["scalev"]).to(DEV) if scaled else None
    return p, rng


def run(ctx, p, ids, offsets=None, y=None, out=None, scratch=None, stream=None):
    if out is None:
        out = torch.full((p["rows"], p["N"]), float("nan"), dtype=torch.bfloat16, device=DEV)
    if scratch is None:
        size = ctx.adapter_scratch_bytes(p["rows"], p["K"], p["rank"])
        scratch = torch.full((max(16, size),), 0xFF, dtype=torch.uint8, device=DEV)      # NaN where nothing is written
    idd, off = i32(ids), i32(offsets)
    ctx.moe_add_adapters(p["x"], p["a"], p["b"], idd, p["y"] if y is None else y, out, scratch, p["rows"], p["N"], p["K"],
                         p["rank"], p["adapters"], len(ids), offsets=off, scale=p["scale"], stream=stream)
    torch.cuda.synchronize()
    return out


def check(p, ids, offsets, out):
    ref, size_t, size_y = ao.add_adapters(p["xv"], p["av"], p["bv"], p["scalev"], ids, p["yv"], offsets)
    got = dev_bf16_to_f64(out)
    bound = 2.0 ** -8 * np.abs(ref) + (p["K"] / 16 + 64) * U * size_t + ((p["rank"] + 8) * U + 2.0 ** -16) * size_y
    err = np.abs(got - ref)
    assert (err <= bound).all(), (float((err / (bound + 1e-30)).max()), np.argwhere(err > bound)[:5])
    bounds = np.arange(p["rows"] + 1) if offsets is None else np.asarray(offsets)
    plain = np.ones(p["rows"], bool)
    for i, adapter in enumerate(ids):
        if 0 <= adapter < p["adapters"]:
            plain[bounds[i]:bounds[i + 1]] = False
    keep = torch.from_numpy(plain).to(DEV)
    assert torch.equal(out[keep].view(torch.int16), p["y"][keep].view(torch.int16))


def cut(rng, rows, segments, tail=0):
    """Offsets of uneven segments, some empty, the last `tail` rows behind them all."""
    cuts = np.sort(rng.integers(0, rows - tail + 1, segments - 1)) if segments > 1 else np.zeros(0, np.int64)
    return np.concatenate([[0], cuts, [rows - tail]])


@pytest.mark.parametrize("rows,N,K,rank,adapters", [
    (1, 8, 8, 8, 1), (1, 4096, 7168, 16, 3), (5, 72, 40, 8, 2), (16, 264, 128, 24, 4), (17, 520, 1000, 16, 5),
    (64, 4096, 7168, 16, 32), (100, 1032, 2056, 40, 7), (256, 512, 512, 64, 256), (33, 256, 4112, 128, 3), (300, 200, 96, 120, 11)])
def test_single_tokens(ctx, rows, N, K, rank, adapters):
    p, rng = make(rows + N, rows, N, K, rank, adapters)
    ids = rng.integers(-1 if rows > 4 else 0, adapters, rows)
    check(p, ids, None, run(ctx, p, ids))
    assert ctx.moe_last_device_status() == (0, 0)


@pytest.mark.parametrize("rows,N,K,rank,adapters,segments,tail", [
    (128, 256, 256, 16, 1, 1, 0), (129, 264, 264, 16, 2, 2, 0), (1000, 520, 1032, 64, 3, 4, 7), (700, 2104, 4112, 24, 9, 40, 0),
    (513, 136, 72, 8, 4, 300, 0), (2000, 384, 640, 128, 5, 9, 100), (1024, 1024, 512, 32, 1, 3, 0), (640, 72, 2048, 104, 6, 5, 3),
    (4096, 768, 768, 64, 40, 64, 0), (3000, 128, 128, 16, 500, 500, 1)])
def test_segments(ctx, rows, N, K, rank, adapters, segments, tail):
    p, rng = make(rows + K, rows, N, K, rank, adapters)
    offsets = cut(rng, rows, segments, tail)
    ids = rng.integers(-1 if segments > 2 else 0, adapters, segments)
    check(p, ids, offsets, run(ctx, p, ids, offsets))
    assert ctx.moe_last_device_status() == (0, 0)


@pytest.mark.parametrize("rows,N,K,rank,adapters,segments,tail", [
    (1, 8, 8, 8, 1, 1, 0), (15, 64, 64, 16, 2, 1, 3), (17, 72, 136, 24, 2, 2, 0), (127, 200, 520, 40, 3, 3, 0), (5000, 264, 264, 16, 3, 4, 9),
    (9000, 72, 72, 8, 2, 3, 1), (1100, 4096, 1032, 64, 2, 2, 0), (600, 1032, 4096, 128, 2, 3, 0), (300, 16, 8, 72, 3, 2, 5),
    (2300, 8, 512, 48, 4, 6, 0), (1030, 3000, 24, 56, 5, 3, 0)])
def test_long_segments_of_odd_sizes(ctx, rows, N, K, rank, adapters, segments, tail):
    p, rng = make(rows + rank, rows, N, K, rank, adapters)
    offsets = cut(rng, rows, segments, tail)
    ids = rng.integers(-1 if segments > 2 else 0, adapters, segments)
    check(p, ids, offsets, run(ctx, p, ids, offsets))


def test_segments_without_rows(ctx):
    """Many empty segments at the same row, in front, between and behind."""
    p, rng = make(12, 400, 136, 200, 16, 5)
    offsets = np.array([0] * 40 + [150] * 70 + [151, 151, 280] + [400] * 50)
    ids = rng.integers(0, 5, len(offsets) - 1)
    check(p, ids, offsets, run(ctx, p, ids, offsets))


def test_rows_behind_the_32nd_bit(ctx):
    """x and y of more than 2^32 bytes: the first and the last rows."""
    rows, N, K, rank = 280_000, 8192, 8192, 16
    x = torch.zeros(rows, K, dtype=torch.bfloat16, device=DEV)
    y = torch.zeros(rows, N, dtype=torch.bfloat16, device=DEV)
    rng = np.random.default_rng(13)
    q = dict(rows=rows, N=N, K=K, rank=rank, adapters=2, x=x, y=y, scale=None, scalev=None)
    for name, v in (("a", rng.standard_normal((2, rank, K)) / np.sqrt(K)), ("b", rng.standard_normal((2, N, rank)) / np.sqrt(rank))):
        q[name], q[name + "v"] = bf16(v)
    part = 130
    ends, values = bf16(rng.standard_normal((2 * part, K)))
    x[:part], x[-part:] = ends[:part], ends[part:]
    out = run(ctx, q, [0, 1], [0, rows // 2, rows], out=y)                          # in place
    got = torch.cat([out[:part], out[-part:]])
    few = dict(q, rows=2 * part, xv=values, yv=np.zeros((2 * part, N)), y=torch.zeros_like(got))
    check(few, [0, 1], [0, part, 2 * part], got)
    assert (out[part:-part] == 0).all()


def test_one_long_segment_among_single_rows(ctx):
    rows, adapters = 1200, 50
    p, rng = make(3, rows, 640, 1024, 16, adapters)
    counts = [1] * 30 + [1000] + [1] * 80 + [0, 0, 87] + [1] * 3
    offsets = np.concatenate([[0], np.cumsum(counts)])
    ids = rng.integers(0, adapters, len(counts))
    ids[5], ids[20] = -1, -9
    check(p, ids, offsets, run(ctx, p, ids, offsets))


@pytest.mark.parametrize("rows,segments", [(40, 40), (900, 3)])
def test_in_place_without_scale_and_repeated(ctx, rows, segments):
    p, rng = make(4, rows, 328, 520, 24, 5, scaled=False)
    offsets = None if segments == rows else cut(rng, rows, segments)
    ids = rng.integers(-1, 5, segments)
    want = run(ctx, p, ids, offsets)
    check(p, ids, offsets, want)
    for _ in range(3):
        assert torch.equal(run(ctx, p, ids, offsets).view(torch.int16), want.view(torch.int16))
    y = p["y"].clone()
    run(ctx, p, ids, offsets, y=y, out=y)
    assert torch.equal(y.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("rows,segments", [(20, 20), (600, 4)])
def test_no_adapter_and_no_segment_copy_every_bit(ctx, rows, segments):
    p, rng = make(5, rows, 136, 72, 8, 2)
    p["y"][0, 0], p["y"][1, 1], p["y"][2, 2] = float("nan"), -0.0, float("inf")
    offsets = None if segments == rows else cut(rng, rows, segments)
    out = run(ctx, p, [-1] * segments, offsets)
    assert torch.equal(out.view(torch.int16), p["y"].view(torch.int16))
    out = run(ctx, p, [], [0])
    assert torch.equal(out.view(torch.int16), p["y"].view(torch.int16))


@pytest.mark.parametrize("rows,segments", [(20, 20), (600, 4)])
def test_indices_out_of_range_are_reported(ctx, rows, segments):
    p, rng = make(6, rows, 136, 72, 8, 2)
    offsets = None if segments == rows else np.array([0, 100, 101, 400, 600])
    ids = [0] * segments
    ids[2] = 2
    out = run(ctx, p, ids, offsets)
    assert ctx.moe_last_device_status() == (4, 2)
    check(p, ids, offsets, out)
    ids[2] = 2 ** 31 - 1
    check(p, ids, offsets, run(ctx, p, ids, offsets))
    assert ctx.moe_last_device_status() == (4, 2)


@pytest.mark.parametrize("rows,segments", [(32, 32), (512, 4)])
def test_values_that_are_not_numbers_stay_in_their_rows(ctx, rows, segments):
    p, rng = make(7, rows, 200, 264, 16, 3)
    offsets = None if segments == rows else np.array([0, 130, 200, 300, 512])
    ids = np.arange(segments) % 3
    want = run(ctx, p, ids, offsets)
    bad = {0: 0, 17: 17, 31: 31} if segments == rows else {5: 5, 131: 131, 511: 511}
    row = list(bad)
    p["x"][row[0], 3], p["x"][row[1], 263], p["x"][row[2], 100] = float("nan"), float("inf"), -float("inf")
    out = run(ctx, p, ids, offsets)
    good = torch.ones(rows, dtype=torch.bool, device=DEV)
    good[row] = False
    assert torch.equal(out[good].view(torch.int16), want[good].view(torch.int16))
    assert not out[row].isfinite().any()
    # an adapter of NaN spoils its own requests alone
    p, rng = make(7, rows, 200, 264, 16, 3)
    p["a"][1, 2, 5] = float("nan")
    out = run(ctx, p, ids, offsets)
    own = torch.from_numpy(np.repeat(ids, 1 if offsets is None else np.diff(offsets)) == 1).to(DEV)
    assert out[own].isnan().all() and torch.equal(out[~own].view(torch.int16), want[~own].view(torch.int16))


@pytest.mark.parametrize("rows,segments", [(24, 24), (700, 3)])
def test_input_gradient_by_exchanged_factors(ctx, rows, segments):
    """d_x of y = x + scale b (a x): the call on d_y with the factors exchanged, against differences of the oracle."""
    p, rng = make(8, rows, 96, 160, 16, 3)
    offsets = None if segments == rows else cut(rng, rows, segments)
    ids = rng.integers(0, 3, segments)
    d, dv = bf16(rng.standard_normal((rows, 96)))
    back = dict(rows=rows, N=160, K=96, rank=16, adapters=3, x=d, xv=dv, a=p["b"].transpose(1, 2).contiguous(),
                av=p["bv"].transpose(0, 2, 1), b=p["a"].transpose(1, 2).contiguous(), bv=p["av"].transpose(0, 2, 1),
                y=torch.zeros(rows, 160, dtype=torch.bfloat16, device=DEV), yv=np.zeros((rows, 160)), scale=p["scale"],
                scalev=p["scalev"])
    dx = run(ctx, back, ids, offsets)
    check(back, ids, offsets, dx)
    f = lambda v: (ao.add_adapters(v, p["av"], p["bv"], p["scalev"], ids, p["yv"], offsets)[0] * dv).sum(1)  # noqa: E731
    for c in (0, 77, 159):
        up, down = p["xv"].copy(), p["xv"].copy()
        up[:, c] += 0.5
        down[:, c] -= 0.5
        num, got = f(up) - f(down), dev_bf16_to_f64(dx)[:, c]
        assert (np.abs(num - got) <= 2.0 ** -8 * np.abs(num) + 1e-3 * np.abs(dv).max()).all()


@pytest.mark.parametrize("rows,segments", [(48, 48), (1500, 6)])
def test_two_graphs_with_their_own_scratch(ctx, rows, segments):
    p, rng = make(9, rows, 520, 776, 32, 4)
    offsets = None if segments == rows else cut(rng, rows, segments)
    ids = rng.integers(-1, 4, segments)
    want = run(ctx, p, ids, offsets)
    idd, off = i32(ids), i32(offsets)
    side, held = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for s in side:
        scratch = torch.empty(ctx.adapter_scratch_bytes(rows, p["K"], p["rank"]), dtype=torch.uint8, device=DEV)
        out, g = torch.empty_like(want), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            ctx.moe_add_adapters(p["x"], p["a"], p["b"], idd, p["y"], out, scratch, rows, p["N"], p["K"], p["rank"],
                                 p["adapters"], segments, offsets=off, scale=p["scale"])
        held.append((g, out, scratch))
    for _ in range(5):
        for (g, out, _), s in zip(held, side):
            with torch.cuda.stream(s):
                out.zero_()
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out.view(torch.int16), want.view(torch.int16)) for _, out, _ in held)


def test_refusals(ctx):
    rows, N, K, rank = 8, 64, 64, 16
    p, _ = make(10, rows, N, K, rank, 2)
    ids = torch.zeros(rows, dtype=torch.int32, device=DEV)
    out = torch.zeros_like(p["y"])
    scratch = torch.zeros(ctx.adapter_scratch_bytes(rows, K, rank), dtype=torch.uint8, device=DEV)
    good = dict(x=p["x"], a=p["a"], b=p["b"], adapter_of=ids, y_in=p["y"], y_out=out, scratch=scratch, rows=rows, N=N, K=K,
                rank=rank, adapters=2, segments=rows)
    odd = torch.zeros(rows * N + 8, dtype=torch.bfloat16, device=DEV)[1:rows * N + 1]
    for change, code in [(dict(x=None), 1), (dict(a=None), 1), (dict(b=None), 1), (dict(adapter_of=None), 1), (dict(y_in=None), 1),
                         (dict(y_out=None), 1), (dict(N=60), 2),
                         (dict(K=4), 2), (dict(rank=12), 2), (dict(rank=136), 2), (dict(rank=0), 2), (dict(adapters=0), 2),
                         (dict(segments=rows + 1), 2), (dict(segments=3), 1), (dict(rows=-1), 2), (dict(segments=-1), 2),
                         (dict(adapters=2 ** 27), 2), (dict(y_in=odd), 1), (dict(scale=torch.zeros(8, device=DEV)[1:3]), 1),
                         (dict(offsets=torch.zeros(12, dtype=torch.int32, device=DEV)[1:10]), 1)]:
        with pytest.raises(binding.MoeError) as err:
            ctx.moe_add_adapters(**{**good, **change})
        assert err.value.code == code, change
    ctx.moe_add_adapters(**{**good, "rows": 0, "segments": 0})
    assert ctx.moe_last_launch_count() == 0
    assert ctx.adapter_scratch_bytes(8, 12, 8) == 0 and ctx.adapter_scratch_bytes(8, 16, 256) == 0
