"""Adapters where it can go wrong: ends of segments inside a tile's slabs, elements that are not finite.  Bounds are those of test_gpu_adapters."""
import os

import numpy as np
import pytest
import torch

from moe_testlib import DEV, dev_bf16_to_f64
from oracle import around_oracle as ao
from paper_2607_23264_b200 import binding
from test_gpu_adapters import U, bf16, check, make, run

pytestmark = pytest.mark.gpu


def context(kernel):
    before = os.environ.get("MOE_TUNING")
    os.environ["MOE_TUNING"] = f"x.adapter_tiles={int(kernel == 'tiles')}"
    try:
        return binding.Context(1, 64, 64, 1, 1)
    finally:
        if before is None:
            os.environ.pop("MOE_TUNING", None)
        else:
            os.environ["MOE_TUNING"] = before


@pytest.fixture(scope="module")
def contexts():
    return {kernel: context(kernel) for kernel in ("rows", "tiles")}


@pytest.fixture(scope="module")
def tiles(contexts):
    return contexts["tiles"]


@pytest.mark.parametrize("rank", [16, 64, 128])
@pytest.mark.parametrize("bounds", [[0, 45, 173, 300], [0, 1, 34, 161, 288, 300], [0, 97]])
def test_a_segments_end_over_many_tiles_of_columns(tiles, rank, bounds):
    """The last rows of a segment fill a part of 32; with more tiles of columns to a CTA (8, or 9 with N = 4104) than it keeps in
    flight (4, and 6 above 64 ranks) the place of that part is loaded again and again, in place too."""
    rows, N = bounds[-1], 4104
    p, rng = make(rank + rows, rows, N, 264, rank, 3)
    ids = rng.integers(0, 3, len(bounds) - 1)
    want = run(tiles, p, ids, bounds)
    check(p, ids, bounds, want)
    for _ in range(10):
        y = p["y"].clone()
        run(tiles, p, ids, bounds, y=y, out=y)
        assert torch.equal(y.view(torch.int16), want.view(torch.int16))
    assert tiles.moe_last_device_status() == (0, 0)


def compare(p, ids, offsets, out):
    """NaN and infinities where the formula has them, the bound elsewhere."""
    with np.errstate(invalid="ignore", over="ignore"):
        ref, size_t, size_y = ao.add_adapters(p["xv"], p["av"], p["bv"], p["scalev"], ids, p["yv"], offsets)
        got = dev_bf16_to_f64(out)
        bound = 2.0 ** -8 * np.abs(ref) + (p["K"] / 16 + 64) * U * size_t + ((p["rank"] + 8) * U + 2.0 ** -16) * size_y
        fine = np.isfinite(ref)
        assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)])
        assert (np.abs(got - ref) <= bound)[fine].all()
    return ref


BOTH = [(kernel, *case) for kernel in ("rows", "tiles") for case in (
    (300, 200, 264, 24, [0, 140, 141, 300]), (140, 520, 72, 128, [0, 140]), (530, 72, 264, 16, [0, 10, 522, 530]))]


@pytest.mark.parametrize("kernel,rows,N,K,rank,bounds", BOTH + [          # without offsets there is one kernel
    ("rows", 24, 72, 264, 8, None), ("rows", 300, 200, 264, 16, None), ("rows", 64, 136, 40, 64, None),
    ("rows", 40, 136, 264, 128, None)])
def test_factors_that_are_not_finite(contexts, kernel, rows, N, K, rank, bounds):
    """t is a whole number of up to 12 bits: its second bf16 term is zero or of either sign, and an infinite element of b must
    still give an infinity of t's sign, NaN only for t = 0."""
    ctx = contexts[kernel]
    p, rng = make(rows + rank, rows, N, K, rank, 3)
    for name, v in (("x", rng.integers(-8, 9, (rows, K))), ("a", rng.integers(-8, 9, (3, rank, K)))):
        p[name], p[name + "v"] = bf16(v)
    p["x"][::7], p["xv"][::7] = 0, 0
    p["scalev"] = np.array([1, 0.5, 2], np.float32)
    p["scale"] = torch.from_numpy(p["scalev"]).to(DEV)
    b = p["bv"].copy()
    b[0, 3, 1], b[0, 8, 7], b[1, N - 1, 0], b[1, 17, rank - 1], b[2, 0, 2] = np.inf, -np.inf, np.inf, -np.inf, np.nan
    b[2, 40, 3], b[2, 40, 4] = np.inf, -np.inf
    p["b"], p["bv"] = bf16(b)
    p["y"][0, 1], p["yv"][0, 1] = float("nan"), np.nan
    p["y"][1, 3], p["yv"][1, 3] = float("-inf"), -np.inf
    ids = np.arange(rows if bounds is None else len(bounds) - 1) % 3
    out = run(ctx, p, ids, bounds)
    ref = compare(p, ids, bounds, out)
    assert np.isinf(ref).any() and np.isnan(ref).any()
    y = p["y"].clone()
    run(ctx, p, ids, bounds, y=y, out=y)
    assert torch.equal(y.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("kernel,bounds", [("rows", None), ("rows", [0, 20, 150]), ("tiles", [0, 20, 150])])
def test_sums_beyond_the_largest_bf16(contexts, kernel, bounds):
    """A sum of x a that fp32 holds and a rounding to bf16 would make infinite."""
    rows, N, K, rank = 150, 136, 72, 24
    p, rng = make(1, rows, N, K, rank, 2, scaled=False)
    x, a, b = p["xv"], p["av"], 2.0 ** -100 * p["bv"]
    x[:, :2] = 0
    x[5], x[149] = 0, 0
    x[5, :2], x[149, :2] = 2.0 ** 64, -2.0 ** 64
    a[:, 4, 0], a[:, 4, 1] = 1.9921875 * 2.0 ** 63, 1.5 * 2.0 ** 55       # the largest bf16 and three quarters of its step
    b[:, 7, 4] = 0
    for name, v in (("x", x), ("a", a), ("b", b)):
        p[name], p[name + "v"] = bf16(v)
    ids = np.arange(rows) % 2 if bounds is None else [0, 1]
    ref = compare(p, ids, bounds, run(contexts[kernel], p, ids, bounds))
    assert np.isfinite(ref).all() and np.abs(ref).max() > 1e6
