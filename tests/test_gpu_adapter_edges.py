"""Adapters where it can go wrong: ends of segments inside a tile's slabs.  Bounds are those of test_gpu_adapters."""
import os

import numpy as np
import pytest
import torch

from paper_2607_23264_b200 import binding
from test_gpu_adapters import check, make, run

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


@pytest.fixture(scope="module", params=["rows", "tiles"])
def ctx(request):
    """Calls with offsets have two kernels: both."""
    return context(request.param)


@pytest.fixture(scope="module")
def tiles():
    return context("tiles")


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
