"""Arithmetic that has to be exact, on the GPU: the reciprocal behind the choice of experts, the division behind E4M3 codes.

Helpers of the library's headers are compared with the general operations in a small library of their own
(exact_arithmetic.cu); the quantisation calls with the oracle, on every pair of bf16 mantissas of a block's maximum and a
value of it."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import blk_oracle as blk
from paper_2607_23264_b200 import binding, build, inputs as gen
from moe_testlib import DEV, bits_to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def exact(tmp_path_factory):
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "exact_arithmetic.cu")
    out = str(tmp_path_factory.mktemp("exact") / "libexact.so")
    try:
        subprocess.run([build._nvcc(), *build.NVCC_FLAGS, "-shared", src, "-o", out], check=True, capture_output=True, text=True)
    except FileNotFoundError:
        pytest.skip("no nvcc here")
    lib = ctypes.CDLL(out)
    for name in ("exact_reciprocals", "exact_sigmoids", "exact_quotients", "exact_codes"):
        getattr(lib, name).restype = ctypes.c_longlong
    return lib


@pytest.mark.parametrize("exponent", [0, 1, 2, 37, 63, 115])
def test_reciprocal_of_every_mantissa(exact, exponent):
    assert exact.exact_reciprocals(exponent) == 0


def test_sigmoid_without_branches(exact):
    assert exact.exact_sigmoids() == 0


def test_quotients(exact):
    """2^32 pairs of a value and a scale."""
    for part in range(16):
        assert exact.exact_quotients(part) == 0, part


@pytest.mark.parametrize("seed", [1, 2, 3, 4])
def test_codes_where_codes_end(exact, seed):
    """A million scales with the values next to every midpoint of two codes."""
    assert exact.exact_codes(seed) == 0


def mantissa_pairs(exponent):
    """Rows of three blocks: for each bf16 mantissa of the block's maximum (2^exponent x 1.m) and each distance in exponents,
    the values of all mantissas and both signs, as far as they are not above the maximum."""
    m = 1 + np.arange(128) / 128
    rows = []
    for distance in range(0, 22):
        v = np.ldexp(m, -distance)
        v = np.concatenate([v, -v])
        for top in m:
            row = np.zeros((3, 128))
            row[:, 0] = top
            row[:, 1:].flat[:256] = np.where(np.abs(v) <= top, v, 0.0)
            rows.append(row.reshape(-1))
    with np.errstate(under="ignore"):
        return gen.f32_to_bf16_bits(np.ldexp(np.stack(rows), exponent).astype(np.float32))


@pytest.mark.parametrize("exponent", [0, 3, -20, -80, -81, -82, -91, 108, 109, 110, 127, -110, -126, -131])
def test_quantise_every_pair_of_mantissas(exponent):
    """Scales from subnormal to the largest: both ways of dividing and the limits between them, bit for bit."""
    ctx = binding.Context(1, 64, 64, 1, 1)
    bits = mantissa_pairs(exponent)
    rows, cols = bits.shape
    values = gen.bf16_bits_to_f32(bits)
    assert np.isfinite(values).all()
    codes = torch.full((rows, cols), 0x7F, dtype=torch.uint8, device=DEV)
    scales = torch.full((cols // 128, rows), float("nan"), device=DEV)
    x = bits_to_dev(bits)
    ctx.moe_quantize_rows_blk(x, rows, cols, codes, scales)
    torch.cuda.synchronize()
    ref_c, ref_s = blk.quantize_rows(values)
    assert np.array_equal(scales.cpu().numpy(), ref_s)
    assert np.array_equal(codes.cpu().numpy(), ref_c)
    # one row per matrix: the same blocks by the weights' kernel
    codes.fill_(0x7F)
    by_row = torch.full((rows, 1, cols // 128), float("nan"), device=DEV)
    ctx.moe_quantize_weights_blk(x, rows, 1, cols, codes, by_row)
    torch.cuda.synchronize()
    assert np.array_equal(by_row[:, 0].t().cpu().numpy(), ref_s)
    assert np.array_equal(codes.cpu().numpy(), ref_c)
