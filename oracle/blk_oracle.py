"""CPU oracle for FP8 in blocks of 128.  TEST INFRASTRUCTURE ONLY.

E4M3 codes with one fp32 scale per block: 1 x 128 along the columns for rows, 128 x 128 for weights; the last block may
be short.  scale = fp32(amax) / 448 (1 for an all-zero block), code = convert(fp32(value) / scale); these decisions are
taken in fp32, the precision of the kernels, so that codes and scales compare bit for bit; products are fp64.  Format and
conversion are those of ``fp8_oracle``.  Row scales are returned as [blocks][rows], weight scales as [row blocks][column
blocks].

Pins (tests/test_blk_oracle.py): a scalar brute-force product, block independence, the distance to unquantised values,
and single-block cases against ``fp8_oracle``.
"""
from __future__ import annotations

import numpy as np

from oracle import fp8_oracle as f8
from oracle import moe_oracle as orc


def _scale(amax: np.ndarray) -> np.ndarray:
    amax = np.asarray(amax, dtype=np.float32)
    return np.where(amax > 0, amax / np.float32(448.0), np.float32(1.0)).astype(np.float32)


def _blocks(n: int):
    return [(b, min(b + 128, n)) for b in range(0, n, 128)]


def quantize_rows(values: np.ndarray):
    """[rows, cols] -> codes uint8 [rows, cols], scales fp32 [ceil(cols/128), rows]."""
    v = np.asarray(values, dtype=np.float32)
    codes = np.zeros(v.shape, dtype=np.uint8)
    spans = _blocks(v.shape[1])
    scales = np.ones((len(spans), v.shape[0]), dtype=np.float32)
    for b, (lo, hi) in enumerate(spans):
        scales[b] = _scale(np.abs(v[:, lo:hi]).max(axis=1))
        codes[:, lo:hi] = f8.e4m3_encode((v[:, lo:hi] / scales[b][:, None]).astype(np.float32))
    return codes, scales


def quantize_weights(values: np.ndarray):
    """[N, K] -> codes uint8 [N, K], scales fp32 [ceil(N/128), ceil(K/128)]."""
    v = np.asarray(values, dtype=np.float32)
    codes = np.zeros(v.shape, dtype=np.uint8)
    rows, cols = _blocks(v.shape[0]), _blocks(v.shape[1])
    scales = np.ones((len(rows), len(cols)), dtype=np.float32)
    for i, (r0, r1) in enumerate(rows):
        for j, (c0, c1) in enumerate(cols):
            scales[i, j] = _scale(np.abs(v[r0:r1, c0:c1]).max())
            codes[r0:r1, c0:c1] = f8.e4m3_encode((v[r0:r1, c0:c1] / scales[i, j]).astype(np.float32))
    return codes, scales


def dequantize_rows(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    return f8.e4m3_decode(codes) * np.repeat(np.asarray(scales, np.float64), 128, axis=0)[: codes.shape[1]].T


def dequantize_weights(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    full = np.repeat(np.repeat(np.asarray(scales, np.float64), 128, axis=0), 128, axis=1)
    return f8.e4m3_decode(codes) * full[: codes.shape[0], : codes.shape[1]]


def gemm(a_codes, a_scales, w_codes, w_scales) -> np.ndarray:
    """out[r, n] = sum_k a[r, k] w[n, k] of the dequantised operands, fp64."""
    return dequantize_rows(a_codes, a_scales) @ dequantize_weights(w_codes, w_scales).T


def magnitude(a_codes, a_scales, w_codes, w_scales) -> np.ndarray:
    """sum_k |a[r, k] w[n, k]|: what a rounding error of the sums is relative to."""
    return np.abs(dequantize_rows(a_codes, a_scales)) @ np.abs(dequantize_weights(w_codes, w_scales)).T


def expert_rows(xq, sx, gate, up):
    """h of one expert's rows, fp64, before its quantisation.  gate, up: (codes, scales)."""
    return orc.silu(gemm(xq, sx, *gate)) * gemm(xq, sx, *up)
