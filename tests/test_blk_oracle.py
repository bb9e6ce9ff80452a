"""Pins of the oracle for FP8 in blocks of 128."""
import numpy as np

from oracle import blk_oracle as blk
from oracle import fp8_oracle as f8


def test_single_block_rows_are_the_per_row_scheme():
    rng = np.random.default_rng(0)
    v = rng.standard_normal((5, 96)).astype(np.float32)
    v[2] = 0.0
    codes, scales = blk.quantize_rows(v)
    ref_c, ref_s = f8.quantize_rows(v)
    assert np.array_equal(codes, ref_c) and np.array_equal(scales[0], ref_s) and scales[0, 2] == 1.0


def test_blocks_are_independent_and_short_blocks_count():
    rng = np.random.default_rng(1)
    v = rng.standard_normal((3, 272)).astype(np.float32)
    codes, scales = blk.quantize_rows(v)
    assert scales.shape == (3, 3)
    loud = v.copy()
    loud[:, 256:] *= 100                                   # the short last block only
    c2, s2 = blk.quantize_rows(loud)
    assert np.array_equal(c2[:, :256], codes[:, :256]) and np.array_equal(s2[:2], scales[:2]) and (s2[2] > scales[2]).all()
    w = rng.standard_normal((200, 144)).astype(np.float32)
    wc, ws = blk.quantize_weights(w)
    assert ws.shape == (2, 2)
    one_c, one_s = blk.quantize_weights(w[128:, 128:])
    assert np.array_equal(wc[128:, 128:], one_c) and ws[1, 1] == one_s[0, 0]
    # each value is within half an E4M3 step (2^-4 of it, or 2^-10 of the block's scale) of what it was
    err = np.abs(blk.dequantize_weights(wc, ws) - w)
    full = np.repeat(np.repeat(ws, 128, 0), 128, 1)[:200, :144]
    assert (err <= np.abs(w) * 2.0 ** -4 * 1.001 + full * 2.0 ** -10).all()


def test_product_against_scalar_loops():
    rng = np.random.default_rng(2)
    a, w = rng.standard_normal((2, 144)).astype(np.float32), rng.standard_normal((130, 144)).astype(np.float32)
    ac, sa = blk.quantize_rows(a)
    wc, sw = blk.quantize_weights(w)
    got = blk.gemm(ac, sa, wc, sw)
    val = f8.e4m3_decode(np.arange(256, dtype=np.uint8))
    for r in range(2):
        for n in (0, 1, 127, 128, 129):
            total = 0.0
            for k in range(144):
                total += val[ac[r, k]] * float(sa[k // 128, r]) * val[wc[n, k]] * float(sw[n // 128, k // 128])
            assert abs(total - got[r, n]) < 1e-9
