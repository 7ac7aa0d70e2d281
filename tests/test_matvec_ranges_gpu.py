"""mxfp8_e2m1_matvec by ranges of the scale bytes, against the oracle: tiles whose bytes all lie in 64 .. 127 fold the scales into
the weights and chain a tile's eight tensor instructions, all others keep a part of every scale for the sums.  Every variant
of the kernel, with as many warps to a row group as the size gives it."""
import numpy as np
import pytest

import oracle as orc
from paper_2506_08027_b200 import synth
from test_matvec_gpu import dev, run

pytestmark = pytest.mark.gpu

TABLE = np.array([orc.fp8_decode(c, orc.E2M1) for c in range(16)])


def pack(codes, scales):
    import torch
    from paper_2506_08027_b200 import binding as B
    matrices, rows, cols = codes.shape
    slots = np.zeros((matrices * rows, cols // 16, 16), np.uint8)
    flat = codes.reshape(slots.shape)
    slots[:, :, :8] = flat[:, :, 0::2] | flat[:, :, 1::2] << 4
    packed = torch.empty(B.mxfp8_e2m1_packed_bytes(matrices, rows, cols), dtype=torch.uint8, device="cuda")
    B.mxfp8_e2m1_pack(dev(slots.reshape(-1, cols)), dev(scales.reshape(-1)), matrices, packed)
    return packed


def weights(matrices, rows, cols, low, high, seed):
    """Codes and scale bytes low .. high - 1; says whether some pairs of row tiles (and so every single one of them) have
    all their bytes in 64 .. 127 or outside."""
    rng = np.random.default_rng(seed)
    codes = rng.integers(0, 16, (matrices, rows, cols), dtype=np.uint8)
    scales = rng.integers(low, high, (matrices, rows, cols // 32), dtype=np.uint8)
    r, k = rows // 32 * 32, cols // 128 * 4
    tiles = scales[:, :r, :k].reshape(matrices, r // 32, 32, k // 4, 4)
    fast = ((tiles >= 64) & (tiles <= 127)).all(axis=(2, 4))
    return pack(codes, scales), codes, scales, fast


def check(y, want, mag, cols, out):
    """Products are exact.  At worst each of the 17 additions of a tensor instruction (16 products and the accumulator) loses a
    whole step of the running magnitude, 2^-23.  A tile of 128 columns chains eight instructions (scales folded) or two per
    group of 32 columns; every tile, or every group, is added once (half a step), and so are at most eight warps' parts; last
    comes the output's own rounding, half a step."""
    sums = (2 * 8 * 17 + cols / 32 + 8) * 2.0 ** -24 * mag
    err = np.abs(y - want)
    assert (err <= sums + (2.0 ** -8 if out == "bf16" else 2.0 ** -24) * (np.abs(want) + sums) + 2.0 ** -133).all(), (err / (mag + 1e-300)).max()


RANGES = [(64, 128, "all"), (117, 122, "all"), (100, 140, "none"), (63, 128, "some")]


@pytest.mark.parametrize("low,high,fast_tiles", RANGES)
@pytest.mark.parametrize("tokens", [1, 8, 9, 16, 17, 33, 64])
@pytest.mark.parametrize("rows,cols", [(64, 128), (96, 2048), (77, 1184), (18976, 288)])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_one_matrix(low, high, fast_tiles, tokens, rows, cols, out):
    """8, 16 or 32 tokens at a time, few row tiles and many (18976 rows), whole tiles and ragged edges."""
    packed, codes, scales, fast = weights(1, rows, cols, low, high, rows + cols)
    assert fast.all() if fast_tiles == "all" else not fast.any() if fast_tiles == "none" else True
    x, y = run(synth.student_t((tokens, cols), tokens), packed, 1, None, rows, out)
    want, mag = orc.matvec_f64(x, codes, scales)
    check(y, want, mag, cols, out)


@pytest.mark.parametrize("low,high", [(64, 128), (117, 122), (100, 140)])
@pytest.mark.parametrize("tokens,choices,matrices", [(1, 1, 2), (8, 6, 64), (40, 2, 3), (33, 6, 5), (200, 5, 4), (1024, 1, 2)])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_chosen_matrices(low, high, tokens, choices, matrices, out):
    """More and fewer matrices than slots, matrices with many times eight slots, numbers that name none."""
    rows, cols = 64, 384
    rng = np.random.default_rng(tokens)
    ids = rng.integers(-1, matrices + 1, (tokens, choices)).astype(np.int32)
    packed, codes, scales, fast = weights(matrices, rows, cols, low, high, 7)
    assert fast.all() == (high <= 128)
    x, y = run(synth.gaussian((tokens, cols), 2), packed, matrices, ids, rows, out)
    want, mag = orc.matvec_f64(x, codes, scales, ids)
    check(y, want, mag, cols, out)
    assert not y[(ids.reshape(-1) < 0) | (ids.reshape(-1) >= matrices)].any()


@pytest.mark.parametrize("rows,cols,tokens", [(75823, 416, 8), (75823, 416, 16), (75823, 416, 33), (40016, 416, 33), (75776, 96, 8)])
@pytest.mark.parametrize("low,high", [(117, 122), (100, 140)])
def test_one_matrix_whose_row_groups_have_fewer_warps(rows, cols, tokens, low, high):
    """So many row tiles that two warps or one walk all columns of a row group (40016 rows: two of four for 32 tokens at a
    time and four for fewer; 75776 and more: one)."""
    packed, codes, scales, _ = weights(1, rows, cols, low, high, rows)
    x, y = run(synth.student_t((tokens, cols), tokens), packed, 1, None, rows, "fp32")
    want, mag = orc.matvec_f64(x, codes, scales)
    check(y, want, mag, cols, "fp32")


@pytest.mark.parametrize("rows,cols", [(768, 416), (1536, 416), (1552, 288)])
@pytest.mark.parametrize("low,high", [(117, 122), (100, 140)])
@pytest.mark.parametrize("by_matrix", [False, True])
def test_chosen_matrices_whose_row_groups_have_fewer_warps(rows, cols, low, high, by_matrix):
    """100 CTA columns, one per slot or one per matrix: two warps to a row group of 768-row matrices, one of 1536 rows and more."""
    matrices, tokens, choices = (100, 67, 3) if by_matrix else (130, 50, 2)
    rng = np.random.default_rng(rows)
    ids = rng.integers(0, matrices, (tokens, choices)).astype(np.int32)
    ids[rng.random(ids.shape) < 0.1] = -1
    packed, codes, scales, _ = weights(matrices, rows, cols, low, high, 9)
    x, y = run(synth.gaussian((tokens, cols), 2), packed, matrices, ids, rows, "bf16")
    want, mag = orc.matvec_f64(x, codes, scales, ids)
    check(y, want, mag, cols, "bf16")


@pytest.mark.parametrize("rows", [1024, 18944])
@pytest.mark.parametrize("tokens", [8, 16, 128])
def test_every_code_under_every_folded_scale(rows, tokens):
    """One scale byte 64 .. 127 per row tile, so that it is folded; single products, bit for bit.  Row r of a tile holds code
    (column + r) mod 16."""
    cols = 128
    codes = ((np.arange(cols)[None, :] + np.arange(rows)[:, None]) % 16).astype(np.uint8)[None]
    b = 64 + np.arange(rows) // 16 % 64
    scales = np.repeat(b.astype(np.uint8)[None, :, None], cols // 32, axis=2)
    packed = pack(codes, scales)
    for magnitude in (1.0, 2.0 ** -60, 1.5 * 2.0 ** 60):
        for first in range(0, cols, tokens) if tokens > 16 else (0, 40, cols - tokens):
            x = np.zeros((tokens, cols), np.float32)
            x[np.arange(tokens), np.arange(tokens) + first] = magnitude
            _, y = run(x, packed, 1, None, rows, "fp32")
            want = TABLE[codes[0].T[first:first + tokens]] * np.exp2(b - 127.0) * magnitude
            assert np.array_equal(y, want)


@pytest.mark.parametrize("other", [127, 0, 200])
def test_large_activations_under_small_scales(other):
    """Sums that would pass FP32's range before their scale and do not after it.  One byte of the last row decides which way
    the tile takes: with 127 all its bytes lie in 64 .. 127."""
    rows, cols = 16, 256
    bytes_of_rows = np.array([64, 65, 66, 70, 80, 90, 95, 100, 105, 110, 112, 114, 116, 117, 117, other], np.uint8)
    codes = np.full((1, rows, cols), 7, np.uint8)               # 6.0
    codes[:, :, 1::3] = 15                                      # -6.0
    scales = np.repeat(bytes_of_rows.reshape(1, rows, 1), cols // 32, axis=2)
    x, y = run(np.full((3, cols), 1.5 * 2.0 ** 126), pack(codes, scales), 1, None, rows, "fp32")
    want, mag = orc.matvec_f64(x, codes, scales)
    assert mag[:, :15].max() < 2.0 ** 128 < mag[0, 0] * 2.0 ** 63
    check(y[:, :15], want[:, :15], mag[:, :15], cols, "fp32")
