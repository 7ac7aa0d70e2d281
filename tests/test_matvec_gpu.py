"""mxfp8_e2m1_pack and mxfp8_e2m1_matvec (products of a few tokens with MXFP4 matrices) against the oracle."""
import numpy as np
import pytest

import oracle as orc
from paper_2506_08027_b200 import synth

pytestmark = pytest.mark.gpu


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def packed_weights(w, matrices):
    """Converted and packed by the library; (packed, codes [m, rows, cols], scales) of the same conversion."""
    import torch
    from paper_2506_08027_b200 import binding as B
    total, cols = w.shape
    src = dev(w.astype(np.float32)).to(torch.bfloat16)
    q, s, _, _ = B.alloc_quantize_outputs(total, cols, B.ROW, B.SF_LINEAR)
    B.mxfp8_quantize(src, B.ROW, B.RULE_PAPER, B.E2M1, q, s, None, None, B.SF_LINEAR)
    packed = torch.full((B.mxfp8_e2m1_packed_bytes(matrices, total // matrices, cols),), 0xA5, dtype=torch.uint8, device="cuda")
    B.mxfp8_e2m1_pack(q, s, matrices, packed)
    codes = orc.unpack_codes16(q.cpu().numpy(), orc.E2M1)
    return packed, codes.reshape(matrices, -1, cols), s.cpu().numpy().reshape(matrices, -1, cols // 32)


def random_weights(matrices, rows, cols, seed, low=100, high=140):
    """Codes and scales drawn directly, laid out by the oracle's statement of the layout or the library's pack kernel."""
    import torch
    from paper_2506_08027_b200 import binding as B
    rng = np.random.default_rng(seed)
    codes = rng.integers(0, 16, (matrices, rows, cols)).astype(np.uint8)
    scales = rng.integers(low, high, (matrices, rows, cols // 32)).astype(np.uint8)
    flat = codes.reshape(-1, cols // 16, 16)
    slots = np.zeros_like(flat)
    slots[:, :, :8] = flat[:, :, 0::2] | flat[:, :, 1::2] << 4
    packed = torch.empty(B.mxfp8_e2m1_packed_bytes(matrices, rows, cols), dtype=torch.uint8, device="cuda")
    B.mxfp8_e2m1_pack(dev(slots.reshape(-1, cols)), dev(scales.reshape(-1)), matrices, packed)
    return packed, codes, scales


def run(x, packed, matrices, ids, rows, out):
    import torch
    from paper_2506_08027_b200 import binding as B
    xd = dev(x.astype(np.float32)).to(torch.bfloat16)
    slots = x.shape[0] * (1 if ids is None else ids.shape[1])
    y = torch.full((slots, rows), float("nan"), dtype=torch.bfloat16 if out == "bf16" else torch.float32, device="cuda")
    B.mxfp8_e2m1_matvec(xd, packed, matrices, None if ids is None else dev(ids), y)
    assert B.mxfp8_device_status() == 0
    return xd.float().cpu().numpy(), y.double().cpu().numpy()


def check(y, want, mag, cols, out):
    """Products of a BF16 and an E2M1 value are exact.  At worst every addition inside a tensor instruction loses a whole step
    of the running magnitude (2^-23; two instructions of 16 products per group), and every group and every partial
    sum of the eight warps adds half a step; then the output's own rounding."""
    sums = (2 * 2 * 17 + cols / 32 + 16) * 2.0 ** -24 * mag
    err = np.abs(y - want)
    assert (err <= sums + (2.0 ** -8 if out == "bf16" else 2.0 ** -24) * (np.abs(want) + sums) + 2.0 ** -133).all(), (err / (mag + 1e-300)).max()


@pytest.mark.parametrize("matrices,rows,cols", [(1, 1, 32), (1, 16, 128), (2, 17, 160), (3, 5, 352), (1, 100, 96)])
def test_pack_is_the_stated_layout(matrices, rows, cols):
    w = synth.student_t((matrices * rows, cols), 3)
    packed, codes, scales = packed_weights(w, matrices)
    want = np.concatenate([orc.e2m1_packed(codes[m], scales[m]) for m in range(matrices)])
    assert np.array_equal(packed.cpu().numpy(), want)


@pytest.mark.parametrize("tokens", [1, 2, 7, 8, 9, 16, 17, 33, 64])
@pytest.mark.parametrize("rows,cols", [(1, 32), (16, 128), (17, 96), (100, 1408), (257, 2080), (64, 4128)])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_one_matrix(tokens, rows, cols, out):
    packed, codes, scales = random_weights(1, rows, cols, rows + cols)
    x, y = run(synth.student_t((tokens, cols), tokens), packed, 1, None, rows, out)
    want, mag = orc.matvec_f64(x, codes, scales)
    check(y, want, mag, cols, out)


@pytest.mark.parametrize("tokens,choices,matrices", [(1, 1, 2), (1, 6, 8), (8, 6, 64), (3, 2, 100), (40, 2, 3), (33, 6, 5), (1024, 1, 2), (200, 5, 4)])
@pytest.mark.parametrize("kind", ["random", "same", "holes"])
def test_chosen_matrices(tokens, choices, matrices, kind):
    rows, cols = 45, 288
    rng = np.random.default_rng(tokens)
    ids = rng.integers(0, matrices, (tokens, choices)).astype(np.int32)
    if kind == "same":
        ids[:] = matrices - 1
    if kind == "holes":
        ids[rng.random(ids.shape) < 0.4] = -1
        ids[rng.random(ids.shape) < 0.1] = matrices
    packed, codes, scales = random_weights(matrices, rows, cols, 7)
    x, y = run(synth.gaussian((tokens, cols), 2), packed, matrices, ids, rows, "fp32")
    want, mag = orc.matvec_f64(x, codes, scales, ids)
    check(y, want, mag, cols, "fp32")
    assert not y[(ids.reshape(-1) < 0) | (ids.reshape(-1) >= matrices)].any()


@pytest.mark.parametrize("tokens", [1, 8, 13, 33, 70])
@pytest.mark.parametrize("rows,cols", [(19007, 288), (18944, 1152)])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_one_matrix_of_many_rows(tokens, rows, cols, out):
    """Enough row tiles that two share a warp's activations; the last group of them ragged."""
    packed, codes, scales = random_weights(1, rows, cols, rows)
    x, y = run(synth.student_t((tokens, cols), tokens), packed, 1, None, rows, out)
    want, mag = orc.matvec_f64(x, codes, scales)
    check(y, want, mag, cols, out)


@pytest.mark.parametrize("tokens,choices,matrices,rows,cols", [(8, 6, 64, 413, 288), (100, 4, 48, 413, 96), (8, 6, 12, 2816, 1184)])
def test_chosen_matrices_of_many_rows(tokens, choices, matrices, rows, cols):
    rng = np.random.default_rng(tokens)
    ids = rng.integers(-1, matrices, (tokens, choices)).astype(np.int32)
    packed, codes, scales = random_weights(matrices, rows, cols, 9)
    x, y = run(synth.gaussian((tokens, cols), 2), packed, matrices, ids, rows, "fp32")
    want, mag = orc.matvec_f64(x, codes, scales, ids)
    check(y, want, mag, cols, "fp32")


def test_scales_outside_the_fast_range_in_some_tiles():
    """Tiles whose scales all lie in 2^-63 .. 1 and tiles with one byte outside take different ways to the same sums."""
    import torch
    from paper_2506_08027_b200 import binding as B
    rows, cols = 19008, 512
    rng = np.random.default_rng(4)
    codes = rng.integers(0, 16, (1, rows, cols)).astype(np.uint8)
    scales = rng.integers(64, 128, (1, rows, cols // 32)).astype(np.uint8)
    odd = rng.random(scales.shape) < 0.002
    scales[odd] = rng.choice([0, 1, 63, 128, 129, 200, 254], odd.sum()).astype(np.uint8)
    flat = codes.reshape(-1, cols // 16, 16)
    slots = np.zeros_like(flat)
    slots[:, :, :8] = flat[:, :, 0::2] | flat[:, :, 1::2] << 4
    packed = torch.empty(B.mxfp8_e2m1_packed_bytes(1, rows, cols), dtype=torch.uint8, device="cuda")
    B.mxfp8_e2m1_pack(dev(slots.reshape(-1, cols)), dev(scales.reshape(-1)), 1, packed)
    x, y = run(synth.gaussian((5, cols), 3), packed, 1, None, rows, "fp32")
    want, mag = orc.matvec_f64(x, codes, scales)
    small = mag < 2.0 ** 127                        # nothing near the top of FP32's range
    assert small.any()
    err = np.abs(y - want)
    assert (err[small] <= ((2 * 2 * 17 + cols / 32 + 16) * 2.0 ** -24 * mag[small] + 2.0 ** -24 * np.abs(want[small])) * (1 + 2.0 ** -20) + 2.0 ** -133).all()


def test_a_large_matrix_and_long_rows():
    """14336 columns and, apart, a packed tensor of more than 2^31 bytes (the last matrix lies behind that offset)."""
    import torch
    from paper_2506_08027_b200 import binding as B
    packed, codes, scales = random_weights(1, 48, 14336, 5)
    x, y = run(synth.gaussian((3, 14336), 1), packed, 1, None, 48, "fp32")
    want, mag = orc.matvec_f64(x, codes, scales)
    check(y, want, mag, 14336, "fp32")
    matrices, rows, cols = 260, 4096, 4096
    one = B.mxfp8_e2m1_packed_bytes(1, rows, cols)
    big = torch.zeros(matrices, one, dtype=torch.uint8, device="cuda")
    assert big.numel() > 2 ** 31
    small, codes, scales = random_weights(1, 16, cols, 6)
    big[-1, :small.numel()] = small
    x, y = run(synth.gaussian((1, cols), 1), big, matrices, np.array([[matrices - 1]], np.int32), rows, "fp32")
    want, mag = orc.matvec_f64(x, codes, scales)
    check(y[:, :16], want, mag, cols, "fp32")
    assert not y[:, 16:].any()


def test_small_integers_are_exact():
    """Whole numbers, unit scales: every partial sum is one FP32 holds."""
    rng = np.random.default_rng(1)
    import torch
    from paper_2506_08027_b200 import binding as B
    packed, codes, scales = random_weights(2, 33, 640, 3, 127, 128)
    x = rng.integers(-8, 9, (9, 640)).astype(np.float32)
    ids = rng.integers(0, 2, (9, 3)).astype(np.int32)
    x, y = run(x, packed, 2, ids, 33, "fp32")
    assert np.array_equal(y, orc.matvec_f64(x, codes, scales, ids)[0])


def test_every_code_and_every_scale_byte():
    """One row per scale byte, one column per code, single products: exact, 2^-127 .. 2^127 and NaN, overflow to Inf as
    FP32 rounds it."""
    import torch
    from paper_2506_08027_b200 import binding as B
    rows, cols = 256, 32
    codes = np.tile(np.arange(32, dtype=np.uint8) % 16, (1, rows, 1))
    scales = np.arange(256, dtype=np.uint8).reshape(1, rows, 1)
    flat = codes.reshape(-1, 2, 16)
    slots = np.zeros_like(flat)
    slots[:, :, :8] = flat[:, :, 0::2] | flat[:, :, 1::2] << 4
    packed = torch.empty(B.mxfp8_e2m1_packed_bytes(1, rows, cols), dtype=torch.uint8, device="cuda")
    B.mxfp8_e2m1_pack(dev(slots.reshape(rows, cols)), dev(scales.reshape(-1)), 1, packed)
    for magnitude in (1.0, 2.0 ** -60, 1.5 * 2.0 ** 60):
        for half in (0, 16):
            x = np.zeros((16, cols), np.float32)
            x[np.arange(16), np.arange(16) + half] = magnitude
            _, y = run(x, packed, 1, None, rows, "fp32")
            table = np.array([orc.fp8_decode(c, orc.E2M1) for c in range(16)])
            with np.errstate(over="ignore", invalid="ignore"):
                want = (table[:, None] * np.exp2(np.arange(255) - 127.0) * magnitude).astype(np.float32)
            assert np.array_equal(y[:, :255].astype(np.float32), want)
            assert np.isnan(y[:, 255]).all()


@pytest.mark.parametrize("other", [127, 0, 200])
def test_large_activations_under_small_scales_do_not_overflow(other):
    """Sums that pass FP32's range before their scale and not after it; one row's byte decides which way the tile takes."""
    import torch
    from paper_2506_08027_b200 import binding as B
    rows, cols = 16, 64
    bytes_of_rows = np.array([0, 1, 10, 40, 62, 63, 64, 65, 80, 90, 100, 110, 115, 115, 64, other], np.uint8)
    codes = np.full((1, rows, cols), 7, np.uint8)               # 6.0
    codes[:, :, 1::3] = 15                                      # -6.0
    if other == 127:
        bytes_of_rows = np.maximum(bytes_of_rows, 64)           # all inside 64 .. 127
    scales = np.repeat(bytes_of_rows.reshape(1, rows, 1), cols // 32, axis=2)
    flat = codes.reshape(-1, cols // 16, 16)
    slots = np.zeros_like(flat)
    slots[:, :, :8] = flat[:, :, 0::2] | flat[:, :, 1::2] << 4
    packed = torch.empty(B.mxfp8_e2m1_packed_bytes(1, rows, cols), dtype=torch.uint8, device="cuda")
    B.mxfp8_e2m1_pack(dev(slots.reshape(-1, cols)), dev(scales.reshape(-1)), 1, packed)
    x, y = run(np.full((3, cols), 1.5 * 2.0 ** 126), packed, 1, None, rows, "fp32")
    want, mag = orc.matvec_f64(x, codes, scales)
    check(y[:, :15], want[:, :15], mag[:, :15], cols, "fp32")


def test_special_values_reach_their_token_only():
    packed, codes, scales = random_weights(1, 32, 256, 8)
    codes_used = codes[0]
    x = synth.gaussian((12, 256), 5)
    x[3, 17], x[5, 200], x[7, 31] = np.nan, np.inf, -np.inf
    xv, y = run(x, packed, 1, None, 32, "fp32")
    with np.errstate(invalid="ignore"):
        want, mag = orc.matvec_f64(xv, codes, scales)
    clean = [t for t in range(12) if t not in (3, 5, 7)]
    check(y[clean], want[clean], mag[clean], 256, "fp32")
    assert np.isnan(y[3]).all()
    for t, k in ((5, 200), (7, 31)):
        zero = (codes_used[:, k] & 7) == 0                   # zero times infinity is NaN
        assert np.isnan(y[t][zero]).all() and np.isinf(y[t][~zero]).all()
        assert np.array_equal(np.sign(y[t][~zero]), np.sign(want[t][~zero]))


def test_captured_and_on_another_stream():
    import torch
    from paper_2506_08027_b200 import binding as B
    packed, codes, scales = random_weights(4, 64, 512, 2)
    x = torch.randn(5, 512, device="cuda").to(torch.bfloat16)
    ids = torch.randint(0, 4, (5, 2), dtype=torch.int32, device="cuda")
    want = torch.empty(10, 64, device="cuda")
    B.mxfp8_e2m1_matvec(x, packed, 4, ids, want)
    got, other = torch.zeros(10, 64, device="cuda"), torch.zeros(10, 64, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.mxfp8_e2m1_matvec(x, packed, 4, ids, got)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    B.mxfp8_e2m1_matvec(x, packed, 4, ids, other, stream=s)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(other, want)


def test_few_tokens_through_their_experts():
    """One decoding step of a mixture-of-experts layer: up product, squared relu, down product, weighted sum."""
    import torch
    from paper_2506_08027_b200 import binding as B
    tokens, top_k, experts, hidden, ffn = 6, 3, 8, 256, 352
    up, cu, su = packed_weights(0.1 * synth.gaussian((experts * ffn, hidden), 1), experts)
    down, cd, sd = packed_weights(0.1 * synth.gaussian((experts * hidden, ffn), 2), experts)
    rng = np.random.default_rng(3)
    ids = np.stack([rng.permutation(experts)[:top_k] for _ in range(tokens)]).astype(np.int32)
    w = rng.random((tokens, top_k)).astype(np.float32)
    xv, h = run(synth.gaussian((tokens, hidden), 4), up, experts, ids, ffn, "bf16")
    act = np.square(np.maximum(h, 0)).astype(np.float32)
    one_each = ids.reshape(-1, 1)
    av, y = run(act, down, experts, one_each, hidden, "fp32")
    out = torch.empty(tokens, hidden, device="cuda")
    rows_in_slot_order = torch.arange(tokens * top_k, dtype=torch.int32, device="cuda").view(tokens, top_k)
    B.mxfp8_moe_combine(torch.from_numpy(y).float().cuda(), rows_in_slot_order, dev(w), out)
    want, mag = orc.matvec_f64(av, cd, sd, one_each)
    check(y, want, mag, ffn, "fp32")
    want = (want.reshape(tokens, top_k, hidden) * w[:, :, None].astype(np.float64)).sum(axis=1)
    bound = (mag.reshape(tokens, top_k, hidden) * w[:, :, None]).sum(axis=1)
    assert (np.abs(out.double().cpu().numpy() - want) <= (100 + ffn / 32) * 2.0 ** -24 * bound).all()
