"""The few-token layer of experts where a CTA has more units than warps, where experts take several entries, and where the choice goes the other way.

With 148 multiprocessors of 16 warps a warp of the first launch takes whole units (16 gate and 16 up rows for one entry) from 2368 units on; fewer are
split by column tiles.  Checks and tolerances are those of test_moe_tokens_gpu.py."""
import pytest
import torch

from paper_2506_08027_b200 import binding as B
from test_moe_tokens_gpu import choice, layer, matrices, run

pytestmark = pytest.mark.gpu


def check(tokens, top_k, experts, cols, inner, kind, renormalize, out, logits=None):
    g = torch.Generator(device="cuda").manual_seed(tokens * 1000 + cols)
    gate_up, gv = matrices(experts, 2 * inner, cols, g)
    down, dv = matrices(experts, cols, inner, g)
    x = torch.randn(tokens, cols, generator=g, device="cuda").to(torch.bfloat16)
    if logits is None:
        logits = torch.randn(tokens, experts, generator=g, device="cuda")
        logits[1] = float("-inf")
    y, ids, weights = run(x, logits, top_k, (gate_up, down), inner, kind, renormalize, out)
    want_ids, want_weights = choice(logits, top_k, renormalize)
    assert torch.equal(ids.cpu(), want_ids)
    assert bool(((weights.cpu().double() - want_weights).abs() <= 300 * 2.0 ** -23 * want_weights + 1e-38).all())
    want, slack = layer(x, want_ids, want_weights, gv, dv, inner, kind)
    slack = slack + 300 * 2.0 ** -23 * want.abs()
    step = torch.finfo(out).eps / 2
    assert bool(((y.double() - want).abs() <= step * (want.abs() + slack) + slack + 1e-30).all())
    again, _, _ = run(x, logits, top_k, (gate_up, down), inner, kind, renormalize, out, extra=False)
    assert torch.equal(again, y)


@pytest.mark.parametrize("tokens,top_k,experts,cols,inner,kind,renormalize,out", [
    # entries of eight slots in the first launch, of four in the second; about 4000 units of nine column tiles: one whole unit per warp, and a rest
    (16, 6, 64, 1056, 1408, B.ACT_SILU, True, torch.float32),
    # entries of 16 and of eight; 322 units per entry, at least eight entries
    (32, 2, 8, 1056, 5152, B.ACT_SILU, False, torch.float32),
    # one expert with 64 slots: four entries of 16, eight of eight, 12 warps in the second launch
    (64, 1, 1, 544, 10016, B.ACT_GELU_TANH, True, torch.bfloat16),
    # more groups of 32 output rows than clusters of two CTAs (74), several entries of some experts, 12 warps
    (40, 3, 5, 2432, 640, B.ACT_RELU, True, torch.float32),
    # the same with 16 warps, and with few slots per expert
    (24, 2, 3, 2656, 224, B.ACT_SILU, True, torch.float32),
    (48, 2, 64, 2432, 96, B.ACT_SILU, False, torch.float32),
    # all of the limits but the sizes: 64 tokens, 256 experts, 16 of them for each
    (64, 16, 256, 64, 32, B.ACT_SILU, True, torch.float32),
])
def test_layer(tokens, top_k, experts, cols, inner, kind, renormalize, out):
    check(tokens, top_k, experts, cols, inner, kind, renormalize, out)


def test_every_token_chooses_the_same_experts():
    logits = torch.zeros(33, 12, device="cuda")
    logits[:, [2, 11, 5]] = torch.tensor([3.0, 2.0, 1.0], device="cuda")
    check(33, 3, 12, 320, 544, B.ACT_SILU, True, torch.float32, logits)


@pytest.mark.parametrize("experts", [64, 200, 256])
@pytest.mark.parametrize("top_k", [1, 5, 16])
@pytest.mark.parametrize("renormalize", [True, False])
def test_choice_of_many_tokens_at_ties_zeros_infinities_and_nan(experts, top_k, renormalize):
    """More than 2^14 comparisons: a warp per token takes the largest one after the other.  Ties between lanes and within one (e and e + 32)."""
    cols, inner, tokens = 32, 32, 20
    g = torch.Generator(device="cuda").manual_seed(experts)
    packed = matrices(experts, 2 * inner, cols, g)[0], matrices(experts, cols, inner, g)[0]
    inf, nan, low = float("inf"), float("nan"), torch.finfo(torch.float32).min
    logits = torch.randn(tokens, experts, generator=g, device="cuda")
    logits[0] = 0.0                                                            # all equal, both zeros
    logits[0, ::2] = -0.0
    logits[1] = -inf
    logits[1, [33, 1, 34, 63]] = 1.0                                           # lane 1 twice, lanes 2 and 31
    logits[2] = nan
    logits[2, [5, 37]] = torch.tensor([-5.0, -5.0], device="cuda")
    logits[3] = -inf
    logits[4, [7, 39, 40]] = inf
    logits[5] = low                                                            # the type's lowest value is a logit like others
    logits[5, 20] = -inf
    logits[6] = torch.arange(experts, device="cuda").float() * 1e-3
    logits[7] = -torch.arange(experts, device="cuda").float()
    logits[8] = nan
    logits[9, ::3] = nan
    logits[10, 1::2] = -inf
    logits[11] = (torch.arange(experts, device="cuda") % 32 == 3).float()      # every element of one lane
    logits[12, [1, 2]] = torch.tensor([200.0, -200.0], device="cuda")
    logits[13] = -1e-42                                                        # equal subnormal numbers
    logits[13, 50] = 1e-42
    x = torch.randn(tokens, cols, generator=g, device="cuda").to(torch.bfloat16)
    y, ids, weights = run(x, logits, top_k, packed, inner, B.ACT_SILU, renormalize, torch.float32)
    want_ids, want = choice(logits, top_k, renormalize)
    assert torch.equal(ids.cpu(), want_ids)
    assert bool(((weights.cpu().double() - want).abs() <= 300 * 2.0 ** -23 * want + 1e-38).all())
    assert bool((y[3] == 0).all()) and bool((y[8] == 0).all()) and bool(y.isfinite().all())


@pytest.mark.parametrize("sign", [1, -1])
def test_an_intermediate_between_the_largest_numbers_of_bf16_and_fp32(sign):
    """m = (2^64 (1 - 2^-12))^2 = 2^128 (1 - 2^-11 + 2^-24) is an FP32 number that BF16 rounds to infinity.  Times 2^-30 it is in range; the other columns of the down
    matrix are zero.  m is kept to 2^-16 of itself, everything else here is exact."""
    cols, inner = 64, 64
    packed = []
    down = torch.zeros(cols, inner, device="cuda")
    down[:, 0] = sign * 2.0 ** -30
    for w in (torch.ones(2 * inner, cols, device="cuda"), down):
        q = torch.empty(w.shape, dtype=torch.uint8, device="cuda")
        s = torch.empty(w.numel() // 32, dtype=torch.uint8, device="cuda")
        B.mxfp8_quantize(w, B.ROW, B.RULE_PAPER, B.E2M1, q, s, None, None, B.SF_LINEAR)
        packed.append(torch.empty(B.mxfp8_e2m1_packed_bytes(1, *w.shape), dtype=torch.uint8, device="cuda"))
        B.mxfp8_e2m1_pack(q, s, 1, packed[-1])
    x = torch.zeros(1, cols, dtype=torch.bfloat16, device="cuda")
    x[0, 0], x[0, 1], x[0, 2] = 2.0 ** 63, 2.0 ** 63 * (1 - 2.0 ** -8), 2.0 ** 55 * 0.875
    assert float(x.double().sum()) == 2.0 ** 64 * (1 - 2.0 ** -12)
    y, _, _ = run(x, torch.zeros(1, 1, device="cuda"), 1, packed, inner, B.ACT_NONE, True, torch.float32)
    want = sign * 2.0 ** 98 * (1 - 2.0 ** -11 + 2.0 ** -24)
    assert bool(((y.double() - want).abs() <= 2.0 ** -16 * abs(want)).all())


@pytest.mark.parametrize("tokens,top_k,experts", [(1, 1, 1), (3, 2, 2), (4, 4, 4), (7, 1, 1), (16, 2, 8), (23, 3, 4), (33, 2, 40), (64, 1, 1), (64, 4, 5)])
def test_an_intermediate_is_held_in_32_bits_where_the_outputs_are(tokens, top_k, experts):
    """m = s^2 of a 12-bit s needs all 24 bits of an FP32 number.  With one column of the down matrices 1 and the others zero, and choices of equal weight (a half or a quarter
    of m each, exactly; with three, a third is rounded twice), y is m to the last bit."""
    cols, inner = 64, 96
    packed = []
    down = torch.zeros(experts, cols, inner, device="cuda")
    down[:, :, 5] = 1.0
    for w in (torch.ones(experts, 2 * inner, cols, device="cuda"), down):
        q = torch.empty(experts * w.shape[1], w.shape[2], dtype=torch.uint8, device="cuda")
        s = torch.empty(w.numel() // 32, dtype=torch.uint8, device="cuda")
        B.mxfp8_quantize(w.reshape(q.shape), B.ROW, B.RULE_PAPER, B.E2M1, q, s, None, None, B.SF_LINEAR)
        packed.append(torch.empty(B.mxfp8_e2m1_packed_bytes(*w.shape), dtype=torch.uint8, device="cuda"))
        B.mxfp8_e2m1_pack(q, s, experts, packed[-1])
    g = torch.Generator(device="cuda").manual_seed(tokens)
    a, b = (torch.randint(0, n, (tokens,), generator=g, device="cuda") for n in (128, 16))
    x = torch.zeros(tokens, cols, dtype=torch.bfloat16, device="cuda")
    x[:, 0], x[:, 33] = (1 + a / 128.0).to(torch.bfloat16), (b * 2.0 ** -11).to(torch.bfloat16)
    m = x.double().sum(dim=1).square()
    logits = torch.zeros(tokens, experts, device="cuda")
    y, _, _ = run(x, logits, top_k, packed, inner, B.ACT_NONE, True, torch.float32)
    off = (y.double() - m.unsqueeze(1)).abs() / m.unsqueeze(1)
    # three times a rounded third, three roundings of the sum
    assert float(off.max()) <= (5 * 2.0 ** -24 if top_k == 3 else 0.0)
    # two parts, to 2^-16, and the outputs' rounding
    y, _, _ = run(x, logits, top_k, packed, inner, B.ACT_NONE, True, torch.bfloat16)
    assert float(((y.double() - m.unsqueeze(1)).abs() / m.unsqueeze(1)).max()) <= 2.0 ** -8 + 2.0 ** -15
