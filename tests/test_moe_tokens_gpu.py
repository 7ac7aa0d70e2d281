"""A mixture-of-experts layer for a few tokens with E2M1 matrices, against the definition in 64 bits.

An FP32 sum of c products that the kernels form (tensor-core sums of 128 columns, then FP32) is off by at most (c / 8 + 64) * 2^-23 of the sum of its
terms' absolute values (the tensor cores truncate: a whole step per addition of a group).  The activation has a few 2^-22, m is kept to 2^-16."""
import pytest
import torch

from paper_2506_08027_b200 import binding as B

pytestmark = pytest.mark.gpu


def matrices(count, rows, cols, g, scale=0.03):
    """Random matrices through the library's conversion: packed bytes and their values in 64 bits."""
    w = scale * torch.randn(count * rows, cols, generator=g, device="cuda")
    q = torch.empty(count * rows, cols, dtype=torch.uint8, device="cuda")
    s = torch.empty(count * rows * (cols // 32), dtype=torch.uint8, device="cuda")
    B.mxfp8_quantize(w, B.ROW, B.RULE_PAPER, B.E2M1, q, s, None, None, B.SF_LINEAR)
    values = torch.empty(count * rows, cols, device="cuda")
    B.mxfp8_dequantize(q, s, B.ROW, B.E2M1, B.SF_LINEAR, values)
    packed = torch.empty(B.mxfp8_e2m1_packed_bytes(count, rows, cols), dtype=torch.uint8, device="cuda")
    B.mxfp8_e2m1_pack(q, s, count, packed)
    return packed, values.double().reshape(count, rows, cols)


def act(v, kind):
    if kind == B.ACT_RELU:
        return v.clamp(min=0)
    if kind == B.ACT_RELU2:
        return v.clamp(min=0).square()
    if kind == B.ACT_SILU:
        return v * torch.sigmoid(v)
    if kind == B.ACT_GELU_TANH:
        return torch.nn.functional.gelu(v, approximate="tanh")
    return v


def choice(logits, top_k, renormalize):
    """The definition, token by token."""
    ids = torch.full((logits.shape[0], top_k), -1, dtype=torch.int32)
    weights = torch.zeros(logits.shape[0], top_k, dtype=torch.float64)
    for t, row in enumerate(logits.double().cpu().tolist()):
        live = [e for e, l in enumerate(row) if l > float("-inf")]
        order = sorted(live, key=lambda e: (-row[e], e))[:top_k]
        if not order:
            continue
        top = row[order[0]]
        share = lambda e: torch.exp(torch.tensor(0.0 if row[e] == top else row[e] - top, dtype=torch.float64)).item()
        total = sum(share(e) for e in (order if renormalize else live))
        for j, e in enumerate(order):
            ids[t, j], weights[t, j] = e, share(e) / total
    return ids, weights


def layer(x, ids, weights, gate_up, down, inner, kind):
    """y, and how far an FP32 evaluation may be from it."""
    tokens, cols = x.shape
    y = torch.zeros(tokens, cols, dtype=torch.float64, device="cuda")
    slack = torch.zeros_like(y)
    A, M = (cols / 8 + 64) * 2.0 ** -23, (inner / 8 + 64) * 2.0 ** -23
    for t in range(tokens):
        for j, e in enumerate(ids[t].tolist()):
            if e < 0:
                continue
            a, size = gate_up[e] @ x[t].double(), gate_up[e].abs() @ x[t].double().abs()
            g, u, gs, us = act(a[:inner], kind), a[inner:], A * size[:inner], A * size[inner:]
            slope = 2 * (1 + a[:inner].abs()) if kind == B.ACT_RELU2 else 1.2       # of the activations
            m = g * u
            ms = slope * gs * (u.abs() + us) + g.abs() * us + 2.0 ** -16 * m.abs() + 2.0 ** -20 * (g * u).abs() + (2.0 ** -20 * g.abs() * u.abs())
            w = float(weights[t, j])
            y[t] += w * (down[e] @ m)
            slack[t] += w * (down[e].abs() @ (ms + (M + 2.0 ** -20) * m.abs()))
    return y, slack


def run(x, logits, top_k, packed, inner, kind, renormalize, out, extra=True):
    tokens, cols = x.shape
    y = torch.full((tokens + 2, cols), 7.0, dtype=out, device="cuda")
    ids = torch.full((tokens, top_k), -9, dtype=torch.int32, device="cuda") if extra else None
    weights = torch.full((tokens, top_k), -9.0, device="cuda") if extra else None
    n = B.mxfp8_e2m1_moe_ws_bytes(tokens, top_k, inner)
    ws = torch.full((n + 16,), 0xFF, dtype=torch.uint8, device="cuda")          # NaN wherever nothing is written
    B.mxfp8_e2m1_moe(x, logits, top_k, packed[0], packed[1], inner, kind, renormalize, y[1:-1], ids, weights, ws[:n])
    torch.cuda.synchronize()
    assert bool((y[0] == 7).all()) and bool((y[-1] == 7).all()) and bool((ws[n:] == 0xFF).all())
    return y[1:-1], ids, weights


CASES = [
    # tokens, top_k, experts, cols, inner, activation, renormalize, output
    (1, 1, 1, 32, 32, B.ACT_SILU, True, torch.float32),
    (1, 2, 4, 128, 64, B.ACT_SILU, True, torch.bfloat16),
    (1, 8, 64, 512, 256, B.ACT_SILU, True, torch.float32),
    (3, 4, 8, 160, 96, B.ACT_GELU_TANH, False, torch.float32),
    (7, 2, 3, 1056, 352, B.ACT_NONE, True, torch.float32),
    (8, 3, 60, 256, 416, B.ACT_RELU, False, torch.bfloat16),
    (9, 1, 2, 288, 128, B.ACT_SILU, True, torch.float32),
    (17, 16, 16, 96, 160, B.ACT_SILU, True, torch.float32),
    (33, 2, 5, 640, 1408, B.ACT_RELU2, True, torch.float32),
    (64, 8, 256, 64, 32, B.ACT_SILU, False, torch.float32),
    (64, 1, 1, 256, 2080, B.ACT_SILU, True, torch.bfloat16),
    (2, 2, 2, 4128, 64, B.ACT_SILU, True, torch.float32),
]


@pytest.mark.parametrize("tokens,top_k,experts,cols,inner,kind,renormalize,out", CASES)
def test_layer(tokens, top_k, experts, cols, inner, kind, renormalize, out):
    g = torch.Generator(device="cuda").manual_seed(tokens * 1000 + cols)
    gate_up, gv = matrices(experts, 2 * inner, cols, g)
    down, dv = matrices(experts, cols, inner, g)
    x = torch.randn(tokens, cols, generator=g, device="cuda").to(torch.bfloat16)
    logits = torch.randn(tokens, experts, generator=g, device="cuda")
    if tokens > 2:
        logits[1] = float("-inf")                       # an empty place of the batch
        logits[2, : experts - 1] = float("-inf")        # one expert is left
    y, ids, weights = run(x, logits, top_k, (gate_up, down), inner, kind, renormalize, out)
    want_ids, want_weights = choice(logits, top_k, renormalize)
    assert torch.equal(ids.cpu(), want_ids)
    # expf and up to 256 additions
    assert bool(((weights.cpu().double() - want_weights).abs() <= 300 * 2.0 ** -23 * want_weights + 1e-38).all())
    want, slack = layer(x, want_ids, want_weights, gv, dv, inner, kind)
    slack = slack + 300 * 2.0 ** -23 * want.abs()
    step = torch.finfo(out).eps / 2
    assert bool(((y.double() - want).abs() <= step * (want.abs() + slack) + slack + 1e-30).all())
    if tokens > 2:
        assert bool((y[1] == 0).all())
    again, _, _ = run(x, logits, top_k, (gate_up, down), inner, kind, renormalize, out, extra=False)
    assert torch.equal(again, y)


def test_choice_at_ties_zeros_infinities_and_nan():
    experts, cols, inner = 40, 32, 32
    g = torch.Generator(device="cuda").manual_seed(1)
    packed = matrices(experts, 2 * inner, cols, g)[0], matrices(experts, cols, inner, g)[0]
    inf, nan, low = float("inf"), float("nan"), torch.finfo(torch.float32).min
    logits = torch.zeros(8, experts, device="cuda")
    logits[0, ::2] = -0.0                                                    # both zeros are equal
    logits[1] = -inf
    logits[1, [3, 38, 39]] = torch.tensor([1.0, 1.0, 1.0], device="cuda")
    logits[2] = nan
    logits[2, 33] = -5.0
    logits[3] = -inf
    logits[4, [7, 35]] = inf
    logits[5] = low                                                          # the type's lowest value is a logit like others
    logits[5, 20] = -inf
    logits[6] = torch.arange(experts, device="cuda").float() * 1e-3
    logits[7, [1, 2]] = torch.tensor([200.0, -200.0], device="cuda")
    x = torch.randn(8, cols, generator=g, device="cuda").to(torch.bfloat16)
    for renormalize in (True, False):
        for top_k in (1, 4):
            y, ids, weights = run(x, logits, top_k, packed, inner, B.ACT_SILU, renormalize, torch.float32)
            want_ids, want = choice(logits, top_k, renormalize)
            assert torch.equal(ids.cpu(), want_ids)
            assert bool(((weights.cpu().double() - want).abs() <= 300 * 2.0 ** -23 * want + 1e-38).all())
            assert bool((y[3] == 0).all()) and bool(y.isfinite().all())


def test_special_scales_and_codes_pass_through():
    """A scale byte 0xFF makes the outputs of its expert's tokens NaN and of no others."""
    experts, cols, inner, tokens = 4, 64, 64, 4
    g = torch.Generator(device="cuda").manual_seed(2)
    gate_up, down = matrices(experts, 2 * inner, cols, g)[0], matrices(experts, cols, inner, g)[0]
    down.reshape(experts, -1)[2, 1024] = 255                                 # row 0, columns 0 .. 31
    logits = torch.full((tokens, experts), -9.0, device="cuda")
    for t in range(tokens):
        logits[t, t] = 3.0
    x = torch.randn(tokens, cols, generator=g, device="cuda").to(torch.bfloat16)
    y, _, _ = run(x, logits, 1, (gate_up, down), inner, B.ACT_SILU, True, torch.float32)
    assert bool(y[2, 0].isnan()) and int(y.isnan().sum()) == 1


def test_wide_scales():
    """Scale bytes over the whole range, in both products."""
    experts, cols, inner, tokens = 3, 256, 128, 5
    g = torch.Generator(device="cuda").manual_seed(3)
    gate_up, gv = matrices(experts, 2 * inner, cols, g, scale=2.0 ** -64)
    down, dv = matrices(experts, cols, inner, g, scale=2.0 ** 90)
    x = torch.randn(tokens, cols, generator=g, device="cuda").to(torch.bfloat16)
    logits = torch.randn(tokens, experts, generator=g, device="cuda")
    y, ids, weights = run(x, logits, 2, (gate_up, down), inner, B.ACT_NONE, True, torch.float32)
    want, slack = layer(x, ids.cpu(), weights.cpu().double(), gv, dv, inner, B.ACT_NONE)
    # m lies near 2^-120, and the second part of it on BF16's grid of subnormal numbers, 2^-133 apart
    floor = 2.0 ** -134 * inner * float(dv.abs().max())
    assert bool(((y.double() - want).abs() <= slack + 2.0 ** -20 * want.abs() + floor).all())


@pytest.mark.parametrize("sign", [1, -1])
def test_an_infinite_intermediate_stays_infinite(sign):
    """The first token's m overflows FP32 (2^100 * 2^100); with weights that are all 1 the formula gives an infinity of its sign, and the second
    token, whose m is 64 * 64, must not notice.  All of the second token's numbers are powers of two, so its outputs are exact."""
    cols, inner = 64, 96
    packed = []
    for rows, c in ((2 * inner, cols), (cols, inner)):
        q = torch.empty(rows, c, dtype=torch.uint8, device="cuda")
        s = torch.empty(rows * (c // 32), dtype=torch.uint8, device="cuda")
        B.mxfp8_quantize(torch.ones(rows, c, device="cuda"), B.ROW, B.RULE_PAPER, B.E2M1, q, s, None, None, B.SF_LINEAR)
        packed.append(torch.empty(B.mxfp8_e2m1_packed_bytes(1, rows, c), dtype=torch.uint8, device="cuda"))
        B.mxfp8_e2m1_pack(q, s, 1, packed[-1])
    x = torch.zeros(2, cols, dtype=torch.bfloat16, device="cuda")
    x[0, 0] = sign * 2.0 ** 100
    x[1] = 1.0
    logits = torch.zeros(2, 1, device="cuda")
    kind = B.ACT_RELU if sign > 0 else B.ACT_NONE
    y, _, _ = run(x, logits, 1, packed, inner, kind, True, torch.float32)
    assert bool((y[0] == float("inf")).all())                            # (-2^100)^2 as well
    assert bool((y[1] == inner * 64.0 * 64.0).all())


def test_graph_streams_and_two_calls_at_once():
    tokens, top_k, experts, cols, inner = 6, 3, 16, 512, 256
    g = torch.Generator(device="cuda").manual_seed(4)
    packed = matrices(experts, 2 * inner, cols, g)[0], matrices(experts, cols, inner, g)[0]
    x = torch.randn(tokens, cols, generator=g, device="cuda").to(torch.bfloat16)
    logits = torch.randn(tokens, experts, generator=g, device="cuda")
    n = B.mxfp8_e2m1_moe_ws_bytes(tokens, top_k, inner)
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    ys = [torch.zeros(tokens, cols, device="cuda") for _ in range(2)]

    def call(k):
        B.mxfp8_e2m1_moe(x, logits, top_k, packed[0], packed[1], inner, B.ACT_SILU, True, ys[k], None, None, ws[k])
    call(0)
    torch.cuda.synchronize()
    first = ys[0].clone()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for k, s in enumerate(streams):
        with torch.cuda.stream(s):
            for _ in range(4):
                call(k)
    torch.cuda.synchronize()
    assert torch.equal(ys[0], first) and torch.equal(ys[1], first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(0)
        call(0)
    x.mul_(-1.5)
    logits.copy_(torch.randn(tokens, experts, generator=g, device="cuda"))         # another choice
    graph.replay()
    torch.cuda.synchronize()
    call(1)
    torch.cuda.synchronize()
    assert torch.equal(ys[0], ys[1]) and not torch.equal(ys[0], first)
