"""The calls around a block's products together, as a training step and a served block use them, against the formulas in 64 bits."""
import os
import socket

import pytest
import torch

from paper_2506_08027_b200 import binding as B
from paper_2506_08027_b200.dp import DataParallelLinear, GradientClipping

pytestmark = pytest.mark.gpu


def rms(v, eps=1e-5):
    return v / torch.sqrt(v.square().mean(dim=1, keepdim=True) + eps)


def near(got, want, tolerance):
    return float((got.double() - want).norm() / want.norm()) <= tolerance


def test_training_step_of_a_block():
    """Seam forward with the next product's input converted, linear layer, seam backward, clipping of all gradients; captured and replayed."""
    T, H, F = 256, 512, 384
    g = torch.Generator(device="cuda").manual_seed(1)
    bf = torch.bfloat16

    def rand(*shape, scale=1.0):
        return (scale * torch.randn(*shape, generator=g, device="cuda")).to(bf)
    y, h_in, w, dout = rand(T, H), rand(T, H), rand(F, H, scale=0.05), rand(T, F, scale=0.01)
    gp, gq = (1 + 0.1 * rand(H).float()).to(bf), (1 + 0.1 * rand(H).float()).to(bf)
    dh = rand(T, H, scale=0.01)
    seam = B.make_seam(gp, gq, None, 1, 0.5, 1.0)
    h, x = torch.empty_like(h_in), torch.empty_like(y)
    rp, rn = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    q = B.alloc_quantize_outputs(T, H, B.BOTH, B.SF_SWIZZLED)
    out, dx, dw = torch.empty(T, F, dtype=bf, device="cuda"), torch.empty(T, H, dtype=bf, device="cuda"), torch.empty(F, H, dtype=bf, device="cuda")
    lws = torch.empty(B.mxfp8_linear_ws_bytes(T, H, F), dtype=torch.uint8, device="cuda")
    dy, dh_in, dgp, dgq = torch.empty_like(y), torch.empty_like(h), torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    gws = torch.empty(B.mxfp8_residual_rmsnorm_grad_ws_bytes(seam, T, H), dtype=torch.uint8, device="cuda")
    clipping = GradientClipping([dw, dgp, dgq])

    def step():
        B.mxfp8_residual_rmsnorm(seam, y, h_in, h, x, rp, rn)
        B.mxfp8_residual_rmsnorm_quantize(seam, y, h_in, h, rp, rn, B.BOTH, B.RULE_PAPER, B.E4M3, *q, B.SF_SWIZZLED)
        B.mxfp8_linear(x, w, dout, B.RULE_PAPER, out, dx, dw, lws)
        B.mxfp8_residual_rmsnorm_grad(seam, dx, dh, y, h, rp, rn, dy, dh_in, dgp, dgq, None, gws)
        return clipping.clip(0.25)
    step()
    torch.cuda.synchronize()
    assert B.mxfp8_device_status() == 0
    # the copies that the conversion wrote are those that the linear layer makes of x (BF16 stream: x is the same rounding)
    want = B.alloc_quantize_outputs(T, H, B.BOTH, B.SF_SWIZZLED)
    B.mxfp8_quantize(x, B.BOTH, B.RULE_PAPER, B.E4M3, *want, B.SF_SWIZZLED)
    assert all(torch.equal(a, b) for a, b in zip(q, want))
    y64, h64 = y.double(), h_in.double() + 0.5 * rms(y.double()) * gq.double()
    assert near(h, h64, 2.0 ** -8)                                       # one rounding to BF16
    x64 = rms(h.double()) * gp.double()
    assert near(x, x64, 2.0 ** -8)
    # the products see E4M3 values (half a step: 2^-4 of each operand, so 2^-3 for sums of them, far less for many terms)
    assert near(out, x64 @ w.double().t(), 2.0 ** -3)
    leaf = {k: v.detach().clone().requires_grad_() for k, v in dict(y=y64, h=h_in.double(), gp=gp.double(), gq=gq.double()).items()}
    s = leaf["h"] + 0.5 * rms(leaf["y"]) * leaf["gq"]
    ((rms(s) * leaf["gp"] * dx.double()).sum() + (s * dh.double()).sum()).backward()
    # h was rounded in between: 2^-9 of each element in xh, so a few 2^-8 in the gradients
    for got, name in ((dy, "y"), (dh_in, "h")):
        assert near(got, leaf[name].grad, 2.0 ** -6), name
    norm, factor = [float(v) for v in clipping.norm]
    for got, name in ((dgp, "gp"), (dgq, "gq")):
        assert near(got / factor, leaf[name].grad, 2.0 ** -6), name
    scaled = torch.cat([t.double().reshape(-1) for t in (dw, dgp, dgq)]).norm()
    assert factor < 1 and abs(float(scaled) - 0.25) <= 2.0 ** -8 * 0.25      # what is left is the largest norm, BF16 roundings apart
    # the whole step captured and replayed on other inputs
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    y.mul_(-1.5)
    dout.mul_(2.0)
    graph.replay()
    torch.cuda.synchronize()
    first = [t.clone() for t in (h, x, dy, dh_in, dgp, dgq, dw, clipping.norm)]
    step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, (h, x, dy, dh_in, dgp, dgq, dw, clipping.norm)))


def test_a_served_block_of_experts():
    """Norm, experts, seam, experts: a few tokens through two blocks, nothing waits for the host."""
    tokens, top_k, experts, cols, inner = 5, 2, 6, 256, 160
    g = torch.Generator(device="cuda").manual_seed(2)
    bf = torch.bfloat16
    packed, value = [], []
    for rows, width in ((2 * inner, cols), (cols, inner)):
        w = 0.05 * torch.randn(experts * rows, width, generator=g, device="cuda")
        q, s = torch.empty(experts * rows, width, dtype=torch.uint8, device="cuda"), torch.empty(experts * rows * (width // 32), dtype=torch.uint8, device="cuda")
        B.mxfp8_quantize(w, B.ROW, B.RULE_PAPER, B.E2M1, q, s, None, None, B.SF_LINEAR)
        v = torch.empty(experts * rows, width, device="cuda")
        B.mxfp8_dequantize(q, s, B.ROW, B.E2M1, B.SF_LINEAR, v)
        p = torch.empty(B.mxfp8_e2m1_packed_bytes(experts, rows, width), dtype=torch.uint8, device="cuda")
        B.mxfp8_e2m1_pack(q, s, experts, p)
        packed.append(p)
        value.append(v.double().reshape(experts, rows, width))
    router = torch.randn(experts, cols, generator=g, device="cuda")
    gp, gq = torch.ones(cols, dtype=bf, device="cuda"), torch.ones(cols, dtype=bf, device="cuda")
    seam = B.make_seam(gp, gq)
    h = torch.randn(tokens, cols, generator=g, device="cuda").to(bf)
    y = torch.zeros_like(h)
    x = torch.empty_like(h)
    rp, rn = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")
    ws = torch.empty(B.mxfp8_e2m1_moe_ws_bytes(tokens, top_k, inner), dtype=torch.uint8, device="cuda")
    h64 = h.double()
    B.mxfp8_residual_rmsnorm(seam, y, h, h, x, rp, rn)                     # no block before the first: y is zero
    for _ in range(2):
        logits = x.float() @ router.t()
        ids = torch.empty(tokens, top_k, dtype=torch.int32, device="cuda")
        weights = torch.empty(tokens, top_k, device="cuda")
        B.mxfp8_e2m1_moe(x, logits, top_k, packed[0], packed[1], inner, B.ACT_SILU, True, y, ids, weights, ws)
        B.mxfp8_residual_rmsnorm(seam, y, h, h, x, rp, rn)
        # the same block in 64 bits with the experts that were chosen
        x64, y64 = rms(h64), torch.zeros_like(h64)
        for t in range(tokens):
            for j in range(top_k):
                a = value[0][int(ids[t, j])] @ x64[t]
                y64[t] += float(weights[t, j]) * (value[1][int(ids[t, j])] @ (torch.nn.functional.silu(a[:inner]) * a[inner:]))
        h64 = h64 + rms(y64)
    torch.cuda.synchronize()
    # BF16 at six places in a row (x, y, h of two blocks), each half a step 2^-8, through products that add their errors up at random
    assert near(h, h64, 6 * 2.0 ** -8) and near(x, rms(h64), 7 * 2.0 ** -8)


def test_clipping_of_the_sharded_layer_in_a_group_of_one():
    import torch.distributed as dist
    T, H, F = 128, 256, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w, dy = (torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16) for s in ((T, H), (F, H), (T, F)))
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    os.environ.setdefault("MASTER_ADDR", "127.0.0.1")
    dist.init_process_group("nccl", init_method="tcp://127.0.0.1:%d" % port, rank=0, world_size=1)
    try:
        layer = DataParallelLinear(T, H, F)
        gain = torch.full((H,), 2.0, device="cuda")
        clipping = GradientClipping([layer.dw_shard], [gain])
        _, _, dw = layer.step(x, w, dy)
        before = dw.clone()
        alone = float(torch.sqrt(before.double().square().sum() + gain.double().square().sum()))
        clipping.world = 2                                   # the way of several ranks, whose sum is this rank's alone
        norm, factor = [float(v) for v in clipping.clip(0.5 * alone)]
        torch.cuda.synchronize()
        assert abs(norm - alone) <= 1e-6 * alone and abs(factor - 0.5) <= 1e-6
        assert torch.equal(dw, before * factor) and torch.equal(gain, torch.full_like(gain, 2.0) * factor)
        again = GradientClipping([layer.dw_shard], [gain]).clip(1e9)
        torch.cuda.synchronize()
        assert float(again[1]) == 1.0 and abs(float(again[0]) - 0.5 * alone) <= 1e-6 * alone
    finally:
        dist.destroy_process_group()
