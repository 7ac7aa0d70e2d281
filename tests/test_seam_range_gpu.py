"""The seam's gradient over the range of FP32.

Scaling a row's h by a power of two s and its 1 / rms by 1 / s leaves the normalised row as it is, and the same holds for y.  With dx scaled by s too,
every product and sum of the formulas is the same number times a power of two, so the results are the unscaled ones times powers of two,
bit by bit, as long as nothing leaves the range of normal FP32 (or BF16) numbers on the way.  No tolerance is needed."""
import pytest
import torch

from paper_2506_08027_b200 import binding as B

pytestmark = pytest.mark.gpu

T = {"bf16": torch.bfloat16, "fp32": torch.float32}


def gradient(d, seam, shapes):
    out = {k: torch.full(shape, 7.0, dtype=dtype, device="cuda") for k, (shape, dtype) in shapes.items()}
    rows, cols = d["y"].shape
    ws = torch.empty(B.mxfp8_residual_rmsnorm_grad_ws_bytes(seam, rows, cols), dtype=torch.uint8, device="cuda")
    B.mxfp8_residual_rmsnorm_grad(seam, d["dx"], d["dh"], d["y"], d["h"], d["rp"], d["rn"], out["dy"], out["dh_in"], out["d_gamma_pre"], out.get("d_gamma_post"),
                                  out.get("d_gate"), ws)
    torch.cuda.synchronize()
    return out


# one, two and four vectors per thread of the aligned kernel; one and two elements per access of the others; rows in shared memory
@pytest.mark.parametrize("cols", [512, 5120, 8200, 333, 1410, 5003, 8201])
@pytest.mark.parametrize("types", [("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp32")])
@pytest.mark.parametrize("post,gated", [(True, False), (True, True), (False, True)])
@pytest.mark.parametrize("power", [-66, 66])
def test_small_and_large_rows(cols, types, post, gated, power):
    rows, per_gate, s = 11, 4, 2.0 ** power
    g = torch.Generator(device="cuda").manual_seed(cols + 7 * post)
    rand = lambda *shape, scale=1.0, at=0.0, dtype=torch.float32: (at + scale * torch.randn(*shape, generator=g, device="cuda")).to(dtype)
    block, stream = T[types[0]], T[types[1]]
    gates = -(-rows // per_gate)
    seam = B.make_seam(rand(cols, scale=0.2, at=1.0, dtype=stream), rand(cols, scale=0.2, at=1.0, dtype=stream) if post else None,
                       rand(gates, cols, scale=0.5, dtype=stream) if gated else None, per_gate, 0.75, 0.5)
    # values that are not far below one: none gets near the subnormal numbers when it is scaled
    away = lambda t: torch.where(t.abs() < 2.0 ** -10, torch.full_like(t, 2.0 ** -10), t)
    d = dict(y=away(rand(rows, cols, scale=0.7)).to(block), h=away(rand(rows, cols, scale=2.0)).to(stream), dx=away(rand(rows, cols)).to(block), dh=away(rand(rows, cols)).to(stream))
    d["rn"] = d["h"].float().square().mean(dim=1).rsqrt()
    d["rp"] = d["y"].float().square().mean(dim=1).rsqrt() if post else None
    shapes = dict(dy=((rows, cols), block), dh_in=((rows, cols), stream), d_gamma_pre=((cols,), torch.float32))
    if post:
        shapes["d_gamma_post"] = ((cols,), torch.float32)
    if gated:
        shapes["d_gate"] = ((gates, cols), torch.float32)
    want = gradient(d, seam, shapes)
    scaled = dict(d, h=d["h"] * s, rn=d["rn"] / s, dx=d["dx"] * s)
    factor = dict(dy=1.0, dh_in=1.0, d_gamma_pre=s, d_gamma_post=1.0, d_gate=1.0)
    if post:
        scaled.update(y=d["y"] * s, rp=d["rp"] / s)
        factor["dy"] = 1 / s
    got = gradient(scaled, seam, shapes)
    for k, w in want.items():
        assert bool(w.isfinite().all()) and torch.equal(got[k], w * factor[k]), k
