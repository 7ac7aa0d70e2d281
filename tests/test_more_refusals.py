"""What the calls around a block's products refuse, before anything reaches a device.  No GPU: addresses are made up."""
import ctypes

import pytest
import torch

from paper_2506_08027_b200 import binding as B

A = 1 << 20                       # an aligned address that nothing reads


def seam(**other):
    d = dict(rows=64, cols=128, block_dtype=B.BF16, stream_dtype=B.BF16, param_dtype=B.BF16, gamma_post=A, gate=None, rows_per_gate=1, gamma_pre=A,
             branch_scale=1.0, residual_scale=1.0, eps=1e-5)
    return B._Seam(**{**d, **other})


SEAMS = [(dict(rows=0), B.ERR_SHAPE), (dict(cols=0), B.ERR_SHAPE), (dict(rows=-3), B.ERR_SHAPE), (dict(eps=-1.0), B.ERR_SHAPE), (dict(eps=float("nan")), B.ERR_SHAPE),
         (dict(gate=A, rows_per_gate=0), B.ERR_SHAPE), (dict(block_dtype=7), B.ERR_ENUM), (dict(stream_dtype=-1), B.ERR_ENUM), (dict(param_dtype=2), B.ERR_ENUM),
         (dict(gamma_pre=None), B.ERR_NULL), (dict(gamma_pre=A + 1), B.ERR_ALIGN), (dict(gamma_post=A + 1), B.ERR_ALIGN), (dict(gate=A + 1), B.ERR_ALIGN),
         (dict(cols=16385), B.ERR_UNSUPPORTED), (dict(rows=1 << 41), B.ERR_UNSUPPORTED)]


@pytest.mark.parametrize("wrong,status", SEAMS)
def test_descriptions_of_a_seam(wrong, status):
    L, s = B.lib(), seam(**wrong)
    assert L.mxfp8_residual_rmsnorm(s, A, A, A, A, A, A, None) == status
    assert L.mxfp8_residual_rmsnorm_quantize(s, A, A, A, A, A, B.ROW, B.RULE_PAPER, B.E4M3, A, A, None, None, B.SF_SWIZZLED, None) == status
    assert L.mxfp8_residual_rmsnorm_grad(s, A, A, A, A, A, A, A, A, A, A, None, A, 1 << 30, None) == status
    assert L.mxfp8_residual_rmsnorm_grad_ws_bytes(s) == 0


def test_pointers_of_a_seam():
    L = B.lib()
    forward = lambda s=seam(), y=A, h_in=A, h=A, x=A, rp=A, rn=A: L.mxfp8_residual_rmsnorm(s, y, h_in, h, x, rp, rn, None)
    assert L.mxfp8_residual_rmsnorm(None, A, A, A, A, A, A, None) == B.ERR_NULL
    for k in ("y", "h_in", "h", "rp", "rn"):
        assert forward(**{k: None}) == B.ERR_NULL
        assert forward(**{k: A + 1}) == B.ERR_ALIGN
    assert forward(x=A + 1) == B.ERR_ALIGN
    assert forward(s=seam(stream_dtype=B.FP32), h=A + 2) == B.ERR_ALIGN
    quantize = lambda s=seam(), h=A, orientation=B.ROW, elem=B.E4M3, q=A, sc=A: L.mxfp8_residual_rmsnorm_quantize(
        s, A, A, h, A, A, orientation, B.RULE_PAPER, elem, q, sc, A, A, B.SF_SWIZZLED, None)
    assert quantize(s=seam(param_dtype=B.FP32)) == B.ERR_UNSUPPORTED
    assert quantize(s=seam(cols=144)) == B.ERR_SHAPE and quantize(s=seam(rows=33), orientation=B.COL) == B.ERR_SHAPE
    assert quantize(orientation=0) == B.ERR_ENUM and quantize(elem=2) == B.ERR_ENUM
    assert quantize(q=None) == B.ERR_NULL and quantize(sc=A + 8) == B.ERR_ALIGN and quantize(h=A + 2) == B.ERR_ALIGN

    def grad(s=seam(), dx=A, dh=A, y=A, h=A, rp=A, rn=A, dy=A, dh_in=A, pre=A, post=A, gate=None, ws=A, n=1 << 30):
        return L.mxfp8_residual_rmsnorm_grad(s, dx, dh, y, h, rp, rn, dy, dh_in, pre, post, gate, ws, n, None)
    for k in ("y", "h", "rp", "rn"):
        assert grad(**{k: None}) == B.ERR_NULL
    for k in ("dx", "dh", "y", "h", "rp", "rn", "dy", "dh_in", "pre", "post"):
        assert grad(**{k: A + 1}) == B.ERR_ALIGN
    assert grad(gate=A) == B.ERR_NULL and grad(s=seam(gamma_post=None)) == B.ERR_NULL         # gradients of weights that the seam does not have
    assert grad(ws=None) == B.ERR_WORKSPACE and grad(n=8) == B.ERR_WORKSPACE and grad(ws=A + 8) == B.ERR_ALIGN


def items(*entries):
    c = (B._GradItem * max(1, len(entries)))()
    for k, (src, dst, numel, dtype) in enumerate(entries):
        c[k].src, c[k].dst, c[k].numel, c[k].dtype = src, dst, numel, dtype
    return c


GOOD = (A, A, 100, B.FP32)


@pytest.mark.parametrize("entry,status", [((A, A, 100, 3), B.ERR_ENUM), ((A, A, -1, B.FP32), B.ERR_SHAPE), ((None, A, 1, B.FP32), B.ERR_NULL),
                                          ((A + 2, A, 1, B.FP32), B.ERR_ALIGN), ((A + 1, A, 1, B.BF16), B.ERR_ALIGN), ((A, A, 1 << 40, B.BF16), B.ERR_UNSUPPORTED)])
def test_gradients(entry, status):
    L, c = B.lib(), items(GOOD, entry)
    n = L.mxfp8_grad_ws_bytes(c, 2)
    assert L.mxfp8_grad_sumsq(c, 2, A, A, n, None) == status
    assert L.mxfp8_grad_scale(c, 2, A, 1.0, A, None) == status
    assert L.mxfp8_grad_clip(c, 2, 1.0, A, A, n, None) == status


def test_arguments_beside_the_gradients():
    L, c = B.lib(), items(GOOD)
    n = L.mxfp8_grad_ws_bytes(c, 1)
    assert L.mxfp8_grad_ws_bytes(c, -1) == 0
    for bad in (-1.0, float("nan")):
        assert L.mxfp8_grad_clip(c, 1, bad, A, A, n, None) == B.ERR_SHAPE and L.mxfp8_grad_scale(c, 1, A, bad, A, None) == B.ERR_SHAPE
    assert L.mxfp8_grad_clip(c, -1, 1.0, A, A, n, None) == B.ERR_SHAPE and L.mxfp8_grad_clip(None, 1, 1.0, A, A, n, None) == B.ERR_NULL
    assert L.mxfp8_grad_clip(c, 1, 1.0, None, A, n, None) == B.ERR_NULL and L.mxfp8_grad_clip(c, 1, 1.0, A + 1, A, n, None) == B.ERR_ALIGN
    assert L.mxfp8_grad_clip(c, 1, 1.0, A, None, n, None) == B.ERR_WORKSPACE and L.mxfp8_grad_clip(c, 1, 1.0, A, A, n - 1, None) == B.ERR_WORKSPACE
    assert L.mxfp8_grad_clip(c, 1, 1.0, A, A + 4, n, None) == B.ERR_ALIGN
    assert L.mxfp8_grad_sumsq(c, 1, None, A, n, None) == B.ERR_NULL and L.mxfp8_grad_sumsq(c, 1, A + 4, A, n, None) == B.ERR_ALIGN
    assert L.mxfp8_grad_scale(c, 1, None, 1.0, A, None) == B.ERR_NULL and L.mxfp8_grad_scale(c, 1, A + 4, 1.0, A, None) == B.ERR_ALIGN
    assert L.mxfp8_grad_clip(items((A, None, 5, B.FP32)), 1, 1.0, A, A, n, None) == B.ERR_NULL


def test_few_token_layer():
    L = B.lib()

    def moe(x=A, logits=A, tokens=2, cols=64, experts=4, top_k=2, gate_up=A, down=A, inner=32, act=B.ACT_SILU, y=A, out=B.BF16, ids=A, weights=A, ws=A, n=1 << 20):
        return L.mxfp8_e2m1_moe(x, logits, tokens, cols, experts, top_k, gate_up, down, inner, act, 1, y, out, ids, weights, ws, n, None)
    for k in ("x", "logits", "gate_up", "down", "y"):
        assert moe(**{k: None}) == B.ERR_NULL
    for k in ("x", "gate_up", "down", "ws"):
        assert moe(**{k: A + 8}) == B.ERR_ALIGN
    for k in ("logits", "ids", "weights"):
        assert moe(**{k: A + 2}) == B.ERR_ALIGN
    assert moe(y=A + 1) == B.ERR_ALIGN and moe(out=B.FP32, y=A + 2) == B.ERR_ALIGN
    assert moe(out=5) == B.ERR_ENUM and moe(act=5) == B.ERR_ENUM and moe(act=-1) == B.ERR_ENUM
    for k, v in (("tokens", 0), ("cols", 0), ("cols", 48), ("inner", 40), ("inner", -32), ("experts", 0), ("top_k", 0), ("top_k", 5)):
        assert moe(**{k: v}) == B.ERR_SHAPE, (k, v)
    assert moe(tokens=65) == B.ERR_UNSUPPORTED and moe(experts=257) == B.ERR_UNSUPPORTED and moe(experts=40, top_k=17) == B.ERR_UNSUPPORTED
    assert moe(ws=None) == B.ERR_WORKSPACE and moe(n=100) == B.ERR_WORKSPACE
    assert L.mxfp8_e2m1_moe_ws_bytes(0, 2, 32) == 0 and L.mxfp8_e2m1_moe_ws_bytes(65, 2, 32) == 0


@pytest.fixture
def no_device(monkeypatch):
    monkeypatch.setattr(B, "_stream_for", lambda stream, *tensors: 5)
    monkeypatch.setattr(B, "_current_device", lambda: -1)                 # what a host tensor says of itself

    class Nothing:
        def __getattr__(self, name):
            return lambda *args: 1 << 40 if name.endswith("_bytes") else 0
    monkeypatch.setattr(B, "lib", Nothing)


def test_the_binding_refuses_tensors_that_do_not_agree(no_device):
    f, b = torch.float32, torch.bfloat16
    t = lambda *shape, dtype=b: torch.zeros(*shape, dtype=dtype)
    s = B.make_seam(t(128), t(128), t(2, 128), 4)
    good = dict(seam=s, y=t(8, 128), h_in=t(8, 128), h=t(8, 128), x=t(8, 128), rstd_post=t(8, dtype=f), rstd_pre=t(8, dtype=f))
    B.mxfp8_residual_rmsnorm(**good)
    for wrong in (dict(h=t(8, 128, dtype=f)), dict(x=t(8, 127)), dict(h_in=t(7, 128), h=t(7, 128)), dict(rstd_pre=t(7, dtype=f)), dict(rstd_post=t(8)),
                  dict(y=t(12, 128), h_in=t(12, 128), h=t(12, 128), x=None, rstd_pre=t(12, dtype=f), rstd_post=t(12, dtype=f)),       # three rows of the gate are needed
                  dict(seam=B.make_seam(t(64), t(64)))):
        with pytest.raises((ValueError, TypeError)):
            B.mxfp8_residual_rmsnorm(**{**good, **wrong})
    with pytest.raises(ValueError):
        B.mxfp8_residual_rmsnorm(**{**good, "y": t(128, 8).t()})
    grad = dict(seam=s, dx=t(8, 128), dh=t(8, 128), y=t(8, 128), h=t(8, 128), rstd_post=t(8, dtype=f), rstd_pre=t(8, dtype=f), dy=t(8, 128), dh_in=t(8, 128),
                d_gamma_pre=t(128, dtype=f), d_gamma_post=t(128, dtype=f), d_gate=t(2, 128, dtype=f), ws=t(8))
    B.mxfp8_residual_rmsnorm_grad(**grad)
    for wrong in (dict(d_gate=t(1, 128, dtype=f)), dict(d_gamma_pre=t(128)), dict(dx=t(8, 128, dtype=f)), dict(dh_in=t(8, 64)),
                  dict(seam=B.make_seam(t(128)), d_gate=None), dict(seam=B.make_seam(t(128), t(128)))):
        with pytest.raises(ValueError):
            B.mxfp8_residual_rmsnorm_grad(**{**grad, **wrong})
    for wrong in ((t(128), t(64)), (t(128), t(128, dtype=f)), (t(2, 64),), (t(128), None, t(128)), (t(128), None, t(2, 128), 0)):
        with pytest.raises(ValueError):
            B.make_seam(*wrong)
    moe = dict(x=t(2, 64), logits=t(2, 4, dtype=f), top_k=2, gate_up=t(8), down=t(8), inner=32, act=B.ACT_SILU, renormalize=True, y=t(2, 64),
               ids=t(2, 2, dtype=torch.int32), weights=t(2, 2, dtype=f), ws=t(8))
    for wrong in (dict(x=t(2, 64, dtype=f)), dict(logits=t(2, 4)), dict(ids=t(2, 2, dtype=torch.int64)), dict(weights=t(2, 3, dtype=f)),
                  dict(logits=t(3, 4, dtype=f)), dict(y=t(2, 32)), dict(ids=t(2, 3, dtype=torch.int32)), dict()):            # the last: matrices too small
        with pytest.raises((ValueError, TypeError)):
            B.mxfp8_e2m1_moe(**{**moe, **wrong})
    for grads, results in (([t(4)], [t(4, dtype=f)]), ([t(4)], [t(5)]), ([t(4)], []), ([t(4)], None)):                       # the last: a host tensor
        with pytest.raises(ValueError):
            B.make_grad_items(grads, results)
    assert ctypes.sizeof(B._GradItem) == 32 and ctypes.sizeof(B._Seam) == 80
