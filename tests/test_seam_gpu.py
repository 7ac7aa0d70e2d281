"""The seam between two blocks, forward and backward, against the formulas in 64 bits.

Tolerances count roundings: u = 2^-24 for one FP32 rounding, half a step of the stored type for a result.  A mean over c columns
that 256 threads (at least) form has at most c / 128 + 64 additions on the way to any term, so its relative error is below D = (c / 128 + 64) u
of the sum of its terms' absolute values; everything elementwise has at most eight roundings.
"""
import pytest
import torch

from paper_2506_08027_b200 import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
T = {"bf16": torch.bfloat16, "fp32": torch.float32}
TYPES = [("bf16", "bf16", "bf16"), ("bf16", "fp32", "fp32"), ("fp32", "fp32", "bf16"), ("fp32", "bf16", "fp32")]
SHAPES = [(1, 1), (2, 7), (5, 100), (3, 1409), (37, 768), (301, 2048), (2, 4096), (3, 5120), (2, 16384), (1500, 40), (700, 256), (9, 8200), (4, 16376), (1201, 1024)]


def half_step(t):
    return torch.finfo(t).eps / 2


def place(shape, dtype, shift=0):
    """A tensor inside a larger buffer of a known pattern, `shift` elements behind a 16-byte boundary, and the buffer."""
    n = 1
    for s in shape:
        n *= s
    buf = torch.full((n + 64,), 7.0, dtype=dtype, device="cuda")
    return buf[16 + shift:16 + shift + n].view(shape), buf


def untouched(buf, n, shift=0):
    assert bool((buf[:16 + shift] == 7.0).all()) and bool((buf[16 + shift + n:] == 7.0).all()), "written outside the tensor"


def inputs(rows, cols, types, post, per_gate, seed=0, shift=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 31 * rows + cols)
    block, stream, params = (T[t] for t in types)

    def rand(*shape, dtype, scale=1.0, at=0.0):
        t, _ = place(shape, dtype, shift)
        t.copy_(at + scale * torch.randn(*shape, generator=g, device="cuda"))
        return t
    d = dict(y=rand(rows, cols, dtype=block, scale=0.7), h_in=rand(rows, cols, dtype=stream, scale=2.0), gamma_pre=rand(cols, dtype=params, scale=0.2, at=1.0))
    d["gamma_post"] = rand(cols, dtype=params, scale=0.2, at=1.0) if post else None
    gates = -(-rows // per_gate) if per_gate else 0
    d["gate"] = rand(gates, cols, dtype=params, scale=0.5) if per_gate else None
    d["dx"], d["dh"] = rand(rows, cols, dtype=block, scale=1e-3), rand(rows, cols, dtype=stream, scale=1e-3)
    return d


def gate_rows(d, rows, per_gate):
    return torch.ones(1, 1, dtype=torch.float64, device="cuda") if d["gate"] is None else d["gate"].double()[torch.arange(rows, device="cuda") // per_gate]


CASES = [(s, TYPES[i % 4], (True, False, True, True, False)[i % 5], (0, 1, 3, 0, 100, 613)[(i + i // 6) % 6], i % 3 == 1) for i, s in enumerate(SHAPES)]
CASES += [((260, 1152), t, p, g, False) for t in TYPES for p, g in ((True, 65), (False, 0), (True, 0))]


@pytest.mark.parametrize("shape,types,post,per_gate,odd", CASES)
def test_forward(shape, types, post, per_gate, odd):
    rows, cols = shape
    shift, eps = int(odd), 1e-5
    d = inputs(rows, cols, types, post, per_gate, shift=shift)
    block, stream = T[types[0]], T[types[1]]
    seam = B.make_seam(d["gamma_pre"], d["gamma_post"], d["gate"], max(1, per_gate), 0.75, 0.5, eps)
    h, hbuf = place((rows, cols), stream, shift)
    x, xbuf = place((rows, cols), block, shift)
    rp, rpbuf = place((rows,), torch.float32)
    rn, rnbuf = place((rows,), torch.float32)
    B.mxfp8_residual_rmsnorm(seam, d["y"], d["h_in"], h, x, rp if post else None, rn)
    torch.cuda.synchronize()
    for buf, n, s in ((hbuf, rows * cols, shift), (xbuf, rows * cols, shift), (rpbuf, rows, 0), (rnbuf, rows, 0)):
        untouched(buf, n, s)
    D = (cols / 128 + 64) * U
    n = d["y"].double()
    if post:
        want = (n.square().mean(dim=1) + eps) ** -0.5
        assert bool(((rp.double() - want).abs() <= (D + 3 * U) * want).all())
        n = n * want.unsqueeze(1) * d["gamma_post"].double()
    branch = 0.75 * gate_rows(d, rows, per_gate) * n
    want = 0.5 * d["h_in"].double() + branch
    slack = (D + 8 * U) * (branch.abs() + (0.5 * d["h_in"].double()).abs())
    assert bool(((h.double() - want).abs() <= (half_step(stream) if stream != torch.float32 else U) * (want.abs() + slack) + slack).all())
    # from here on what the call stored
    s = h.double()
    want = (s.square().mean(dim=1) + eps) ** -0.5
    assert bool(((rn.double() - want).abs() <= (D + 3 * U) * want).all())
    want = s * rn.double().unsqueeze(1) * d["gamma_pre"].double()
    assert bool(((x.double() - want).abs() <= (half_step(block) + 3 * U) * want.abs()).all())
    # in place, and without the norm's output
    again = d["h_in"].clone()
    B.mxfp8_residual_rmsnorm(seam, d["y"], again, again, None, rp if post else None, rn)
    assert torch.equal(again, h)


@pytest.mark.parametrize("shape,types,post,per_gate,odd", CASES)
def test_backward(shape, types, post, per_gate, odd):
    rows, cols = shape
    shift, eps, bs, rs = int(odd), 1e-5, 0.75, 0.5
    d = inputs(rows, cols, types, post, per_gate, seed=1, shift=shift)
    block, stream = T[types[0]], T[types[1]]
    seam = B.make_seam(d["gamma_pre"], d["gamma_post"], d["gate"], max(1, per_gate), bs, rs, eps)
    y, h = d["y"].double(), d["h_in"].double()
    rp = ((y.square().mean(dim=1) + eps) ** -0.5).float()
    rn = ((h.square().mean(dim=1) + eps) ** -0.5).float()
    dy, dybuf = place((rows, cols), block, shift)
    dh_in, dhbuf = place((rows, cols), stream, shift)
    outs = {k: place(d[k].shape, torch.float32) for k in ("gamma_pre", "gamma_post", "gate") if d[k] is not None}
    ws = torch.empty(B.mxfp8_residual_rmsnorm_grad_ws_bytes(seam, rows, cols), dtype=torch.uint8, device="cuda")
    got = [outs[k][0] if k in outs else None for k in ("gamma_pre", "gamma_post", "gate")]
    B.mxfp8_residual_rmsnorm_grad(seam, d["dx"], d["dh"], d["y"], d["h_in"], rp if post else None, rn, dy, dh_in, *got, ws)
    torch.cuda.synchronize()
    for buf in (dybuf, dhbuf):
        untouched(buf, rows * cols, shift)
    for t, buf in outs.values():
        untouched(buf, t.numel())
    D, mean = (cols / 128 + 64) * U, lambda v: v.mean(dim=1, keepdim=True)
    rnc, rpc = rn.double().unsqueeze(1), rp.double().unsqueeze(1)
    dx, dh, gp = d["dx"].double(), d["dh"].double(), d["gamma_pre"].double()
    xh, t = h * rnc, dx * gp
    c1 = mean(t * xh)
    G = dh + rnc * (t - xh * c1)
    slack = 8 * U * (dh.abs() + rnc * (t.abs() + (xh * c1).abs())) + rnc * xh.abs() * (D + 4 * U) * mean((t * xh).abs())
    want = rs * G
    assert bool(((dh_in.double() - want).abs() <= (half_step(stream)) * want.abs() + 2 * rs * slack).all())
    gate = gate_rows(d, rows, per_gate)
    w = bs * gate * G
    wslack = bs * gate.abs() * (slack + 4 * U * G.abs())
    if post:
        yh, gamma = y * rpc, d["gamma_post"].double()
        u = w * gamma
        want = rpc * (u - yh * mean(u * yh))
        k = (bs * gate * gamma * yh)
        # the mean is put together from three sums over the row
        terms = mean((k * dh).abs()) + mean((k * rnc * t).abs()) + rnc * mean((t * xh).abs()) * mean((k * xh).abs())
        dslack = rpc * (gamma.abs() * wslack + 8 * U * (u.abs() + (yh * mean(u * yh)).abs()) + yh.abs() * 2 * (D + 8 * U) * terms)
    else:
        yh, want, dslack = y, w, wslack
    assert bool(((dy.double() - want).abs() <= half_step(block) * want.abs() + 2 * dslack).all())
    # sums over rows: at most 128 additions on the way to a term for so few rows
    R = (min(rows, 128) + 64) * U

    def close(got, terms, term_slack, index=None):
        gates = got.shape[0] if got.dim() == 2 else 1
        at = torch.arange(rows, device="cuda") // per_gate if got.dim() == 2 else torch.zeros(rows, dtype=torch.long, device="cuda")
        zero = torch.zeros(gates, cols, dtype=torch.float64, device="cuda")
        want, size, more = (zero.clone().index_add_(0, at, v) for v in (terms, terms.abs(), term_slack))
        assert bool(((got.double().view(gates, cols) - want).abs() <= (R + 8 * U) * size + 2 * more + 1e-40).all())
    close(got[0], dx * xh, 4 * U * (dx * xh).abs())
    if post:
        close(got[1], w * yh, yh.abs() * wslack)
    if d["gate"] is not None:
        n = yh * (d["gamma_post"].double() if post else 1.0)
        close(got[2], bs * G * n, bs * n.abs() * (slack + 4 * U * G.abs()))
    # the same again, one output at a time and without one of the inputs
    for name in ("dy", "dh_in", "d_gamma_pre", "d_gamma_post", "d_gate"):
        full = dict(dy=dy, dh_in=dh_in, d_gamma_pre=got[0], d_gamma_post=got[1], d_gate=got[2])
        if full[name] is None:
            continue
        one = {k: (torch.zeros_like(v) if k == name else None) for k, v in full.items()}
        B.mxfp8_residual_rmsnorm_grad(seam, d["dx"], d["dh"], d["y"], d["h_in"], rp if post else None, rn, ws=ws, **one)
        assert torch.equal(one[name], full[name]), name
    inplace = d["dh"].clone()
    B.mxfp8_residual_rmsnorm_grad(seam, d["dx"], inplace, d["y"], d["h_in"], rp if post else None, rn, None, inplace, None, None, None, ws)
    assert torch.equal(inplace, dh_in)


def test_backward_against_differences():
    """The loss is <dx, x> + <dh, h>, in FP32 through the forward call; its difference quotients have an error of about the cube root of U."""
    rows, cols, per_gate = 12, 96, 5
    d = inputs(rows, cols, ("fp32", "fp32", "fp32"), True, per_gate, seed=3)
    x, h = torch.empty_like(d["y"]), torch.empty_like(d["y"])
    rp, rn = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")

    def loss(p):
        B.mxfp8_residual_rmsnorm(B.make_seam(p["gamma_pre"], p["gamma_post"], p["gate"], per_gate, 0.75, 0.5), p["y"], p["h_in"], h, x, rp, rn)
        return float((x.double() * d["dx"].double()).sum() + (h.double() * d["dh"].double()).sum())
    loss(d)
    seam = B.make_seam(d["gamma_pre"], d["gamma_post"], d["gate"], per_gate, 0.75, 0.5)
    out = {k: torch.empty_like(d[k]) for k in ("y", "h_in", "gamma_pre", "gamma_post", "gate")}
    ws = torch.empty(B.mxfp8_residual_rmsnorm_grad_ws_bytes(seam, rows, cols), dtype=torch.uint8, device="cuda")
    B.mxfp8_residual_rmsnorm_grad(seam, d["dx"], d["dh"], d["y"], h, rp, rn, out["y"], out["h_in"], out["gamma_pre"], out["gamma_post"], out["gate"], ws)
    for name, grad in out.items():
        way = torch.randn(grad.shape, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
        step = 2.0 ** -8
        up, down = loss({**d, name: d[name] + step * way}), loss({**d, name: d[name] - step * way})
        want = float((grad.double() * way.double()).sum())
        # second-order error step^2 and rounding U / step of a loss of this many terms, both relative to the terms' size
        size = float((grad.double() * way.double()).abs().sum()) + 1e-3 * (rows * cols) ** 0.5
        assert abs((up - down) / (2 * step) - want) <= 40 * (step ** 2 + U / step) * size, name


def test_converted_output_is_that_of_the_separate_call():
    for rows, cols, stream, orientation, layout in ((64, 512, "bf16", B.BOTH, B.SF_SWIZZLED), (96, 160, "fp32", B.ROW, B.SF_LINEAR), (32, 4096, "bf16", B.COL, B.SF_SWIZZLED),
                                                    (1, 4096, "bf16", B.ROW, B.SF_SWIZZLED), (333, 1056, "bf16", B.ROW, B.SF_SWIZZLED),
                                                    (130, 2048, "fp32", B.ROW, B.SF_SWIZZLED), (160, 96, "fp32", B.BOTH, B.SF_LINEAR),
                                                    (1300, 256, "bf16", B.ROW, B.SF_SWIZZLED), (1201, 416, "bf16", B.ROW, B.SF_LINEAR), (1190, 1024, "fp32", B.ROW, B.SF_SWIZZLED),
                                                    (260, 6176, "bf16", B.ROW, B.SF_SWIZZLED), (2, 16384, "bf16", B.ROW, B.SF_LINEAR), (3, 16352, "fp32", B.ROW, B.SF_SWIZZLED)):
        for elem, rule in ((B.E4M3, B.RULE_PAPER), (B.E5M2, B.RULE_OCP), (B.E2M1, B.RULE_PAPER)):
            d = inputs(rows, cols, ("bf16", stream, stream), True, 0, seed=4)
            seam = B.make_seam(d["gamma_pre"], d["gamma_post"], None, 1, 1.0, 1.0, 1e-6)
            h, ref = torch.empty_like(d["h_in"]), torch.empty_like(d["h_in"])
            rp, rn, rn2 = (torch.empty(rows, device="cuda") for _ in range(3))
            outs = [None if o is None else o.fill_(0xA5) for o in B.alloc_quantize_outputs(rows, cols, orientation, layout)]
            want = [None if o is None else o.fill_(0xA5) for o in B.alloc_quantize_outputs(rows, cols, orientation, layout)]
            B.mxfp8_residual_rmsnorm(seam, d["y"], d["h_in"], ref, None, rp, rn2)
            B.mxfp8_residual_rmsnorm_quantize(seam, d["y"], d["h_in"], h, rp, rn, orientation, rule, elem, *outs, layout)
            assert torch.equal(h, ref) and torch.equal(rn, rn2)
            # the separate conversion of y = (h rstd) gamma, rounded to the stream's type as its definition says
            x = ((h.float() * rn.unsqueeze(1)) * d["gamma_pre"].float()).to(h.dtype)
            B.mxfp8_quantize(x, orientation, rule, elem, *want, layout)
            for got, w in zip(outs, want):
                assert (got is None) == (w is None) and (got is None or torch.equal(got, w)), (rows, cols, stream, orientation, elem)


@pytest.mark.parametrize("orientation", [B.ROW, B.BOTH])
def test_conversion_of_infinities_nan_and_zero_rows(orientation):
    """Infinities and NaN in x (from the weights) saturate and stay, and neither enters a block's largest magnitude."""
    rows, cols = 64, 256
    for elem in (B.E4M3, B.E5M2):
        d = inputs(rows, cols, ("bf16", "bf16", "bf16"), True, 0, seed=9)
        d["gamma_pre"][5], d["gamma_pre"][40], d["gamma_pre"][200] = float("inf"), float("nan"), float("-inf")
        d["gamma_pre"][96:128] = float("inf")                        # a block without a finite element
        d["y"][7] = 0
        d["h_in"][7] = 0
        seam = B.make_seam(d["gamma_pre"], d["gamma_post"])
        h, rp, rn = torch.empty_like(d["h_in"]), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        outs, want = (B.alloc_quantize_outputs(rows, cols, orientation, B.SF_SWIZZLED) for _ in range(2))
        B.mxfp8_residual_rmsnorm_quantize(seam, d["y"], d["h_in"], h, rp, rn, orientation, B.RULE_PAPER, elem, *outs, B.SF_SWIZZLED)
        x = ((h.float() * rn.unsqueeze(1)) * d["gamma_pre"].float()).to(h.dtype)
        B.mxfp8_quantize(x, orientation, B.RULE_PAPER, elem, *want, B.SF_SWIZZLED)
        for k, (got, w) in enumerate(zip(outs, want)):
            if got is None:
                continue
            if k % 2 == 0:                                            # codes: any NaN for a NaN
                got, w = (t.view(torch.float8_e4m3fn if elem == B.E4M3 else torch.float8_e5m2).float() for t in (got, w))
                assert torch.equal(got.isnan(), w.isnan())
                got, w = got.nan_to_num(0.0), w.nan_to_num(0.0)
            assert torch.equal(got, w)


def test_zero_rows_and_special_values():
    """All-zero rows with eps > 0 give zeros; a NaN or an infinity stays in its row (and, backward, in its columns' sums)."""
    rows, cols = 6, 512
    d = inputs(rows, cols, ("bf16", "bf16", "bf16"), True, 0, seed=6)
    d["y"][1] = 0
    d["h_in"][1] = 0
    d["y"][3, 17] = float("nan")
    d["h_in"][4, 5] = float("inf")
    seam = B.make_seam(d["gamma_pre"], d["gamma_post"])
    h, x = torch.empty_like(d["h_in"]), torch.empty_like(d["y"])
    rp, rn = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.mxfp8_residual_rmsnorm(seam, d["y"], d["h_in"], h, x, rp, rn)
    assert bool((x[1] == 0).all()) and bool((h[1] == 0).all())
    assert bool(x[3].isnan().all()) and float(rn[4]) == 0.0 and bool(x[4, 5].isnan()) and bool((x[4, 6:] == 0).all())
    assert bool(x[[0, 2, 5]].isfinite().all())


@pytest.mark.parametrize("rows,cols", [(64, 2048), (7, 333)])
def test_streams_graphs_and_two_calls_at_once(rows, cols):
    d = inputs(rows, cols, ("bf16", "bf16", "bf16"), True, 9, seed=8)
    seam = B.make_seam(d["gamma_pre"], d["gamma_post"], d["gate"], 9)
    n = lambda: (torch.empty_like(d["h_in"]), torch.empty_like(d["y"]), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"))
    grads = lambda: (torch.zeros_like(d["y"]), torch.zeros_like(d["h_in"]), torch.zeros(cols, device="cuda"), torch.zeros(cols, device="cuda"),
                     torch.zeros(d["gate"].shape, device="cuda"))
    size = B.mxfp8_residual_rmsnorm_grad_ws_bytes(seam, rows, cols)
    ws = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def call(f, g, w):
        B.mxfp8_residual_rmsnorm(seam, d["y"], d["h_in"], *f)
        B.mxfp8_residual_rmsnorm_grad(seam, d["dx"], d["dh"], d["y"], f[0], f[2], f[3], *g, w)
    first, gfirst = n(), grads()
    call(first, gfirst, ws[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    fs, gs = [n(), n()], [grads(), grads()]
    for s, f, g, w in zip(streams, fs, gs, ws):
        with torch.cuda.stream(s):
            for _ in range(3):
                call(f, g, w)
    torch.cuda.synchronize()
    for f, g in zip(fs, gs):
        assert all(torch.equal(a, b) for a, b in zip(f + g, first + gfirst))
    graph, captured, gcaptured = torch.cuda.CUDAGraph(), n(), grads()
    with torch.cuda.graph(graph):
        call(captured, gcaptured, ws[0])
    d["y"].mul_(0.5)
    d["dx"].mul_(-2.0)
    graph.replay()
    torch.cuda.synchronize()
    call(first, gfirst, ws[1])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(captured + gcaptured, first + gfirst))
