"""Sorting tokens by expert, moving them into MXFP8 and back, and the gradients (App. A.4's layer), against the oracle."""
import numpy as np
import pytest

import oracle as orc
from paper_2506_08027_b200 import synth
from helpers import assert_q_equal, logical_scales_from_swizzled

pytestmark = pytest.mark.gpu


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def as_dtype(x, dtype):
    """float32 array -> (device tensor of `dtype`, its values as float32)."""
    import torch
    t = dev(x.astype(np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    return t, t.float().cpu().numpy()


def routing(tokens, top_k, experts, seed, kind="random"):
    rng = np.random.default_rng(seed)
    if kind == "one":
        return np.full((tokens, top_k), experts - 1, np.int32)
    if kind == "none":
        return np.full((tokens, top_k), -1, np.int32)
    ids = rng.integers(0, experts, (tokens, top_k)).astype(np.int32)
    if kind == "holes":
        ids[rng.random((tokens, top_k)) < 0.3] = -1
        ids[rng.random((tokens, top_k)) < 0.05] = experts + 3
        ids[ids == 0] = min(1, experts - 1)                       # an expert without tokens
    if kind == "skewed":
        ids[rng.random((tokens, top_k)) < 0.9] = experts // 2
    return ids


def gpu_sort(ids, experts, spare=0, ws=None):
    """Sorted by the library, in buffers full of a mark so that what is not written shows."""
    import torch
    from paper_2506_08027_b200 import binding as B
    tokens, top_k = ids.shape
    rows = B.mxfp8_moe_rows(tokens, top_k, experts) + spare
    mark = lambda *s: torch.full(s, -77, dtype=torch.int32, device="cuda")
    off, row_of, slot_of = mark(experts + 1), mark(tokens, top_k), mark(rows)
    need = B.mxfp8_moe_sort_ws_bytes(tokens, top_k, experts)
    ws = torch.full((need,), 0xA5, dtype=torch.uint8, device="cuda") if ws is None and need else ws
    B.mxfp8_moe_sort(dev(ids), experts, off, row_of, slot_of, ws)
    return off, row_of, slot_of


SIZES = [(1, 1, 1), (1, 6, 64), (3, 2, 5), (16, 6, 64), (129, 1, 2), (500, 8, 256), (683, 6, 60), (1365, 3, 7),
         (1367, 3, 7), (4097, 1, 1), (5000, 2, 256), (20011, 7, 255)]


@pytest.mark.parametrize("tokens,top_k,experts", SIZES)
@pytest.mark.parametrize("kind", ["random", "holes", "skewed", "one", "none"])
def test_sort_equals_the_oracle(tokens, top_k, experts, kind):
    from paper_2506_08027_b200 import binding as B
    ids = routing(tokens, top_k, experts, tokens + top_k, kind)
    off, row_of, slot_of = gpu_sort(ids, experts, spare=5)
    w_off, w_row, w_slot = orc.moe_sort(ids, experts, slot_of.numel())
    assert np.array_equal(off.cpu().numpy(), w_off)
    assert np.array_equal(row_of.cpu().numpy(), w_row)
    assert np.array_equal(slot_of.cpu().numpy(), w_slot)
    assert B.mxfp8_device_status() == 0


def test_sort_of_no_tokens():
    import torch
    from paper_2506_08027_b200 import binding as B
    off = torch.full((9,), 7, dtype=torch.int32, device="cuda")
    slot_of = torch.full((256,), 7, dtype=torch.int32, device="cuda")
    none = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    B.mxfp8_moe_sort(none, 8, off, none, slot_of)
    assert not off.any() and (slot_of == -1).all()
    B.mxfp8_moe_combine(torch.ones(0, 16, device="cuda"), none, None, torch.empty(0, 16, device="cuda"))


def check_conversion(got, y, rows, used, orientation, rule, elem, layout, what):
    """got: (q_row, s_row, q_col, s_col) device buffers that held 0xA5; y: the rows in use as float32."""
    from paper_2506_08027_b200 import binding as B
    cols = y.shape[1]
    for o, q, s in ((B.ROW, got[0], got[1]), (B.COL, got[2], got[3])):
        if not orientation & o:
            continue
        q, s = q.cpu().numpy().reshape(rows, cols), s.cpu().numpy()
        assert (q[used:] == 0xA5).all(), "rows behind the last segment were written " + what
        q = q[:used]
        if used == 0:
            assert (s == 0xA5).all()
            continue
        wq, ws = orc.quantize(y, orc.ROW if o == B.ROW else orc.COL, rule, elem)
        if orc.code_bits(elem) < 8:
            q = orc.unpack_codes16(q, elem)
            assert np.array_equal(q, wq), what
        else:
            assert_q_equal(q, wq, elem, what)
        if o == B.ROW:
            logical = logical_scales_from_swizzled(s, rows, cols // 32)[:used] if layout == B.SF_SWIZZLED else s.reshape(rows, cols // 32)[:used]
            assert np.array_equal(logical, ws), "row scales " + what
            if layout == B.SF_LINEAR:
                assert (s.reshape(rows, -1)[used:] == 0xA5).all(), what
        else:
            if layout == B.SF_SWIZZLED:
                logical = logical_scales_from_swizzled(s, cols, rows // 32)[:, :used // 32].T
            else:
                logical = s.reshape(rows // 32, cols)[:used // 32]
                assert (s.reshape(rows // 32, cols)[used // 32:] == 0xA5).all(), what
            assert np.array_equal(logical, ws), "column scales " + what


def run_dispatch(x, dtype, ids, experts, weights, orientation, rule, elem, layout, spare_tiles=1, what=""):
    import torch
    from paper_2506_08027_b200 import binding as B
    tokens, top_k = ids.shape
    cols = x.shape[1]
    src, values = as_dtype(x, dtype)
    off, _, slot_of = gpu_sort(ids, experts, spare=128 * spare_tiles)
    rows = slot_of.numel()
    out = B.alloc_quantize_outputs(rows, cols, orientation, layout)
    for t in out:
        if t is not None:
            t.fill_(0xA5)
    B.mxfp8_moe_dispatch_quantize(src, slot_of, top_k, None if weights is None else dev(weights), off, orientation, rule, elem, *out, layout)
    assert B.mxfp8_device_status() == 0
    w_off, _, w_slot = orc.moe_sort(ids, experts, rows)
    used = int(w_off[-1])
    y = orc.moe_dispatch(values, w_slot[:used], top_k, weights, dtype if dtype == "bf16" else "f32")
    check_conversion(out, y, rows, used, orientation, rule, elem, layout, what)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("orientation", [1, 2, 3])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("layout", [0, 1])
def test_dispatch_equals_the_oracle(dtype, orientation, weighted, layout):
    tokens, top_k, experts, cols = 300, 3, 7, 352
    rng = np.random.default_rng(11)
    x = synth.gradient_like((tokens, cols), 5)
    w = rng.random((tokens, top_k)).astype(np.float32) if weighted else None
    run_dispatch(x, dtype, routing(tokens, top_k, experts, 1, "holes"), experts, w, orientation, orc.RULE_PAPER, orc.E4M3, layout)


@pytest.mark.parametrize("elem", [orc.E4M3, orc.E5M2, orc.E2M3, orc.E3M2, orc.E2M1])
@pytest.mark.parametrize("rule", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_dispatch_formats_and_rules(elem, rule, dtype):
    x = synth.student_t((70, 160), 6)
    w = np.random.default_rng(2).standard_normal((70, 2)).astype(np.float32)
    run_dispatch(x, dtype, routing(70, 2, 5, 3), 5, w, 3, rule, elem, 1)


@pytest.mark.parametrize("tokens,top_k,experts,cols,kind", [
    (1, 1, 1, 32, "random"), (1, 1, 4, 4096, "random"), (1, 6, 8, 64, "one"), (2, 2, 64, 1408, "random"), (40, 2, 3, 96, "none"),
    (128, 1, 1, 128, "random"), (129, 1, 1, 160, "one"), (1000, 6, 64, 1120, "skewed"), (3001, 2, 8, 2048, "holes")])
def test_dispatch_sizes(tokens, top_k, experts, cols, kind):
    x = synth.gaussian((tokens, cols), 7)
    run_dispatch(x, "bf16", routing(tokens, top_k, experts, 4, kind), experts, None, 3, 0, orc.E4M3, 1, what="%d %s" % (tokens, kind))


def test_dispatch_columns_only_of_a_width_that_has_no_row_blocks():
    run_dispatch(synth.gaussian((90, 48), 1), "bf16", routing(90, 2, 4, 4), 4, None, 2, 0, orc.E4M3, 1)
    run_dispatch(synth.gaussian((90, 16), 1), "fp32", routing(90, 2, 4, 4), 4, None, 2, 0, orc.E5M2, 0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_dispatch_of_special_values(dtype):
    """NaN and Inf in the tokens, weights of zero, Inf and NaN, and a token 0 (what a padding row's load reads) of NaN."""
    x = synth.with_nonfinite(synth.gaussian((200, 256), 8), 9, 0.01)
    x[0] = np.nan
    w = np.random.default_rng(1).standard_normal((200, 2)).astype(np.float32)
    w[3], w[4], w[5] = 0.0, np.inf, np.nan
    w[6] = 3e38
    run_dispatch(x, dtype, routing(200, 2, 6, 5, "holes"), 6, w, 3, 0, orc.E4M3, 1)
    run_dispatch(x, dtype, routing(200, 2, 6, 5, "holes"), 6, None, 3, 0, orc.E4M3, 1)


@pytest.mark.parametrize("elem", [orc.E4M3, orc.E5M2, orc.E2M3, orc.E3M2, orc.E2M1])
@pytest.mark.parametrize("orientation", [1, 2, 3])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_dispatch_of_the_whole_range(elem, orientation, dtype):
    """Blocks of subnormals, of the largest values, of zeros of both signs, single Inf and NaN; products that round, underflow
    and overflow."""
    rng = np.random.default_rng(7)
    tokens, cols = 150, 320
    x = rng.standard_normal((tokens, cols)) * np.exp2(rng.integers(-149, 127, (tokens, 1)).astype(np.float64))
    x[rng.random((tokens, cols)) < 0.05] *= -0.0
    x[10:14], x[20, ::2], x[21] = 0.0, -0.0, np.finfo(np.float32).max
    x[22, 64:96], x[23] = -3.3e38, np.float32(1e-45)
    x[30, 17], x[31, 40], x[31, 300], x[32, 0] = np.nan, np.inf, -np.inf, np.inf
    x = x.astype(np.float32)
    w = (rng.standard_normal((tokens, 2)) * np.exp2(rng.integers(-30, 30, (tokens, 2)))).astype(np.float32)
    w[40], w[41], w[42] = 0.0, -0.0, 2.0 ** -126
    for weights in (None, w):
        with np.errstate(over="ignore", invalid="ignore", under="ignore"):
            run_dispatch(x, dtype, routing(tokens, 2, 5, 6, "holes"), 5, weights, orientation, orientation & 1, elem, 1)


def test_dispatch_equals_two_steps_on_a_batch_that_uses_the_tile_counter():
    """Large enough for several tiles per CTA: the same bytes as gathering first and mxfp8_quantize after it."""
    import torch
    from paper_2506_08027_b200 import binding as B
    tokens, top_k, experts, cols = 8192, 6, 64, 2048
    x = synth.device_tensor("activation", (tokens, cols), 3)
    ids = dev(routing(tokens, top_k, experts, 9, "random"))
    off, row_of, slot_of = gpu_sort(ids.cpu().numpy(), experts)
    rows, used = slot_of.numel(), int(off[-1])
    out = B.alloc_quantize_outputs(rows, cols, B.BOTH, B.SF_SWIZZLED)
    for captured in (False, True):
        for t in out:
            t.zero_()
        call = lambda: B.mxfp8_moe_dispatch_quantize(x, slot_of, top_k, None, off, B.BOTH, B.RULE_PAPER, B.E4M3, *out, B.SF_SWIZZLED)
        if captured:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                call()
            g.replay()
        else:
            call()
        y = x[(slot_of[:used].clamp(min=0) // top_k).long()]
        y = torch.where((slot_of[:used] >= 0).unsqueeze(1), y, torch.zeros_like(y))        # +0, which a product with 0 is not
        want = B.alloc_quantize_outputs(used, cols, B.BOTH, B.SF_SWIZZLED)
        B.mxfp8_quantize(y, B.BOTH, B.RULE_PAPER, B.E4M3, *want, B.SF_SWIZZLED)
        assert B.mxfp8_device_status() == 0
        assert torch.equal(out[0][:used], want[0]) and torch.equal(out[2][:used], want[2])
        assert torch.equal(out[1][:want[1].numel()], want[1])
        per = out[3].view(cols // 128, rows // 128, 512)[:, :used // 128]
        assert torch.equal(per.reshape(-1), want[3])


@pytest.mark.parametrize("dtype,tokens,cols,orientation", [
    ("bf16", 9001, 4128, 3), ("bf16", 9001, 4128, 1), ("fp32", 4500, 4160, 3), ("fp32", 70001, 256, 2), ("bf16", 100001, 384, 3)])
def test_dispatch_of_tokens_that_do_not_stay_in_l2(dtype, tokens, cols, orientation):
    """Sources that are walked in groups of columns (uneven ones, single ones): the same bytes as gathering first."""
    import torch
    from paper_2506_08027_b200 import binding as B
    top_k, experts = 2, 5
    off, _, slot_of = gpu_sort(routing(tokens, top_k, experts, 2, "holes"), experts)
    rows, used = slot_of.numel(), int(off[-1])
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(tokens, cols, generator=g, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    w = torch.randn(tokens, top_k, generator=g, device="cuda")
    slots = slot_of[:used].long()
    for weights in (None, w):
        y = x[slots.clamp(min=0) // top_k]
        if weights is not None:
            y = (y.float() * weights.reshape(-1)[slots.clamp(min=0)].unsqueeze(1)).to(x.dtype)
        y = torch.where((slots >= 0).unsqueeze(1), y, torch.zeros((), dtype=y.dtype, device="cuda"))
        want = B.alloc_quantize_outputs(used, cols, orientation, B.SF_LINEAR)
        B.mxfp8_quantize(y, orientation, B.RULE_PAPER, B.E4M3, *want, B.SF_LINEAR)
        got = B.alloc_quantize_outputs(rows, cols, orientation, B.SF_LINEAR)
        for q in got:
            if q is not None:
                q.fill_(0xA5)
        B.mxfp8_moe_dispatch_quantize(x, slot_of, top_k, weights, off, orientation, B.RULE_PAPER, B.E4M3, *got, B.SF_LINEAR)
        assert B.mxfp8_device_status() == 0
        for q, ref in zip(got, want):
            if q is not None:
                assert torch.equal(q.reshape(-1)[:ref.numel()], ref.reshape(-1)) and (q.reshape(-1)[ref.numel():] == 0xA5).all()


def test_bad_device_arrays_are_reported():
    import torch
    from paper_2506_08027_b200 import binding as B
    x = torch.ones(8, 64, device="cuda")
    off, row_of, slot_of = gpu_sort(routing(8, 2, 4, 1), 4)
    rows = slot_of.numel()
    out = B.alloc_quantize_outputs(rows, 64, B.BOTH, B.SF_SWIZZLED)
    go = lambda s, o: B.mxfp8_moe_dispatch_quantize(x, s, 2, None, o, B.BOTH, 0, 0, *out, B.SF_SWIZZLED)
    for end in (-128, rows + 128, 100):
        bad = off.clone()
        bad[-1] = end
        for t in out:
            t.fill_(0xA5)
        go(slot_of, bad)
        assert B.mxfp8_device_status() == B.ERR_DEVICE_ARGS
        assert all((t == 0xA5).all() for t in out)
    for slot in (16, -2, 2 ** 31 - 1):
        bad = slot_of.clone()
        bad[0] = slot
        go(bad, off)
        assert B.mxfp8_device_status() == B.ERR_DEVICE_ARGS
        assert not out[0][0].any()                         # such a row counts as one without a slot
    go(slot_of, off)
    assert B.mxfp8_device_status() == 0
    y, dst = torch.ones(rows, 64, device="cuda"), torch.empty(8, 64, device="cuda")
    for r in (rows, -2, 2 ** 31 - 1):
        bad = row_of.clone()
        bad[3, 1] = r
        B.mxfp8_moe_combine(y, bad, None, dst)
        assert B.mxfp8_device_status() == B.ERR_DEVICE_ARGS
        assert (dst[3] == 1).all() and (dst[2] == 2).all()
        d_w = torch.full((8, 2), 9.0, device="cuda")
        d_y = torch.zeros_like(y)
        B.mxfp8_moe_combine_grad(x, y, bad, slot_of, None, off, d_y, d_w)
        assert B.mxfp8_device_status() == B.ERR_DEVICE_ARGS
        assert d_w[3, 1] == 0 and (d_w[2] == 64).all()
    bad = off.clone()
    bad[-1] = rows + 1
    B.mxfp8_moe_combine_grad(x, y, row_of, slot_of, None, bad, torch.empty_like(y), None)
    assert B.mxfp8_device_status() == B.ERR_DEVICE_ARGS


def test_gradient_stores_no_row_that_the_offsets_do_not_own():
    import torch
    from paper_2506_08027_b200 import binding as B
    x = torch.ones(8, 64, device="cuda")
    off, row_of, slot_of = gpu_sort(routing(8, 2, 4, 1), 4)
    rows, used = slot_of.numel(), int(off[-1])
    y = torch.ones(rows, 64, device="cuda")
    for end in (-1, rows + 1, -2 ** 31, 2 ** 31 - 1):           # no possible end: no row is in use
        bad = off.clone()
        bad[-1] = end
        d_y, d_w = torch.full_like(y, 7.0), torch.full((8, 2), 7.0, device="cuda")
        B.mxfp8_moe_combine_grad(x, y, row_of, slot_of, None, bad, d_y, d_w)
        assert B.mxfp8_device_status() == B.ERR_DEVICE_ARGS
        assert (d_y == 7).all() and (d_w == 0).all()
    more = torch.cat((slot_of, torch.full((128,), -1, dtype=torch.int32, device="cuda")))
    y = torch.ones(rows + 128, 64, device="cuda")
    bad = row_of.clone()
    bad[5, 0] = used + 3                                        # a row of the tensor, behind the last segment
    d_y, d_w = torch.full_like(y, 7.0), torch.full((8, 2), 7.0, device="cuda")
    B.mxfp8_moe_combine_grad(x, y, bad, more, None, off, d_y, d_w)
    assert B.mxfp8_device_status() == B.ERR_DEVICE_ARGS
    assert (d_y[used:] == 7).all() and d_w[5, 0] == 0 and d_w[5, 1] == 64
    for slot in (16, 2 ** 31 - 1, -5):                          # such an entry counts as -1: the row is cleared
        bad = slot_of.clone()
        bad[127] = slot
        assert slot_of[127] == -1
        d_y = torch.full((rows, 64), 7.0, device="cuda")
        B.mxfp8_moe_combine_grad(x, y[:rows], row_of, bad, None, off, d_y, None)
        assert B.mxfp8_device_status() == B.ERR_DEVICE_ARGS
        assert not d_y[127].any()


HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}          # half a step of the type, relative to the value
COLS = [1, 2, 3, 8, 37, 64, 100, 257, 1408, 2050, 4096]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("src,dst", [("bf16", "bf16"), ("fp32", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("top_k", [1, 2, 6, 9])
def test_combine_against_the_oracle(cols, src, dst, top_k):
    """k fused multiply-adds in FP32: each off by at most half a step of a partial sum, which the magnitudes bound; then
    one rounding to the output type."""
    import torch
    from paper_2506_08027_b200 import binding as B
    tokens, experts = 37, 5
    rng = np.random.default_rng(cols + top_k)
    ids = routing(tokens, top_k, experts, 3, "holes")
    ids[4] = -1                                            # a token without any expert
    off, row_of, slot_of = gpu_sort(ids, experts, spare=3)
    rows = slot_of.numel()
    y, yv = as_dtype(synth.student_t((rows, cols), 4), src)
    w = rng.standard_normal((tokens, top_k)).astype(np.float32)
    for weights in (w, None):
        out = torch.full((tokens, cols), float("nan"), dtype=torch.bfloat16 if dst == "bf16" else torch.float32, device="cuda")
        B.mxfp8_moe_combine(y, row_of, None if weights is None else dev(weights), out)
        want, mag = orc.moe_combine_f64(yv, row_of.cpu().numpy(), weights)
        err = np.abs(out.double().cpu().numpy() - want)
        sums = top_k * 2.0 ** -24 * mag * (1 + 2.0 ** -20)
        assert (err <= sums + HALF[dst] * (np.abs(want) + sums)).all(), (err / (mag + 1e-300)).max()
        assert not out[4].any()
    assert B.mxfp8_device_status() == 0


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dy,src", [("bf16", "bf16"), ("fp32", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("top_k", [1, 6, 9])
def test_combine_gradient_against_the_oracle(cols, dy, src, top_k):
    """d_src: one FP32 product and one rounding to the type: bit for bit.  d_weights: a sum of `cols` products by fused
    multiply-adds and additions, at most cols + 16 roundings on the way of any term."""
    import torch
    from paper_2506_08027_b200 import binding as B
    tokens, experts = 37, 5
    rng = np.random.default_rng(cols + top_k)
    ids = routing(tokens, top_k, experts, 3, "holes")
    off, row_of, slot_of = gpu_sort(ids, experts, spare=130)
    rows, used = slot_of.numel(), int(off[-1])
    y, yv = as_dtype(synth.student_t((rows, cols), 4), src)
    g, gv = as_dtype(synth.output_gradient((tokens, cols), 6), dy)
    w = rng.standard_normal((tokens, top_k)).astype(np.float32)
    d_y = torch.full_like(y, 3.0)
    d_w = torch.full((tokens, top_k), float("nan"), device="cuda")
    B.mxfp8_moe_combine_grad(g, y, row_of, slot_of, dev(w), off, d_y, d_w)
    assert B.mxfp8_device_status() == 0
    want = orc.moe_dispatch(gv, slot_of[:used].cpu().numpy(), top_k, w, "f32")
    want, _ = as_dtype(want, src)                          # FP32 product, then one rounding
    assert torch.equal(d_y[:used], want)
    assert (d_y[used:] == 3.0).all(), "rows behind the last segment were written"
    _, dw64, mag = orc.moe_combine_grad_f64(gv, yv, row_of.cpu().numpy(), w, rows)
    err = np.abs(d_w.double().cpu().numpy() - dw64)
    assert (err <= (cols + 16) * 2.0 ** -24 * mag * (1 + 2.0 ** -10) + 2.0 ** -140).all()
    assert (d_w.cpu().numpy()[row_of.cpu().numpy() < 0] == 0).all()
    # each gradient alone gives the same bits
    a, b = torch.full_like(y, 3.0), torch.empty_like(d_w)
    B.mxfp8_moe_combine_grad(g, y, row_of, slot_of, dev(w), off, a, None)
    B.mxfp8_moe_combine_grad(g, y, row_of, slot_of, dev(w), off, None, b)
    assert torch.equal(a, d_y) and torch.equal(b, d_w)


@pytest.mark.parametrize("src,dst", [("bf16", "bf16"), ("fp32", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("top_k,cols", [(1, 2088), (2, 1027), (6, 520), (3, 2052)])
def test_combine_and_gradient_of_a_batch_that_fills_the_machine(src, dst, top_k, cols):
    """Enough tokens that a lane keeps several vectors of a row in flight (sum) and a warp takes a token alone (gradient);
    the last run of columns ragged.  Bounds as above."""
    import torch
    from paper_2506_08027_b200 import binding as B
    tokens, experts = 5003, 8
    rng = np.random.default_rng(cols)
    off, row_of, slot_of = gpu_sort(routing(tokens, top_k, experts, 3, "holes"), experts)
    rows, used = slot_of.numel(), int(off[-1])
    dt = lambda n: torch.bfloat16 if n == "bf16" else torch.float32
    y = torch.randn(rows, cols, device="cuda").to(dt(src))
    w = torch.randn(tokens, top_k, device="cuda")
    out = torch.full((tokens, cols), float("nan"), dtype=dt(dst), device="cuda")
    B.mxfp8_moe_combine(y, row_of, w, out)
    live = (row_of >= 0).unsqueeze(2)
    want = torch.zeros(tokens, cols, dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(want)
    for j in range(top_k):
        term = torch.where(live[:, j], y.double()[row_of[:, j].long().clamp(min=0)] * w[:, j:j + 1].double(), torch.zeros_like(want))
        want += term
        mag += term.abs()
    sums = top_k * 2.0 ** -24 * mag * (1 + 2.0 ** -20)
    assert ((out.double() - want).abs() <= sums + HALF[dst] * (want.abs() + sums)).all()
    g = torch.randn(tokens, cols, device="cuda").to(dt(dst))
    d_y, d_w = torch.full_like(y, 3.0), torch.full((tokens, top_k), float("nan"), device="cuda")
    B.mxfp8_moe_combine_grad(g, y, row_of, slot_of, w, off, d_y, d_w)
    assert B.mxfp8_device_status() == 0
    slot = slot_of[:used].long().clamp(min=0)
    d_want = torch.where((slot_of[:used] >= 0).unsqueeze(1), g.float()[slot // top_k] * w.reshape(-1)[slot].unsqueeze(1), torch.zeros((), device="cuda"))
    assert torch.equal(d_y[:used], d_want.to(dt(src))) and (d_y[used:] == 3.0).all()
    for j in range(top_k):
        terms = torch.where(live[:, j], y.double()[row_of[:, j].long().clamp(min=0)] * g.double(), torch.zeros_like(want))
        assert ((d_w[:, j].double() - terms.sum(dim=1)).abs() <= (cols + 16) * 2.0 ** -24 * terms.abs().sum(dim=1) * (1 + 2.0 ** -10)).all()


@pytest.mark.parametrize("shift", [1, 2, 4])
def test_combine_of_tensors_that_start_between_16_byte_boundaries(shift):
    import torch
    from paper_2506_08027_b200 import binding as B
    off, row_of, slot_of = gpu_sort(routing(20, 2, 3, 1), 3)
    rows = slot_of.numel()
    base = torch.randn(rows * 64 + 8, device="cuda").to(torch.bfloat16)
    src = base[shift:shift + rows * 64].view(rows, 64)
    out = torch.zeros(20 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    dst = out[shift:shift + 20 * 64].view(20, 64)
    B.mxfp8_moe_combine(src, row_of, None, dst)
    want = src.float()[row_of.long()].sum(dim=1).to(torch.bfloat16)
    assert torch.equal(dst, want) and not out[:shift].any() and not out[shift + 20 * 64:].any()


def test_combine_passes_32_bits():
    """A sorted tensor of more than 2^31 elements: rows behind that offset are found."""
    import torch
    from paper_2506_08027_b200 import binding as B
    rows, cols = 540000, 4096
    y = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([[rows - 1, 0], [rows - 2, 524289]], dtype=torch.int32, device="cuda")
    for i, r in enumerate(at.flatten().tolist()):
        y[r] = float(i + 1)
    dst = torch.empty(2, cols, device="cuda")
    B.mxfp8_moe_combine(y, at, None, dst)
    assert (dst[0] == 3).all() and (dst[1] == 7).all()
    slot_of = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    slot_of[at.flatten().long()] = torch.arange(4, dtype=torch.int32, device="cuda")
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    d_w = torch.empty(2, 2, device="cuda")
    w = torch.tensor([[2.0, 3.0], [4.0, 5.0]], device="cuda")
    B.mxfp8_moe_combine_grad(torch.ones(2, cols, device="cuda"), y, at, slot_of, w, off, y, d_w)      # in place: a row is read before it is written
    assert d_w.tolist() == [[4096.0, 8192.0], [3 * 4096.0, 4 * 4096.0]]
    assert (y[rows - 1] == 2).all() and (y[rows - 2] == 4).all() and (y[524289] == 5).all() and not y[1].any()


def test_two_captured_sorts_with_workspaces_of_their_own_on_two_streams():
    import torch
    from paper_2506_08027_b200 import binding as B
    graphs = []
    for seed in (1, 2):
        ids = routing(9000, 4, 64, seed)
        d_ids = dev(ids)
        rows = B.mxfp8_moe_rows(9000, 4, 64)
        bufs = [torch.zeros(n, dtype=torch.int32, device="cuda") for n in (65, 36000, rows)]
        ws = torch.empty(B.mxfp8_moe_sort_ws_bytes(9000, 4, 64), dtype=torch.uint8, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.mxfp8_moe_sort(d_ids, 64, bufs[0], bufs[1].view(9000, 4), bufs[2], ws)
        graphs.append((g, ids, rows, bufs, ws, d_ids))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, item in zip(streams, graphs):
            with torch.cuda.stream(s):
                item[0].replay()
    torch.cuda.synchronize()
    for _, ids, rows, bufs, _, _ in graphs:
        for got, want in zip(bufs, orc.moe_sort(ids, 64, rows)):
            assert np.array_equal(got.cpu().numpy(), want.reshape(-1))


@pytest.mark.parametrize("tokens", [300, 2100])            # sorted by one launch and by two
def test_a_captured_chain_replayed_on_other_routings(tokens):
    """Sort, gathered conversions, weighted sum and its gradient in one graph, captured on a side stream; every replay reads
    what its inputs hold then, and two graphs with buffers of their own run side by side."""
    import torch
    from paper_2506_08027_b200 import binding as B
    top_k, experts, cols = 3, 10, 224
    rows = B.mxfp8_moe_rows(tokens, top_k, experts)

    def buffers():
        i32 = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")
        f = lambda *n, t=torch.float32: torch.zeros(n, dtype=t, device="cuda")
        return dict(ids=i32(tokens, top_k), x=f(tokens, cols, t=torch.bfloat16), w=f(tokens, top_k), dy=f(tokens, cols), h=f(rows, cols, t=torch.bfloat16),
                    off=i32(experts + 1), row_of=i32(tokens, top_k), slot_of=i32(rows), y=f(tokens, cols),
                    d_h=f(rows, cols, t=torch.bfloat16), d_w=f(tokens, top_k),
                    ws=torch.zeros(max(B.mxfp8_moe_sort_ws_bytes(tokens, top_k, experts), 16), dtype=torch.uint8, device="cuda"),
                    fwd=[t.zero_() if t is not None else None for t in B.alloc_quantize_outputs(rows, cols, B.BOTH, B.SF_SWIZZLED)],
                    bwd=[t.zero_() if t is not None else None for t in B.alloc_quantize_outputs(rows, cols, B.ROW, B.SF_SWIZZLED)])

    def chain(b):
        B.mxfp8_moe_sort(b["ids"], experts, b["off"], b["row_of"], b["slot_of"], b["ws"])
        B.mxfp8_moe_dispatch_quantize(b["x"], b["slot_of"], top_k, None, b["off"], B.BOTH, B.RULE_PAPER, B.E4M3, *b["fwd"], B.SF_SWIZZLED)
        B.mxfp8_moe_combine(b["h"], b["row_of"], b["w"], b["y"])
        B.mxfp8_moe_combine_grad(b["dy"], b["h"], b["row_of"], b["slot_of"], b["w"], b["off"], b["d_h"], b["d_w"])
        B.mxfp8_moe_dispatch_quantize(b["dy"], b["slot_of"], top_k, b["w"], b["off"], B.ROW, B.RULE_OCP, B.E5M2, *b["bwd"], B.SF_SWIZZLED)

    def fill(b, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        b["ids"].copy_(dev(routing(tokens, top_k, experts, seed, "holes")))
        for name in ("x", "w", "dy", "h"):
            b[name].copy_(torch.randn(b[name].shape, generator=g, device="cuda"))

    def outputs(b):
        used = int(b["off"][-1])
        tensors = [b["off"], b["row_of"], b["slot_of"], b["y"], b["d_h"][:used], b["d_w"], b["fwd"][0][:used], b["fwd"][2][:used], b["bwd"][0][:used]]
        scales = [b[n][1].view(-1, cols // 32 + (-(cols // 32)) % 4, 128)[:used // 128] for n in ("fwd", "bwd")]
        return [t.clone() for t in tensors + scales]

    plain, graphs, streams = buffers(), [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        b = buffers()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            chain(b)                                       # outside the capture first
            s.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                chain(b)
        graphs.append((g, b))
    for seed in range(4):
        for i, (_, b) in enumerate(graphs):
            fill(b, 10 * seed + i)
        torch.cuda.synchronize()
        for s, (g, _) in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for i, (_, b) in enumerate(graphs):
            fill(plain, 10 * seed + i)
            chain(plain)
            for got, want in zip(outputs(b), outputs(plain)):
                assert torch.equal(got, want)
    assert B.mxfp8_device_status() == 0


@pytest.mark.parametrize("backward", [False, True])
def test_a_layer_of_experts_end_to_end(backward):
    """Sort, dispatch, the grouped products and the way back, as a layer uses them, against the same layer in 64 bits on the
    values that the conversions give (two grouped products with FP32 outputs, weighted sum, gradients)."""
    import torch
    from paper_2506_08027_b200 import binding as B
    tokens, top_k, experts, hidden, ffn = 520, 2, 4, 256, 384
    rng = np.random.default_rng(5)
    ids = routing(tokens, top_k, experts, 2, "holes")
    w = rng.random((tokens, top_k)).astype(np.float32)
    x, xv = as_dtype(synth.gaussian((tokens, hidden), 1), "bf16")
    wt, _ = as_dtype(0.05 * synth.gaussian((experts * ffn, hidden), 2), "bf16")
    off, row_of, slot_of = gpu_sort(ids, experts)
    rows = slot_of.numel()
    E = B.E4M3
    qx = B.alloc_quantize_outputs(rows, hidden, B.BOTH, B.SF_SWIZZLED)
    for t in qx:
        t.zero_()
    B.mxfp8_moe_dispatch_quantize(x, slot_of, top_k, None, off, B.BOTH, B.RULE_PAPER, E, *qx, B.SF_SWIZZLED)
    qw = B.alloc_quantize_outputs(experts * ffn, hidden, B.BOTH, B.SF_SWIZZLED)
    B.mxfp8_quantize(wt, B.BOTH, B.RULE_PAPER, E, *qw, B.SF_SWIZZLED)
    y = torch.zeros(rows, ffn, device="cuda")
    B.mxfp8_grouped_gemm(qx[0], qx[1], qw[0], qw[1], off, B.GROUP_M, rows, ffn, hidden, B.K_MAJOR, E, E, y)
    out = torch.empty(tokens, ffn, device="cuda")
    B.mxfp8_moe_combine(y, row_of, dev(w), out)
    # the same in 64 bits from the decoded operands
    offs, rof, sof = orc.moe_sort(ids, experts, rows)
    used = int(offs[-1])
    sorted_x = orc.moe_dispatch(xv, sof[:used], top_k, None, "bf16")
    dx_row = orc.dequantize_f64(*orc.quantize(sorted_x, orc.ROW), orc.ROW)
    w_np = wt.float().cpu().numpy()
    dw_row = orc.dequantize_f64(*orc.quantize(w_np, orc.ROW), orc.ROW)
    y64 = np.zeros((rows, ffn))
    for e in range(experts):
        y64[offs[e]:offs[e + 1]] = dx_row[offs[e]:offs[e + 1]] @ dw_row[e * ffn:(e + 1) * ffn].T
    out64, _ = orc.moe_combine_f64(y64, rof, w)
    assert np.linalg.norm(out.double().cpu().numpy() - out64) <= 2e-5 * np.linalg.norm(out64)     # the product's bound, 1e-5, and the sum
    if not backward:
        return
    g, gv = as_dtype(synth.gaussian((tokens, ffn), 3), "bf16")
    d_w = torch.empty(tokens, top_k, device="cuda")
    B.mxfp8_moe_combine_grad(g, y, row_of, slot_of, dev(w), off, None, d_w)
    qg = B.alloc_quantize_outputs(rows, ffn, B.BOTH, B.SF_SWIZZLED)
    for t in qg:
        t.zero_()
    B.mxfp8_moe_dispatch_quantize(g, slot_of, top_k, dev(w), off, B.BOTH, B.RULE_PAPER, E, *qg, B.SF_SWIZZLED)
    d_sorted = torch.zeros(rows, hidden, device="cuda")
    B.mxfp8_grouped_gemm(qg[0], qg[1], qw[2], qw[3], off, B.GROUP_M, rows, hidden, ffn, B.MN_MAJOR, E, E, d_sorted)
    d_x = torch.empty(tokens, hidden, device="cuda")
    B.mxfp8_moe_combine(d_sorted, row_of, None, d_x)
    d_wt = torch.empty(experts * ffn, hidden, device="cuda")
    B.mxfp8_grouped_gemm(qg[2], qg[3], qx[2], qx[3], off, B.GROUP_K, ffn, hidden, rows, B.MN_MAJOR, E, E, d_wt)
    assert B.mxfp8_device_status() == 0
    sorted_g = orc.moe_dispatch(gv, sof[:used], top_k, w, "bf16")
    g_row = orc.dequantize_f64(*orc.quantize(sorted_g, orc.ROW), orc.ROW)
    g_col = orc.dequantize_f64(*orc.quantize(sorted_g, orc.COL), orc.COL)
    x_col = orc.dequantize_f64(*orc.quantize(sorted_x, orc.COL), orc.COL)
    w_col = orc.dequantize_f64(*orc.quantize(w_np, orc.COL), orc.COL)
    ds64, dwt64 = np.zeros((rows, hidden)), np.zeros((experts * ffn, hidden))
    for e in range(experts):
        seg = slice(offs[e], offs[e + 1])
        ds64[seg] = g_row[seg] @ w_col[e * ffn:(e + 1) * ffn]
        dwt64[e * ffn:(e + 1) * ffn] = g_col[seg].T @ x_col[seg]
    dx64, _ = orc.moe_combine_f64(ds64, rof)
    _, dw64, _ = orc.moe_combine_grad_f64(gv, y64, rof, w, rows)
    near = lambda got, want: np.linalg.norm(got.double().cpu().numpy() - want) <= 2e-5 * np.linalg.norm(want)
    assert near(d_x, dx64) and near(d_wt, dwt64) and near(d_w, dw64)
