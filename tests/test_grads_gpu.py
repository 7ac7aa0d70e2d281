"""The norm of a set of gradients and clipping by it, against the formulas in 64 bits.

S is a sum of FP32 sums of at most eight squares (eight roundings of 2^-24 each, all terms positive), added in FP64: relative error
below 9 * 2^-24, so the norm's is below 5 * 2^-24 and one rounding; the factor has two FP32 roundings more, a scaled value one product and
the rounding to its type."""
import pytest
import torch

from paper_2506_08027_b200 import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def half_step(t):
    return torch.finfo(t).eps / 2


def gradients(sizes, seed=0, scale=1e-3, pad=3):
    """FP32 and BF16 tensors in turn, `pad` elements apart inside two flat buffers."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = [torch.full((sum(sizes) + pad * len(sizes) + 8,), 5.0, dtype=t, device="cuda") for t in (torch.float32, torch.bfloat16)]
    at, out = [1, 1], []
    for i, n in enumerate(sizes):
        k = i % 2
        v = flat[k][at[k]:at[k] + n]
        v.copy_(scale * torch.randn(n, generator=g, device="cuda"))
        out.append(v)
        at[k] += n + pad
    return out, flat


def norm_of(grads):
    return float(torch.stack([t.double().square().sum() for t in grads]).sum().sqrt()) if grads else 0.0


def clip(grads, results, max_norm):
    items = B.make_grad_items(grads, results)
    ws = torch.full((B.mxfp8_grad_ws_bytes(items) + 8,), 0xA5, dtype=torch.uint8, device="cuda")
    norm = torch.full((4,), 9.0, device="cuda")
    B.mxfp8_grad_clip(items, max_norm, norm[1:3], ws[:-8])
    torch.cuda.synchronize()
    assert float(norm[0]) == 9.0 and float(norm[3]) == 9.0 and bool((ws[-8:] == 0xA5).all())
    return float(norm[1]), float(norm[2])


SIZES = [[1], [0, 5, 0], [7, 8, 9, 15, 16, 17, 31], [16384, 16385, 16383, 3, 65536 + 5], [1000003, 1], [3] * 97, [257] * 1025, [100 + 7 * i for i in range(300)],
         [20000] * 2100]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%dx%d" % (len(s), max(s)))
@pytest.mark.parametrize("where", ["new", "other alignment", "in place"])
def test_clip(sizes, where):
    grads, flat = gradients(sizes)
    want = norm_of(grads)
    before = [f.clone() for f in flat]
    results = None
    if where != "in place":
        out = [torch.full((f.numel() + 1,), 5.0, dtype=f.dtype, device="cuda")[(where == "other alignment"):][:f.numel()] for f in flat]
        results = [out[i % 2][g.storage_offset():g.storage_offset() + g.numel()] for i, g in enumerate(grads)]
    source = [g.clone() for g in grads]
    max_norm = 0.3 * want + 1e-9
    norm, factor = clip(grads, results, max_norm)
    assert abs(norm - want) <= 6 * U * want
    f64 = min(1.0, max_norm / (want + 1e-6))
    assert abs(factor - f64) <= 12 * U * f64
    for i, (g, r, s) in enumerate(zip(grads, results or grads, source)):
        exact = s.double() * factor
        assert bool(((r.double() - exact).abs() <= (half_step(r.dtype) + U) * exact.abs()).all())
        if results:
            assert torch.equal(g, s)
    # nothing between the tensors is written
    for f, b in zip(flat if not results else out, before):
        assert int((f == 5.0).sum()) >= b.numel() - sum(g.numel() for g in grads if g.dtype == f.dtype)


def test_within_the_norm_nothing_changes():
    grads, flat = gradients([1000, 999, 40000])
    before = [f.clone() for f in flat]
    norm, factor = clip(grads, None, 1e3)
    assert factor == 1.0 and all(torch.equal(a, b) for a, b in zip(flat, before))
    results = [torch.zeros_like(g) for g in grads]
    assert clip(grads, results, float("inf"))[1] == 1.0 and all(torch.equal(a, b) for a, b in zip(grads, results))
    assert clip([], None, 1.0) == (0.0, 1.0)
    zeros = [torch.zeros(100, device="cuda")]
    assert clip(zeros, None, 1.0) == (0.0, 1.0)
    ones = [torch.ones(16, device="cuda")]
    assert clip(ones, None, 0.0) == (4.0, 0.0) and bool((ones[0] == 0).all())


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_norm_that_is_not_finite_leaves_the_values(value, dtype):
    g = torch.ones(5000, dtype=dtype, device="cuda")
    g[4999] = value
    out, before = torch.zeros_like(g), g.clone()
    norm, factor = clip([g], [out], 1.0)
    assert factor == 1.0 and (norm != norm if value != value else norm == float("inf"))
    assert torch.equal(torch.nan_to_num(out, nan=3.0), torch.nan_to_num(before, nan=3.0))


@pytest.mark.parametrize("scale", [1e-30, 1e-20, 1e-12, 1e12, 1e17])
@pytest.mark.parametrize("n", [5, 4099])
def test_the_whole_range_of_values(scale, n):
    """Squares that FP32 does not hold are added in FP64."""
    grads, _ = gradients([n, n + 1, n], scale=scale)
    grads[0][2] = 0.0
    grads[0][3] = scale * 1e-9                                # beside much larger ones
    want = norm_of(grads)
    norm, _ = clip(grads, None, 1.0)
    assert abs(norm - want) <= 6 * U * want


def test_sum_of_squares_and_scale_apart():
    """As ranks use them: partial sums added, every part scaled by the whole norm; many items share one call."""
    grads, _ = gradients([501, 77, 3000, 16400, 2], seed=3)
    parts = [B.make_grad_items(grads[:2]), B.make_grad_items(grads[2:])]
    source = [g.clone() for g in grads]
    want = norm_of(grads)
    sums = torch.zeros(2, dtype=torch.float64, device="cuda")
    for k, items in enumerate(parts):
        B.mxfp8_grad_sumsq(items, sums[k:k + 1], torch.empty(B.mxfp8_grad_ws_bytes(items), dtype=torch.uint8, device="cuda"))
    whole = sums.sum().reshape(1)
    norms = torch.zeros(2, 2, device="cuda")
    for k, items in enumerate(parts):
        B.mxfp8_grad_scale(items, whole, 0.5 * want, norms[k])
    torch.cuda.synchronize()
    assert torch.equal(norms[0], norms[1]) and abs(float(norms[0, 0]) - want) <= 6 * U * want
    for g, s in zip(grads, source):
        exact = s.double() * float(norms[0, 1])
        assert bool(((g.double() - exact).abs() <= (half_step(g.dtype) + U) * exact.abs()).all())


def test_graphs_and_streams():
    grads, _ = gradients([100000, 3001, 70000], seed=5)
    results = [torch.zeros_like(g) for g in grads]
    items = B.make_grad_items(grads, results)
    ws = [torch.empty(B.mxfp8_grad_ws_bytes(items), dtype=torch.uint8, device="cuda") for _ in range(2)]
    norm = torch.zeros(2, 2, device="cuda")
    graph = torch.cuda.CUDAGraph()
    B.mxfp8_grad_clip(items, 0.1, norm[0], ws[0])
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.mxfp8_grad_clip(items, 0.1, norm[0], ws[0])
    for g in grads:
        g.mul_(3.0)
    other = B.make_grad_items(grads, [torch.zeros_like(g) for g in grads])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph.replay()
    B.mxfp8_grad_clip(other, 0.1, norm[1], ws[1], stream=side)
    torch.cuda.synchronize()
    want = norm_of(grads)
    assert torch.equal(norm[0], norm[1]) and abs(float(norm[0, 0]) - want) <= 6 * U * want
    assert all(torch.equal(a, b) for a, b in zip(results, other.keep[1]))


def test_offsets_beyond_32_bits():
    n = (1 << 31) + 12345
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[n - 1], g[n // 2] = 1.0, 2.0, 2.0
    norm, factor = clip([g], None, 1.5)
    assert norm == 3.0 and abs(factor - 0.5) <= 1e-6
    assert float(g[0]) == 0.5 and float(g[n - 1]) == 1.0 and float(g[n // 2]) == 1.0 and int((g != 0).sum()) == 3


def test_overlapping_gradients_are_refused():
    flat = torch.zeros(100, device="cuda")
    a, b, c = flat[:40], flat[40:80], flat[39:60]
    out = torch.zeros(100, device="cuda")
    B.make_grad_items([a, b])
    B.make_grad_items([a, b], [out[:40], out[40:80]])
    B.make_grad_items([a, c], [out[:40], out[40:61]])                  # read twice, written apart
    for grads, results in (([a, a], None), ([a, c], None), ([a, b], [out[:40], out[:40]]), ([a, b], [b, out[:40]]), ([a, b], [out[:40], out[39:79]])):
        with pytest.raises(ValueError):
            B.make_grad_items(grads, results)
