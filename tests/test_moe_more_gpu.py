"""The token-movement calls where tests/test_moe_gpu.py does not go: arrays left out, and batches of more than a million slots."""
import numpy as np
import pytest

import oracle as orc
from test_moe_gpu import gpu_sort, routing

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dy,src", [("bf16", "bf16"), ("fp32", "bf16"), ("bf16", "fp32")])
def test_either_gradient_alone_through_the_binding(dy, src):
    """The arrays that only the other gradient reads are None; the same bits as with all of them."""
    import torch
    from paper_2506_08027_b200 import binding as B
    kinds = {"bf16": torch.bfloat16, "fp32": torch.float32}
    tokens, top_k, experts, cols = 150, 3, 5, 264
    off, row_of, slot_of = gpu_sort(routing(tokens, top_k, experts, 3, "holes"), experts, spare=128)
    rows = slot_of.numel()
    g = torch.Generator(device="cuda").manual_seed(1)
    y = torch.randn(rows, cols, generator=g, device="cuda").to(kinds[src])
    d = torch.randn(tokens, cols, generator=g, device="cuda").to(kinds[dy])
    w = torch.randn(tokens, top_k, generator=g, device="cuda")
    both = torch.full_like(y, 3.0), torch.full((tokens, top_k), 3.0, device="cuda")
    B.mxfp8_moe_combine_grad(d, y, row_of, slot_of, w, off, *both)
    rows_only, weights_only = torch.full_like(y, 3.0), torch.full((tokens, top_k), 3.0, device="cuda")
    B.mxfp8_moe_combine_grad(d, None, row_of, slot_of, w, off, rows_only, None)
    B.mxfp8_moe_combine_grad(d, y, row_of, None, w, None, None, weights_only)
    assert B.mxfp8_device_status() == 0
    assert torch.equal(rows_only, both[0]) and torch.equal(weights_only, both[1])
    for missing in ((None, off), (slot_of, None)):
        with pytest.raises(B.Mxfp8Error) as e:
            B.mxfp8_moe_combine_grad(d, None, row_of, missing[0], w, missing[1], rows_only, None)
        assert e.value.status == B.ERR_NULL
    with pytest.raises(B.Mxfp8Error) as e:
        B.mxfp8_moe_combine_grad(d, None, row_of, slot_of, w, off, rows_only, weights_only)
    assert e.value.status == B.ERR_NULL


@pytest.mark.parametrize("cols", [32, 96, 128, 160, 320, 352])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("orientation", [1, 2, 3])
@pytest.mark.parametrize("layout", [0, 1])
def test_dispatch_writes_whole_scale_buffers_as_the_conversion_does(cols, dtype, orientation, layout):
    """A sorted tensor of exactly the rows in use, widths that end inside a tile and inside an atom of the swizzled layout: every
    byte of codes and scales, the layout's padding bytes among them, as mxfp8_quantize of the gathered rows writes it."""
    import torch
    from paper_2506_08027_b200 import binding as B
    tokens, top_k, experts = 170, 2, 3
    off, _, slot_of = gpu_sort(routing(tokens, top_k, experts, 8, "holes"), experts)
    used = int(off[-1])
    slot_of = slot_of[:used].contiguous()
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn(tokens, cols, generator=g, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    y = torch.where((slot_of >= 0).unsqueeze(1), x[slot_of.clamp(min=0).long() // top_k], torch.zeros((), dtype=x.dtype, device="cuda"))
    want, got = (B.alloc_quantize_outputs(used, cols, orientation, layout) for _ in range(2))
    for t in want + got:
        if t is not None:
            t.fill_(0xA5)
    B.mxfp8_quantize(y, orientation, B.RULE_PAPER, B.E4M3, *want, layout)
    B.mxfp8_moe_dispatch_quantize(x, slot_of, top_k, None, off, orientation, B.RULE_PAPER, B.E4M3, *got, layout)
    assert B.mxfp8_device_status() == 0
    for a, b in zip(got, want):
        assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.parametrize("tokens,top_k,experts", [(162501, 8, 256), (312503, 8, 64)])
@pytest.mark.parametrize("kind", ["holes", "skewed", "one"])
def test_sort_of_runs_longer_than_a_warp_keeps(tokens, top_k, experts, kind):
    """From 1212417 slots on a warp's run has more than the 256 slots that stay in its registers: 288 slots, fetched twice
    for the counts and again for the ranks, and 544 slots, fetched three times; the last chunk ragged."""
    from paper_2506_08027_b200 import binding as B
    ids = routing(tokens, top_k, experts, tokens, kind)
    off, row_of, slot_of = gpu_sort(ids, experts, spare=5)
    w_off, w_row, w_slot = orc.moe_sort(ids, experts, slot_of.numel())
    assert np.array_equal(off.cpu().numpy(), w_off)
    assert np.array_equal(row_of.cpu().numpy(), w_row)
    assert np.array_equal(slot_of.cpu().numpy(), w_slot)
    assert B.mxfp8_device_status() == 0


@pytest.mark.parametrize("tokens", [2500, 5600])              # codes of both copies: 57 and 129 MiB
@pytest.mark.parametrize("elem", [orc.E4M3, orc.E5M2, orc.E2M3, orc.E3M2, orc.E2M1])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("weighted", [False, True])
def test_dispatch_on_either_side_of_the_size_at_which_codes_leave_l2_first(tokens, elem, dtype, weighted):
    """The same bytes as gathering, weighting and mxfp8_quantize one after the other."""
    import torch
    from paper_2506_08027_b200 import binding as B
    top_k, experts, cols = 6, 16, 2016
    off, _, slot_of = gpu_sort(routing(tokens, top_k, experts, 8, "holes"), experts)
    used = int(off[-1])
    slot_of = slot_of[:used].contiguous()
    g = torch.Generator(device="cuda").manual_seed(elem)
    x = torch.randn(tokens, cols, generator=g, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    w = torch.randn(tokens, top_k, generator=g, device="cuda") if weighted else None
    slot = slot_of.clamp(min=0).long()
    y = x[slot // top_k]
    if weighted:
        y = (y.float() * w.reshape(-1)[slot].unsqueeze(1)).to(x.dtype)
    y = torch.where((slot_of >= 0).unsqueeze(1), y, torch.zeros((), dtype=x.dtype, device="cuda"))
    want, got = (B.alloc_quantize_outputs(used, cols, B.BOTH, B.SF_SWIZZLED) for _ in range(2))
    B.mxfp8_quantize(y, B.BOTH, B.RULE_OCP, elem, *want, B.SF_SWIZZLED)
    B.mxfp8_moe_dispatch_quantize(x, slot_of, top_k, w, off, B.BOTH, B.RULE_OCP, elem, *got, B.SF_SWIZZLED)
    assert B.mxfp8_device_status() == 0
    for a, b in zip(got, want):
        assert torch.equal(a, b)
