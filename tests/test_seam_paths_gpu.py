"""Every kernel that a seam's shapes, types and alignment pick, with several rows for each CTA (or warp): rings of rows that wrap around, rows of the gate that
change in the middle of a CTA's share, calls in place while other rows are on their way.  Checks and tolerances are those of test_seam_gpu.py, whose
shapes give most CTAs one row: a column's sum passes at most 22 rows of one CTA, 80 parts of a warp of the joining launch and 16 warps on the way, below
the 128 + 64 additions that are counted there."""
import pytest
import torch

from paper_2506_08027_b200 import binding as B
from test_seam_gpu import TYPES, inputs
from test_seam_gpu import test_backward as check_backward
from test_seam_gpu import test_forward as check_forward

pytestmark = pytest.mark.gpu

BB, BF, FB, FF = ("bf16", "bf16", "bf16"), ("bf16", "fp32", "fp32"), ("fp32", "bf16", "fp32"), ("fp32", "fp32", "bf16")
# rows, columns, types, norm after the block, rows per gate (0: none), behind a 16-byte boundary by one element.  Rows of a CTA or warp: for 148 multiprocessors.
CASES = [
    # rows on 16-byte boundaries: a warp per row forward (5, 4 and 5 rows of a warp or more)
    (25001, 200, BB, True, 0, False), (25001, 200, BF, True, 613, False), (20011, 504, FF, False, 7, False), (12001, 1000, BB, True, 613, False),
    (12001, 1000, FB, True, 5, False), (9001, 1000, FF, True, 0, False),
    # a CTA per row; backward one vector per thread (11 rows of a CTA, 14 of the wider ones)
    *((3001, 2048, t, p, g, False) for t in (BB, BF, FB, FF) for p, g in ((True, 5), (False, 0))),
    (3001, 2048, BB, True, 0, False), (3001, 2048, BF, True, 613, False), (3001, 2048, BB, False, 613, False),
    (2003, 4096, BB, True, 0, False), (2003, 4096, BF, True, 613, False), (2003, 4096, FF, False, 5, False),
    # backward two vectors per thread
    (1201, 4104, BB, True, 5, False), (1201, 5120, BF, True, 0, False), (1201, 5120, FB, False, 100, False),
    *((1103, 8192, t, p, g, False) for t in (BB, BF, FB, FF) for p, g in ((True, 0), (True, 5))),
    # eight vectors per thread forward, four backward; FP32 rows that do not fit shared memory with it
    (701, 8200, BB, True, 5, False), (701, 8200, FF, True, 0, False), (701, 16384, BB, True, 0, False), (601, 16384, BF, False, 5, False), (601, 16384, FF, True, 100, False),
    # other rows: one element at a time, two where rows have an even number of them
    (9001, 201, BB, True, 5, False), (9001, 202, BF, True, 613, False), (9001, 200, FF, True, 0, True),
    (7001, 777, FB, True, 5, True), (7001, 778, BB, False, 0, False), (5003, 1409, BF, False, 613, False), (5003, 1410, BB, True, 5, False),
    (3001, 2049, BB, True, 5, False), (3001, 2050, BF, True, 0, False), (2003, 4095, FF, False, 5, False), (2003, 4094, BB, True, 613, False), (1501, 4096, BB, True, 5, True),
    (1009, 6003, BB, True, 5, False), (1009, 6002, BF, True, 100, False), (1009, 8190, FF, False, 0, False),
    # above 8192 columns: 1024 threads forward, column sums in shared memory backward
    (601, 8193, BB, True, 5, False), (601, 8194, BF, True, 0, False), (601, 16383, FF, True, 100, False), (601, 16382, FB, False, 5, False), (601, 16384, BB, True, 5, True),
]


@pytest.mark.parametrize("rows,cols,types,post,per_gate,odd", CASES)
def test_forward(rows, cols, types, post, per_gate, odd):
    check_forward((rows, cols), types, post, per_gate, odd)


@pytest.mark.parametrize("rows,cols,types,post,per_gate,odd", CASES)
def test_backward(rows, cols, types, post, per_gate, odd):
    check_backward((rows, cols), types, post, per_gate, odd)


# one, two and four vectors per thread; one and two elements per access; rows in shared memory
@pytest.mark.parametrize("cols", [512, 5120, 8200, 333, 1410, 8201])
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("post,per_gate", [(True, 0), (True, 40), (False, 40), (False, 0)])
def test_without_one_of_the_incoming_gradients(cols, types, post, per_gate):
    """No dx, or no dh, is the same as one of zeros."""
    rows = 300
    d = inputs(rows, cols, types, post, per_gate, seed=2)
    seam = B.make_seam(d["gamma_pre"], d["gamma_post"], d["gate"], max(1, per_gate), 0.75, 0.5)
    rp = d["y"].float().square().mean(dim=1).rsqrt() if post else None
    rn = d["h_in"].float().square().mean(dim=1).rsqrt()
    ws = torch.empty(B.mxfp8_residual_rmsnorm_grad_ws_bytes(seam, rows, cols), dtype=torch.uint8, device="cuda")

    def call(dx, dh):
        out = [torch.full_like(d["y"], 7.0), torch.full_like(d["h_in"], 7.0)] + [None if d[k] is None else torch.full(d[k].shape, 7.0, device="cuda")
                                                                                   for k in ("gamma_pre", "gamma_post", "gate")]
        B.mxfp8_residual_rmsnorm_grad(seam, dx, dh, d["y"], d["h_in"], rp, rn, *out, ws)
        torch.cuda.synchronize()
        return [t for t in out if t is not None]
    none = lambda k: torch.zeros_like(d[k])
    for dx, dh, zdx, zdh in ((None, d["dh"], none("dx"), d["dh"]), (d["dx"], None, d["dx"], none("dh")), (None, None, none("dx"), none("dh"))):
        assert all(torch.equal(a, b) for a, b in zip(call(dx, dh), call(zdx, zdh)))


def converted(rows, cols, types, post, per_gate, orientation, layout, elem, rule, change=None, shift_y=0, in_place=False):
    """The converted seam against the stored one and a separate conversion of x = (h rstd) gamma, rounded to the stream's type: the same bits."""
    d = inputs(rows, cols, types, post, per_gate, seed=4)
    if change is not None:
        change(d)
    if shift_y:
        buf = torch.zeros(d["y"].numel() + 16, dtype=d["y"].dtype, device="cuda")
        moved = buf[shift_y:shift_y + d["y"].numel()].view(rows, cols)
        moved.copy_(d["y"])
        d["y"] = moved
    seam = B.make_seam(d["gamma_pre"], d["gamma_post"], d["gate"], max(1, per_gate), 0.75, 0.5, 1e-6)
    h, ref = d["h_in"].clone() if in_place else torch.empty_like(d["h_in"]), torch.empty_like(d["h_in"])
    stats = [torch.full((rows,), 7.0, device="cuda") for _ in range(4)]
    outs, want = ([None if o is None else o.fill_(0xA5) for o in B.alloc_quantize_outputs(rows, cols, orientation, layout)] for _ in range(2))
    B.mxfp8_residual_rmsnorm(seam, d["y"], d["h_in"], ref, None, stats[0] if post else None, stats[1])
    B.mxfp8_residual_rmsnorm_quantize(seam, d["y"], h if in_place else d["h_in"], h, stats[2] if post else None, stats[3], orientation, rule, elem, *outs, layout)
    assert torch.equal(h, ref) and torch.equal(stats[0], stats[2]) and torch.equal(stats[1], stats[3])
    x = ((h.float() * stats[3].unsqueeze(1)) * d["gamma_pre"].float()).to(h.dtype)
    B.mxfp8_quantize(x, orientation, rule, elem, *want, layout)
    for got, w in zip(outs, want):
        assert (got is None) == (w is None) and (got is None or torch.equal(got, w))


MANY = [(20001, 256), (12001, 992), (3001, 2048), (2003, 4096), (1201, 5120), (701, 8192), (601, 16384)]


@pytest.mark.parametrize("rows,cols", MANY)
@pytest.mark.parametrize("types", [BB, ("fp32", "bf16", "bf16"), BF, ("fp32", "fp32", "fp32")])
@pytest.mark.parametrize("post,per_gate", [(True, 0), (True, 613), (False, 5)])
def test_rows_converted_where_x_is_computed(rows, cols, types, post, per_gate):
    converted(rows, cols, types, post, per_gate, B.ROW, B.SF_SWIZZLED, B.E4M3, B.RULE_PAPER, in_place=post)


@pytest.mark.parametrize("rows,cols", [(2016, 4096), (992, 8192), (4000, 416)])
@pytest.mark.parametrize("orientation", [B.COL, B.BOTH])
@pytest.mark.parametrize("types,post,per_gate", [(("fp32", "bf16", "bf16"), False, 5), (BF, True, 613)])
def test_columns_converted_behind_it(rows, cols, orientation, types, post, per_gate):
    converted(rows, cols, types, post, per_gate, orientation, B.SF_SWIZZLED, B.E4M3, B.RULE_PAPER)
    converted(rows, cols, types, post, per_gate, orientation, B.SF_LINEAR, B.E5M2, B.RULE_OCP)


@pytest.mark.parametrize("types", [BB, BF])
def test_rows_converted_where_the_block_output_has_another_alignment(types):
    converted(130, 512, types, True, 0, B.ROW, B.SF_SWIZZLED, B.E4M3, B.RULE_PAPER, shift_y=1)
    converted(130, 512, types, True, 9, B.ROW, B.SF_LINEAR, B.E5M2, B.RULE_PAPER, shift_y=2)


@pytest.mark.parametrize("elem", [B.E4M3, B.E5M2])
@pytest.mark.parametrize("rule", [B.RULE_PAPER, B.RULE_OCP])
@pytest.mark.parametrize("types", [BB, BF])
def test_rows_converted_over_the_whole_range_of_values(elem, rule, types):
    """Weights from FP32's smallest numbers to its largest, a block of each: scales from the lowest byte on, subnormal elements, zeros."""
    def change(d):
        power = torch.arange(-149, 128, device="cuda").repeat_interleave(8)[:2208].double()
        d["gamma_pre"].copy_((2.0 ** power * (1 + torch.arange(2208, device="cuda") % 7 / 8.0)).float())
        d["gamma_pre"][64:96] = 0.0
    converted(67, 2208, types, True, 0, B.ROW, B.SF_SWIZZLED, elem, rule, change)
    converted(160, 2208, types, True, 0, B.BOTH, B.SF_SWIZZLED, elem, rule, change)
