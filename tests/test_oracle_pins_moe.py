"""The oracle's mixture-of-experts definitions against hand-worked cases, identities and central differences, and the
refusals of the entry points (no GPU)."""
import ctypes

import numpy as np
import pytest

import oracle as orc
from paper_2506_08027_b200 import binding as B


def test_sort_hand_worked():
    ids = np.array([[2, 0], [0, 2], [-1, 2], [7, 0]], np.int32)
    off, row_of, slot_of = orc.moe_sort(ids, 3, 512)
    assert off.tolist() == [0, 128, 128, 256]
    assert row_of.tolist() == [[128, 0], [1, 129], [-1, 130], [-1, 2]]
    assert slot_of[:4].tolist() == [1, 2, 7, -1] and slot_of[128:132].tolist() == [0, 3, 5, -1] and (slot_of[256:] == -1).all()


@pytest.mark.parametrize("tokens,top_k,experts", [(1, 1, 1), (7, 3, 5), (129, 2, 2), (300, 6, 64), (2, 8, 256)])
def test_rows_bound_is_reached_and_never_passed(tokens, top_k, experts):
    rows = B.mxfp8_moe_rows(tokens, top_k, experts)
    slots, used = tokens * top_k, min(experts, tokens * top_k)
    # the worst routing: every used expert but one holds one slot more than whole segments
    counts = [1] * (used - 1) + [slots - (used - 1)]
    worst = sum(-(-c // 128) * 128 for c in counts)
    assert rows % 128 == 0 and rows >= worst
    rng = np.random.default_rng(tokens)
    for _ in range(20):
        off, _, _ = orc.moe_sort(rng.integers(0, experts, (tokens, top_k)).astype(np.int32), experts, rows)
        assert off[-1] <= rows
    if slots == used:                                   # one slot per expert: the bound is exact
        assert rows == 128 * used


def test_sort_and_dispatch_and_combine_undo_each_other():
    rng = np.random.default_rng(3)
    ids = rng.integers(-1, 6, (50, 3)).astype(np.int32)
    rows = B.mxfp8_moe_rows(50, 3, 6)
    off, row_of, slot_of = orc.moe_sort(ids, 6, rows)
    x = rng.standard_normal((50, 64)).astype(np.float32)
    y = orc.moe_dispatch(x, slot_of, 3)
    back, _ = orc.moe_combine_f64(y, row_of)
    kept = (ids >= 0).sum(axis=1, keepdims=True)
    assert np.allclose(back, kept * x.astype(np.float64), rtol=1e-15)
    for e in range(6):
        live = slot_of[off[e]:off[e + 1]]
        live = live[live >= 0]
        assert (ids.reshape(-1)[live] == e).all() and (np.diff(live) > 0).all() and live.size == (ids == e).sum()


def test_combine_gradient_against_central_differences():
    rng = np.random.default_rng(4)
    ids = rng.integers(-1, 4, (9, 2)).astype(np.int32)
    rows = B.mxfp8_moe_rows(9, 2, 4)
    _, row_of, _ = orc.moe_sort(ids, 4, rows)
    src, w, dy = rng.standard_normal((rows, 5)), rng.random((9, 2)), rng.standard_normal((9, 5))
    d_src, d_w, _ = orc.moe_combine_grad_f64(dy, src, row_of, w, rows)
    loss = lambda s, ww: (orc.moe_combine_f64(s, row_of, ww)[0] * dy).sum()
    h = 1e-6
    for t in range(9):
        for j in range(2):
            up, dn = w.copy(), w.copy()
            up[t, j] += h
            dn[t, j] -= h
            assert abs((loss(src, up) - loss(src, dn)) / (2 * h) - d_w[t, j]) < 1e-7
    for r in list(row_of[row_of >= 0][:6]) + [rows - 1]:
        up, dn = src.copy(), src.copy()
        up[r, 2] += h
        dn[r, 2] -= h
        assert abs((loss(up, w) - loss(dn, w)) / (2 * h) - d_src[r, 2]) < 1e-7


def test_packed_layout_hand_worked():
    codes, scales = np.zeros((17, 160), np.uint8), np.zeros((17, 5), np.uint8)
    codes[9, 45] = 0xD            # tile 0: half 1, row 1, group 1, quarter 1, pair 2, odd column
    codes[16, 128] = 0x3          # second row tile, second column tile, first word, pair 0, even column
    scales[9, 1], scales[16, 4] = 120, 77
    p = orc.e2m1_packed(codes, scales)
    assert p.size == B.mxfp8_e2m1_packed_bytes(1, 17, 160) == 2 * 2 * 1088
    word = lambda tile, w: int.from_bytes(p[tile * 1088 + 4 * w:tile * 1088 + 4 * w + 4].tobytes(), "little")
    assert word(0, (9 * 4 + 1) * 4 + 1) == (1 << (14 + 16)) | (5 << 16)
    assert word(3, 0) == 3 << 6
    assert p[1024 + 4 * 9 + 1] == 120 and p[3 * 1088 + 1024] == 77
    assert np.count_nonzero(p) == 5        # two bytes, one byte, two scales


def test_matvec_hand_worked():
    # 1.5 * 2 in group 0 under 2^1, -6 * 0.25 in group 1 under 2^-2
    codes, scales = np.zeros((2, 1, 64), np.uint8), np.zeros((2, 1, 2), np.uint8)
    codes[1, 0, 3], codes[1, 0, 40] = 3, 15
    scales[1, 0] = [128, 125]
    x = np.zeros((1, 64), np.float32)
    x[0, 3], x[0, 40] = 2.0, 0.25
    y, mag = orc.matvec_f64(x, codes, scales, np.array([[1, 0, 5, -1]]))
    assert y[:, 0].tolist() == [6.0 - 0.375, 0.0, 0.0, 0.0] and mag[0, 0] == 6.375


P = ctypes.c_void_p(0x1000)           # never dereferenced: every call below fails validation first
ODD = ctypes.c_void_p(0x1002)
FOUR = ctypes.c_void_p(0x1004)


def test_refusals_of_the_sort():
    f = B.lib().mxfp8_moe_sort
    assert f(None, 8, 2, 4, P, P, P, 512, None, 0, None) == B.ERR_NULL
    assert f(P, 8, 2, 4, None, P, P, 512, None, 0, None) == B.ERR_NULL
    assert f(P, -1, 2, 4, P, P, P, 512, None, 0, None) == B.ERR_SHAPE
    assert f(P, 8, 0, 4, P, P, P, 512, None, 0, None) == B.ERR_SHAPE
    assert f(P, 8, 2, 0, P, P, P, 512, None, 0, None) == B.ERR_SHAPE
    assert f(P, 8, 2, 4, P, P, P, 511, None, 0, None) == B.ERR_SHAPE           # fewer rows than this batch may need
    assert f(P, 8, 2, 257, P, P, P, 1 << 20, None, 0, None) == B.ERR_UNSUPPORTED
    assert f(P, 1 << 31, 2, 4, P, P, P, 1 << 30, None, 0, None) == B.ERR_UNSUPPORTED
    assert f(ODD, 8, 2, 4, P, P, P, 512, None, 0, None) == B.ERR_ALIGN
    need = B.mxfp8_moe_sort_ws_bytes(100000, 2, 64)
    assert need > 0 and B.mxfp8_moe_sort_ws_bytes(16, 6, 64) == 0
    rows = B.mxfp8_moe_rows(100000, 2, 64)
    assert f(P, 100000, 2, 64, P, P, P, rows, None, 0, None) == B.ERR_WORKSPACE
    assert f(P, 100000, 2, 64, P, P, P, rows, P, need - 1, None) == B.ERR_WORKSPACE
    assert B.mxfp8_moe_rows(0, 2, 4) == 0 and B.mxfp8_moe_rows(5, 0, 4) == 0


def test_refusals_of_the_dispatch():
    f = B.lib().mxfp8_moe_dispatch_quantize
    call = lambda src=P, dt=B.BF16, tokens=8, cols=64, slot=P, rows=512, k=2, w=P, off=P, groups=4, o=B.BOTH, rule=0, elem=0, qr=P, sr=P, qc=P, sc=P, sf=1: \
        f(src, dt, tokens, cols, slot, rows, k, w, off, groups, o, rule, elem, qr, sr, qc, sc, sf, None)
    assert call(dt=5) == B.ERR_ENUM and call(o=0) == B.ERR_ENUM and call(rule=2) == B.ERR_ENUM and call(elem=2) == B.ERR_ENUM and call(sf=2) == B.ERR_ENUM
    assert call(src=None) == B.ERR_NULL and call(slot=None) == B.ERR_NULL and call(off=None) == B.ERR_NULL
    assert call(qr=None) == B.ERR_NULL and call(sc=None) == B.ERR_NULL
    assert call(tokens=-1) == B.ERR_SHAPE and call(cols=0) == B.ERR_SHAPE and call(rows=100) == B.ERR_SHAPE and call(k=0) == B.ERR_SHAPE
    assert call(cols=48) == B.ERR_SHAPE and call(groups=0) == B.ERR_SHAPE
    assert call(cols=40, o=B.COL) == B.ERR_UNSUPPORTED                          # 16-byte rows of codes
    assert call(src=FOUR) == B.ERR_ALIGN and call(slot=FOUR) == B.ERR_ALIGN and call(w=ODD) == B.ERR_ALIGN and call(qc=FOUR) == B.ERR_ALIGN
    assert call(tokens=1 << 31) == B.ERR_UNSUPPORTED
    assert call(tokens=0) == 0 and call(rows=0) == 0                            # nothing to do


def test_refusals_of_the_combine_and_its_gradient():
    f = B.lib().mxfp8_moe_combine
    call = lambda src=P, sdt=0, rows=512, cols=64, row_of=P, w=P, tokens=8, k=2, dst=P, ddt=0: f(src, sdt, rows, cols, row_of, w, tokens, k, dst, ddt, None)
    assert call(sdt=2) == B.ERR_ENUM and call(ddt=-1) == B.ERR_ENUM
    assert call(src=None) == B.ERR_NULL and call(row_of=None) == B.ERR_NULL and call(dst=None) == B.ERR_NULL
    assert call(rows=-1) == B.ERR_SHAPE and call(cols=0) == B.ERR_SHAPE and call(tokens=-1) == B.ERR_SHAPE and call(k=0) == B.ERR_SHAPE
    assert call(src=ODD) == B.ERR_ALIGN and call(dst=ODD) == B.ERR_ALIGN and call(row_of=ODD) == B.ERR_ALIGN and call(w=ODD) == B.ERR_ALIGN
    assert call(tokens=0) == 0
    g = B.lib().mxfp8_moe_combine_grad
    call = lambda dy=P, ddt=0, tokens=8, cols=64, src=P, sdt=0, rows=512, row_of=P, slot=P, k=2, w=P, off=P, groups=4, ds=P, dw=P: \
        g(dy, ddt, tokens, cols, src, sdt, rows, row_of, slot, k, w, off, groups, ds, dw, None)
    assert call(ddt=9) == B.ERR_ENUM and call(sdt=9) == B.ERR_ENUM
    assert call(dy=None) == B.ERR_NULL and call(row_of=None) == B.ERR_NULL and call(ds=None, dw=None) == B.ERR_NULL
    assert call(src=None) == B.ERR_NULL and call(slot=None) == B.ERR_NULL and call(off=None) == B.ERR_NULL
    assert call(cols=0) == B.ERR_SHAPE and call(groups=0) == B.ERR_SHAPE and call(k=0) == B.ERR_SHAPE
    assert call(dy=ODD) == B.ERR_ALIGN and call(dw=ODD) == B.ERR_ALIGN and call(off=ODD) == B.ERR_ALIGN
    assert call(tokens=0) == 0


def test_refusals_of_the_four_bit_product():
    f = B.lib().mxfp8_e2m1_matvec
    call = lambda x=P, tokens=2, cols=64, packed=P, m=1, rows=16, ids=None, per=1, y=P, ydt=0: f(x, tokens, cols, packed, m, rows, ids, per, y, ydt, None)
    assert call(ydt=3) == B.ERR_ENUM
    assert call(x=None) == B.ERR_NULL and call(packed=None) == B.ERR_NULL and call(y=None) == B.ERR_NULL
    assert call(tokens=0) == B.ERR_SHAPE and call(cols=48) == B.ERR_SHAPE and call(rows=0) == B.ERR_SHAPE and call(m=0) == B.ERR_SHAPE
    assert call(m=2) == B.ERR_SHAPE and call(per=2) == B.ERR_SHAPE             # several matrices or choices need the numbers
    assert call(x=FOUR) == B.ERR_ALIGN and call(y=ODD) == B.ERR_ALIGN and call(ids=ODD, m=2) == B.ERR_ALIGN
    assert call(tokens=1025) == B.ERR_UNSUPPORTED and call(tokens=600, per=2, ids=P, m=4) == B.ERR_UNSUPPORTED
    g = B.lib().mxfp8_e2m1_pack
    assert g(None, P, 1, 16, 64, P, None) == B.ERR_NULL and g(P, P, 1, 16, 48, P, None) == B.ERR_SHAPE
    assert g(P, P, 0, 16, 64, P, None) == B.ERR_SHAPE and g(FOUR, P, 1, 16, 64, P, None) == B.ERR_ALIGN
    assert g(P, P, 1 << 20, 1 << 20, 1 << 20, P, None) == B.ERR_UNSUPPORTED
    assert B.mxfp8_e2m1_packed_bytes(3, 16, 128) == 3 * 1088 and B.mxfp8_e2m1_packed_bytes(1, 1, 32) == 1088 and B.mxfp8_e2m1_packed_bytes(1, 0, 32) == 0


def test_the_binding_refuses_foreign_tensors():
    import torch
    cpu = torch.zeros(4, 2, dtype=torch.int32)
    if torch.cuda.is_available():
        with pytest.raises(ValueError):
            B.mxfp8_moe_sort(cpu, 4, cpu, cpu, cpu)
    with pytest.raises(TypeError):
        B.mxfp8_moe_sort(cpu.long(), 4, cpu, cpu, cpu)
    with pytest.raises(TypeError):
        B.mxfp8_e2m1_matvec(torch.zeros(1, 64), cpu, 1, None, torch.zeros(1, 16))
