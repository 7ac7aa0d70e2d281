"""Cases, plain forms and 64-bit references of the mixture-of-experts operators and of the 4-bit matrix-vector product.

``sort``      expert numbers of every token -> segment starts (multiples of 128), row of every slot, slot of every row
``dispatch``  tokens gathered into the sorted order, optionally weighted, and converted to MXFP8 in one pass
``combine``   rows of the experts' outputs gathered back, weighted and summed per token (forward), or its gradient
``matvec``    products of a few tokens with E2M1 (MXFP4) matrices, one matrix for all or one chosen per token

A *slot* is one (token, choice) pair, numbered token * top_k + choice.
"""
import math

import torch

own = False

ROW, COL, BOTH = 1, 2, 3
TILE = 128          # rows of a scale atom: every expert's segment starts at a multiple of it


# ----------------------------------------------------------------------------------- cases

def listed():
    return [
        # a decoding batch of 16 sequences is routed: the smallest call, all latency
        dict(name="sort decode", op="sort", tokens=16, top_k=6, experts=64, skew=1.0, dropped=0.0),
        # the layer of the grouped-GEMM sweep: 8192 tokens, 6 of 64 experts each, uneven popularity
        dict(name="sort layer", op="sort", tokens=8192, top_k=6, experts=64, skew=1.0, dropped=0.0),
        # a long batch over the most experts a grouped product takes, some slots without an expert (capacity limits)
        dict(name="sort long", op="sort", tokens=131071, top_k=8, experts=256, skew=0.5, dropped=0.05),
        # the same layer, forward: BF16 activations, both orientations (FPROP reads rows, WGRAD columns)
        dict(name="dispatch layer", op="dispatch", tokens=8192, top_k=6, experts=64, cols=2048, src="bf16", weighted=False,
             orientation=BOTH, rule="paper", elem="e4m3", swizzled=True, skew=1.0, dropped=0.0),
        # backward of the weighted sum: the output gradient of a ragged batch, weighted, in FP32 and E5M2
        dict(name="dispatch gradient", op="dispatch", tokens=2999, top_k=2, experts=8, cols=4096, src="fp32", weighted=True,
             orientation=BOTH, rule="ocp", elem="e5m2", swizzled=True, skew=0.5, dropped=0.02),
        # a prefill of a few hundred tokens, forward only
        dict(name="dispatch prefill", op="dispatch", tokens=301, top_k=2, experts=16, cols=1408, src="bf16", weighted=False,
             orientation=ROW, rule="paper", elem="e4m3", swizzled=True, skew=0.5, dropped=0.0),
        # the layer's way back: BF16 outputs of the experts, weighted sum of six rows per token
        dict(name="combine layer", op="combine", grad=False, tokens=8192, top_k=6, experts=64, cols=2048, src="bf16", dst="bf16",
             weighted=True, skew=1.0, dropped=0.0),
        # one decoding step of eight sequences, FP32 products in, BF16 out
        dict(name="combine decode", op="combine", grad=False, tokens=8, top_k=2, experts=8, cols=4096, src="fp32", dst="bf16",
             weighted=True, skew=0.5, dropped=0.0),
        # gradient of the layer's weighted sum: every row's gradient and every weight's
        dict(name="combine gradient", op="combine", grad=True, tokens=8192, top_k=6, experts=64, cols=2048, src="bf16", dst="bf16",
             weighted=True, skew=1.0, dropped=0.01),
        # one token through the fused query / key / value projection of an 8B decoder block
        dict(name="matvec one token", op="matvec", tokens=1, top_k=1, matrices=1, rows=6144, cols=4096, out="bf16", chosen=False),
        # one decoding step of sixteen sequences through the gate / up projection of that block
        dict(name="matvec batch", op="matvec", tokens=16, top_k=1, matrices=1, rows=28672, cols=4096, out="bf16", chosen=False),
        # eight sequences, six experts each, through their experts' gate / up projections (2 x 1408 wide)
        dict(name="matvec experts", op="matvec", tokens=8, top_k=6, matrices=64, rows=2816, cols=2048, out="fp32", chosen=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sort", "dispatch", "combine", "combine", "matvec", "matvec"])
    skew, dropped = round(rng.uniform(0.0, 1.5), 2), rng.choice([0.0, 0.0, 0.01, 0.1])
    if op == "sort":
        experts = rng.choice([1, 5, 8, 16, 60, 64, 128, 160, 256])
        top_k = rng.randint(1, min(8, experts))
        return dict(op=op, tokens=_log(rng, 1, 131071), top_k=top_k, experts=experts, skew=skew, dropped=dropped)
    if op == "matvec":
        matrices = rng.choice([1, 1, 8, 16, 64])
        rows, cols = _log(rng, 64, 14336), 32 * _log(rng, 2, 256)
        if matrices > 1:
            rows, cols = min(rows, 4099), min(cols, 4096)
        return dict(op=op, tokens=_log(rng, 1, 16 if matrices > 1 else 64), top_k=rng.randint(1, min(6, matrices)), matrices=matrices, rows=rows, cols=cols,
                    out=rng.choice(["bf16", "fp32"]), chosen=matrices > 1)
    experts = rng.choice([4, 8, 16, 60, 64])
    top_k = rng.randint(1, min(6, experts))
    src = rng.choice(["bf16", "bf16", "fp32"])
    tokens = min(_log(rng, 1, 8192), (8192 * 6 if src == "bf16" else 8192 * 2) // top_k)
    if op == "dispatch":
        return dict(op=op, tokens=tokens, top_k=top_k, experts=experts, cols=32 * rng.randint(1, 64), src=src, weighted=rng.random() < 0.5,
                    orientation=rng.choice([ROW, COL, BOTH, BOTH]), rule=rng.choice(["paper", "ocp"]), elem=rng.choice(["e4m3", "e5m2"]),
                    swizzled=rng.random() < 0.7, skew=skew, dropped=dropped)
    grad = rng.random() < 0.5
    return dict(op=op, grad=grad, tokens=tokens, top_k=top_k, experts=experts, cols=rng.randint(1, 2048), src=src,
                dst=rng.choice(["bf16", "fp32"]), weighted=grad or rng.random() < 0.7, skew=skew, dropped=dropped)


def work(case):
    op, slots = case["op"], case["tokens"] * case["top_k"]
    size = {"bf16": 2, "fp32": 4}
    if op == "sort":
        return dict(bytes=4 * (3 * slots + case["experts"] + 1), flops=0)
    if op == "matvec":
        used = min(case["matrices"], slots)
        weights = used * case["rows"] * case["cols"]
        return dict(bytes=weights * 17 // 32 + 2 * case["tokens"] * case["cols"] + size[case["out"]] * slots * case["rows"],
                    flops=2 * slots * case["rows"] * case["cols"])
    n, h, s = case["tokens"], case["cols"], size[case["src"]]
    if op == "dispatch":
        sides = 2 if case["orientation"] == BOTH else 1
        return dict(bytes=n * h * s + 4 * slots + sides * slots * h * 33 // 32, flops=slots * h)
    if case["grad"]:
        return dict(bytes=n * h * size[case["dst"]] + 2 * slots * h * s + 12 * slots, flops=3 * slots * h)
    return dict(bytes=slots * h * s + n * h * size[case["dst"]] + 8 * slots, flops=2 * slots * h)


# ---------------------------------------------------------------------------------- inputs

DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _routing(case, g):
    """What a router gives: top_k different experts per token by noisy logits, softmax weights over them."""
    n, k, e = case["tokens"], case["top_k"], case.get("experts") or case["matrices"]
    popularity = torch.randn(e, generator=g, device="cuda") * case.get("skew", 0.5)
    logits = torch.randn(n, e, generator=g, device="cuda") + popularity
    top, ids = logits.topk(k, dim=1)
    weights = torch.softmax(top, dim=1).contiguous()
    lost = torch.rand(n, k, generator=g, device="cuda") < case.get("dropped", 0.0)
    return ids.to(torch.int32).masked_fill(lost, -1).contiguous(), weights


def capacity(tokens, top_k, experts):
    """Rows that hold every possible routing: each used expert pads its segment by at most 127 rows."""
    slots = tokens * top_k
    return (slots + (TILE - 1) * min(experts, slots)) // TILE * TILE


def plain_sort(ids, experts, rows):
    """group_offsets [experts + 1], row_of [tokens, top_k], slot_of [rows]; -1 where there is none."""
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < experts), flat, experts)
    counts = torch.zeros(experts + 1, dtype=torch.long, device=ids.device).scatter_add_(0, key, torch.ones_like(key))
    order = torch.sort(key, stable=True).indices
    padded = (counts[:experts] + TILE - 1) // TILE * TILE
    zero = torch.zeros(1, dtype=torch.long, device=ids.device)
    offsets = torch.cat([zero, padded.cumsum(0)])
    first = torch.cat([zero, counts.cumsum(0)])[:experts + 1]           # place of each expert's first slot in `order`
    sorted_key = key[order]
    rank = torch.arange(flat.numel(), device=ids.device) - first[sorted_key]
    row = torch.where(sorted_key < experts, offsets[sorted_key] + rank, torch.full_like(rank, rows))
    row_of = torch.empty_like(flat)
    row_of[order] = torch.where(row < rows, row, torch.full_like(row, -1))
    slot_of = torch.full((rows + 1,), -1, dtype=torch.long, device=ids.device)
    slot_of[row] = order
    return offsets.to(torch.int32), row_of.to(torch.int32).reshape(ids.shape), slot_of[:rows].to(torch.int32)


def scale_bytes(mn, blocks, swizzled):
    return (mn + 127) // 128 * ((blocks + 3) // 4) * 512 if swizzled else mn * blocks


def prepare(case, seed):
    g = _generator(seed)
    ids, weights = _routing(case, g)
    st = dict(case=case, ids=ids, weights=weights, seed=seed)
    n, k = case["tokens"], case["top_k"]

    def empty(*shape, dtype):
        return torch.zeros(*shape, dtype=dtype, device="cuda")

    if case["op"] == "matvec":
        e, r, c = case["matrices"], case["rows"], case["cols"]
        st["x"] = torch.randn(n, c, generator=g, device="cuda").to(torch.bfloat16)
        # what a Gaussian matrix of spread 0.02 becomes: codes of values up to 6, scales near 2^-7; laid out in tiles
        code = torch.randint(0, 256, (e, (r + 15) // 16, (c + 127) // 128, 16, 64), generator=g, device="cuda", dtype=torch.uint8)
        byte = torch.randint(117, 122, (e, (r + 15) // 16, (c + 127) // 128, 16, 4), generator=g, device="cuda", dtype=torch.uint8)
        # rows and columns past the matrix are zero codes under zero scale bytes
        inside_r = (torch.arange((r + 15) // 16 * 16, device="cuda") < r).reshape(-1, 1, 16, 1)
        inside_c = (torch.arange((c + 127) // 128 * 4, device="cuda") * 32 < c).reshape(1, -1, 1, 4)
        inside = inside_r & inside_c                                                       # one flag per 32-wide group
        code = code * inside.repeat_interleave(16, dim=3).to(torch.uint8)
        byte = byte * inside.to(torch.uint8)
        # inside a tile: [half, row % 8, quarter of a group, group] words of eight codes, then [row, group] scale bytes
        code = code.reshape(e, -1, code.shape[2], 2, 8, 4, 4, 4).permute(0, 1, 2, 3, 4, 6, 5, 7).reshape(*code.shape[:3], 1024)
        st["packed"] = torch.cat([code, byte.reshape(*code.shape[:3], 64)], dim=3).contiguous()
        st["y"] = empty(n * k, r, dtype=DTYPE[case["out"]])
        return st
    experts = case["experts"]
    rows = capacity(n, k, experts)
    st["rows"] = rows
    if case["op"] == "sort":
        st["offsets"], st["row_of"], st["slot_of"] = (empty(experts + 1, dtype=torch.int32), empty(n, k, dtype=torch.int32),
                                                      empty(rows, dtype=torch.int32))
        st["ws"] = empty(4 * experts * 1024, dtype=torch.uint8)
        return st
    st["offsets"], st["row_of"], st["slot_of"] = plain_sort(ids, experts, rows)
    h = case["cols"]
    if not case["weighted"]:
        st["weights"] = None
    if case["op"] == "dispatch":
        x = torch.randn(n, h, generator=g, device="cuda")
        if case["weighted"]:                                               # an output gradient: small, uneven from token to token
            x = x * (1e-6 * torch.exp(2.0 * torch.randn(n, 1, generator=g, device="cuda")))
        st["x"] = x.to(DTYPE[case["src"]])
        for o, name, mn, blocks in ((ROW, "row", rows, h // 32), (COL, "col", h, rows // 32)):
            used = case["orientation"] & o
            st["q_" + name] = empty(rows, h, dtype=torch.uint8) if used else None
            st["s_" + name] = empty(scale_bytes(mn, blocks, case["swizzled"]), dtype=torch.uint8) if used else None
        return st
    # the experts' outputs in sorted order, zero in the padding
    live = (st["slot_of"] >= 0).unsqueeze(1)
    st["y"] = (torch.randn(rows, h, generator=g, device="cuda") * live).to(DTYPE[case["src"]])
    if case["grad"]:
        st["dy"] = (1e-3 * torch.randn(n, h, generator=g, device="cuda")).to(DTYPE[case["dst"]])
        st["d_y"] = empty(rows, h, dtype=DTYPE[case["src"]])
        st["d_weights"] = empty(n, k, dtype=torch.float32)
    else:
        st["out"] = empty(n, h, dtype=DTYPE[case["dst"]])
    return st


# ----------------------------------------------------------------------------- plain forms

ELEM = {"e4m3": (448.0, 8, torch.float8_e4m3fn), "e5m2": (57344.0, 15, torch.float8_e5m2)}


def _swizzle(s):
    """[mn, blocks] scale bytes in atoms of 128 x 4: byte (mn % 32) * 16 + (mn % 128) / 32 * 4 + block % 4 of each."""
    mn, nb = s.shape
    s = torch.nn.functional.pad(s, (0, -nb % 4, 0, -mn % 128))
    return s.reshape(s.shape[0] // 128, 4, 32, s.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1)


def _plain_quantize(y, axis, rule, elem, swizzled):
    """MXFP8 codes (as 8-bit floating values) and scale bytes of y, 32 values along `axis` to a block; y is finite."""
    largest, emax, kind = ELEM[elem]
    blocks = y.unflatten(axis, (-1, 32))
    bits = blocks.abs().amax(dim=axis + 1).view(torch.int32)
    field = bits >> 23
    up = ((bits & 0x7FFFFF) > 0x600000).int() if rule == "paper" else 0
    byte = torch.where(field == 0, 0, field - emax + up).clamp(min=0)
    inverse = ((254 - byte) << 23).view(torch.float32)
    q = (blocks * inverse.unsqueeze(axis + 1)).clamp(-largest, largest).to(kind).reshape(y.shape)
    byte = byte.to(torch.uint8)
    if not swizzled:
        return q, byte.reshape(-1)
    return q, _swizzle(byte if axis == 1 else byte.t())


def _gathered(x, slot_of, top_k, weights):
    """Rows of x in sorted order, weighted in 32 bits and rounded to x's type; zero where a row has no slot."""
    slot = slot_of.long().clamp(min=0)
    y = x[slot // top_k].float()
    if weights is not None:
        y = (y * weights.reshape(-1)[slot].unsqueeze(1)).to(x.dtype).float()
    return y * (slot_of >= 0).unsqueeze(1)


def _plain_dispatch(st):
    case = st["case"]
    y = _gathered(st["x"], st["slot_of"], case["top_k"], st["weights"])
    out = {}
    if case["orientation"] & ROW:
        out["q_row"], out["s_row"] = _plain_quantize(y, 1, case["rule"], case["elem"], case["swizzled"])
    if case["orientation"] & COL:
        out["q_col"], out["s_col"] = _plain_quantize(y, 0, case["rule"], case["elem"], case["swizzled"])
    return out


def _plain_combine(st):
    row = st["row_of"].long()
    live = (row >= 0).unsqueeze(2)
    rows = st["y"][row.clamp(min=0)].float() * live
    if st["weights"] is not None:
        rows = rows * st["weights"].unsqueeze(2)
    return rows.sum(dim=1).to(DTYPE[st["case"]["dst"]])


def _plain_combine_grad(st):
    row, slot = st["row_of"].long(), st["slot_of"].long()
    dy = st["dy"].float()
    d_weights = (st["y"][row.clamp(min=0)].float() * dy.unsqueeze(1)).sum(dim=2) * (row >= 0)
    s = slot.clamp(min=0)
    d_y = dy[s // st["case"]["top_k"]] * st["weights"].reshape(-1)[s].unsqueeze(1) * (slot >= 0).unsqueeze(1)
    return d_y.to(st["y"].dtype), d_weights


# Where the codes of a word's eight columns lie: even columns in its low half, odd ones in its high half
SIGN_BIT, VALUE_BITS = (15, 12, 14, 13), (6, 3, 0, 9)


def _decoded(packed, rows, cols):
    """[matrices, rows, cols] values of packed E2M1 tiles in 32 bits."""
    e, rb, kb, _ = packed.shape
    word = packed[..., :1024].contiguous().view(torch.int32).reshape(e, rb, kb, 2, 8, 4, 4)    # half, row % 8, quarter, group
    word = word.permute(0, 1, 3, 4, 2, 6, 5).reshape(e, rb * 16, kb * 16)
    scale = packed[..., 1024:].reshape(e, rb, kb, 16, 4).permute(0, 1, 3, 2, 4).reshape(e, rb * 16, kb * 4)
    sign = torch.stack([word >> (SIGN_BIT[i // 2] + 16 * (i % 2)) for i in range(8)], dim=3) & 1
    code = torch.stack([word >> (VALUE_BITS[i // 2] + 16 * (i % 2)) for i in range(8)], dim=3) & 7
    # two exponent bits, one mantissa bit: m / 2 below the smallest exponent, (1 + m / 2) 2^(e - 1) above
    exponent, half = code >> 1, 0.5 * (code & 1).float()
    value = torch.where(exponent == 0, half, (1 + half) * ((exponent + 126) << 23).view(torch.float32))
    value = (value * (1 - 2 * sign.float())).reshape(e, rb * 16, kb * 128)
    return (value * (scale.int() << 23).view(torch.float32).repeat_interleave(32, dim=2))[:, :rows, :cols]


def _plain_products(st):
    case = st["case"]
    x = st["x"].float()
    if not case["chosen"]:
        return x @ _decoded(st["packed"], case["rows"], case["cols"])[0].t()
    used, at = torch.unique(st["ids"].reshape(-1).long(), return_inverse=True)      # each chosen matrix is decoded once
    w = _decoded(st["packed"][used], case["rows"], case["cols"])
    return torch.bmm(w[at], x.repeat_interleave(case["top_k"], dim=0).unsqueeze(2)).squeeze(2)


def run(state):
    case = state["case"]
    if own:
        return _own(state)
    if case["op"] == "sort":
        return plain_sort(state["ids"], case["experts"], state["rows"])
    if case["op"] == "dispatch":
        return _plain_dispatch(state)
    if case["op"] == "combine":
        return _plain_combine_grad(state) if case["grad"] else _plain_combine(state)
    return _plain_products(state).to(DTYPE[case["out"]])


def _own(st):
    """The calls that a user makes of the library."""
    from paper_2506_08027_b200 import binding as B
    case = st["case"]
    if case["op"] == "sort":
        B.mxfp8_moe_sort(st["ids"], case["experts"], st["offsets"], st["row_of"], st["slot_of"], st["ws"])
        return st["offsets"], st["row_of"], st["slot_of"]
    if case["op"] == "dispatch":
        B.mxfp8_moe_dispatch_quantize(st["x"], st["slot_of"], case["top_k"], st["weights"], st["offsets"], case["orientation"],
                                      B.RULE_PAPER if case["rule"] == "paper" else B.RULE_OCP, B.E4M3 if case["elem"] == "e4m3" else B.E5M2,
                                      st["q_row"], st["s_row"], st["q_col"], st["s_col"],
                                      B.SF_SWIZZLED if case["swizzled"] else B.SF_LINEAR)
        kind, out = ELEM[case["elem"]][2], {}
        for o, name in ((ROW, "row"), (COL, "col")):
            if case["orientation"] & o:
                out["q_" + name], out["s_" + name] = st["q_" + name].view(kind), st["s_" + name]
        return out
    if case["op"] == "combine" and case["grad"]:
        B.mxfp8_moe_combine_grad(st["dy"], st["y"], st["row_of"], st["slot_of"], st["weights"], st["offsets"], st["d_y"], st["d_weights"])
        return st["d_y"], st["d_weights"]
    if case["op"] == "combine":
        B.mxfp8_moe_combine(st["y"], st["row_of"], st["weights"], st["out"])
        return st["out"]
    B.mxfp8_e2m1_matvec(st["x"], st["packed"], case["matrices"], st["ids"] if case["chosen"] else None, st["y"])
    return st["y"]


# ------------------------------------------------------------------------------ in 64 bits

def _two(n):
    """2^n for whole numbers n of an ordinary exponent."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _fp8_grid(v, mantissa, smallest_exponent, largest):
    """Nearest value with so many mantissa bits (even at a tie), not finer than the subnormals, at most the largest."""
    _, e = torch.frexp(v)
    step = _two((e - 1).clamp(min=smallest_exponent) - mantissa)
    return (torch.round(v / step) * step).clamp(-largest, largest)


def _exact_codes(v, axis, rule, elem):
    largest, emax, mantissa, least = {"e4m3": (448.0, 8, 3, -6), "e5m2": (57344.0, 15, 2, -14)}[elem]
    blocks = v.unflatten(axis, (-1, 32))
    peak = blocks.abs().amax(dim=axis + 1, keepdim=True)
    fraction, e = torch.frexp(peak if rule == "ocp" else peak / largest)
    # ocp: floor(log2 peak) - emax; paper: ceil(log2(peak / largest)), exact at powers of two
    exponent = (e - 1 - emax) if rule == "ocp" else torch.where(fraction == 0.5, e - 1, e)
    exponent = torch.where(peak == 0, torch.full_like(exponent, -127), exponent).clamp(-127, 127)
    return _fp8_grid(blocks * _two(-exponent), mantissa, least, largest).reshape(v.shape)


E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)       # by the three value bits


def _exact_products(st):
    case = st["case"]
    e, r, c, k = case["matrices"], case["rows"], case["cols"], case["top_k"]
    if case["tokens"] * k * r * c > (15e8 if case["chosen"] else 15e9):
        return None
    flat = st["packed"].reshape(e, -1)
    table = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
    row, col = torch.arange(r, device="cuda").unsqueeze(1), torch.arange(c, device="cuda").unsqueeze(0)
    tile = ((row // 16) * ((c + 127) // 128) + col // 128) * 1088
    word = (tile + row % 16 // 8 * 512 + row % 8 * 64 + col % 32 // 8 * 16 + col % 128 // 32 * 4) // 4
    group = tile + 1024 + row % 16 * 4 + col % 128 // 32
    pair, high = col % 8 // 2, 16 * (col % 2)
    sign_at = torch.tensor(SIGN_BIT, device="cuda")[pair] + high
    value_at = torch.tensor(VALUE_BITS, device="cuda")[pair] + high
    out = torch.empty(case["tokens"] * k, r, dtype=torch.float64, device="cuda")
    ids = st["ids"].reshape(-1) if case["chosen"] else torch.zeros(case["tokens"], dtype=torch.int32, device="cuda")
    for m in ids.unique().tolist():
        bits = flat[m].view(torch.int32)[word].long()
        w = table[(bits >> value_at) & 7] * (1 - 2 * ((bits >> sign_at) & 1)) * _two(flat[m][group].int() - 127)
        slots = torch.nonzero(ids == m).reshape(-1)
        out[slots] = st["x"].double()[slots // k] @ w.t()
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "sort":
        return None
    n, k = case["tokens"], case["top_k"]
    if case["op"] == "matvec":
        return _exact_products(st)
    w = torch.ones(n, k, dtype=torch.float64, device="cuda") if st["weights"] is None else st["weights"].double()
    row = st["row_of"].reshape(-1).long()
    slots = torch.nonzero(row >= 0).reshape(-1)
    if case["op"] == "dispatch":
        v = torch.zeros(st["rows"], case["cols"], dtype=torch.float64, device="cuda")
        # the definition converts a tensor of the source's type: one rounding before the blocks are formed
        v[row[slots]] = (st["x"].double()[slots // k] * w.reshape(-1)[slots].unsqueeze(1)).to(st["x"].dtype).double()
        out = {}
        for o, name, axis in ((ROW, "row", 1), (COL, "col", 0)):
            if case["orientation"] & o:
                out["q_" + name], out["s_" + name] = _exact_codes(v, axis, case["rule"], case["elem"]), None
        return out
    if not case["grad"]:
        out = torch.zeros(n, case["cols"], dtype=torch.float64, device="cuda")
        return out.index_add_(0, slots // k, st["y"].double()[row[slots]] * w.reshape(-1)[slots].unsqueeze(1))
    d_y = torch.zeros(st["rows"], case["cols"], dtype=torch.float64, device="cuda")
    d_w = torch.zeros(n * k, dtype=torch.float64, device="cuda")
    dy = st["dy"].double()[slots // k]
    d_y[row[slots]] = dy * w.reshape(-1)[slots].unsqueeze(1)
    d_w[slots] = (dy * st["y"].double()[row[slots]]).sum(dim=1)
    return d_y, d_w.reshape(n, k)
