"""Cases, plain forms and 64-bit references of what stands around a block's MXFP8 products.

``boundary``  the seam between two blocks: norm after the block, gate, residual sum, norm before the next one, with the
              next block's input in BF16 / FP32 or converted to MXFP8
``gradient``  its backward pass: gradients of the block's output, of the residual stream, of the norms' weights and the gate
``clip``      norm of all gradients of a step taken together, and the gradients scaled to a largest norm
``moe``       a mixture-of-experts layer for a few tokens with E2M1 (MXFP4) matrices: choice of the experts, gate / up
              products, activation, down products, weighted sum
"""
import math

import torch

own = False

ROW, COL, BOTH = 1, 2, 3
EPS = 1e-5
NORM_EPS = 1e-6                       # added to the gradients' norm before it divides


# ----------------------------------------------------------------------------------- cases

# matrices of a decoder block's fused query / key / value, output, gate / up and down projections, and its two norms
BLOCK = "6144x4096 4096x4096 28672x4096 4096x14336 4096 4096"
SMALL_BLOCK = "2304x768 2304 768x768 768 2047x768 2047 768x2047 768 768 768"


def _seam(name, rows, cols, block, stream, params, post, gate, gates, out, op="boundary"):
    case = dict(op=op, rows=rows, cols=cols, block=block, stream=stream, params=params, post=post, gate=gate, gates=gates, out=out)
    return dict(case, name=name) if name else case


def listed():
    return [
        # eight sequences answer one token each: the smallest call, all latency
        _seam("seam decode", 8, 4096, "bf16", "bf16", "bf16", True, False, 1, "x"),
        # the tokens of a training step, norms on both sides of the block, BF16 throughout
        _seam("seam layer", 8192, 4096, "bf16", "bf16", "bf16", True, False, 1, "x"),
        # the same tokens, the next block's input converted along rows (FPROP) and columns (WGRAD)
        _seam("seam mxfp8", 8192, 4096, "bf16", "bf16", "bf16", True, False, 1, "both"),
        # a stream in 32 bits with a gate for every sequence, an odd width, no norm after the block
        _seam("seam gated", 2999, 1409, "bf16", "fp32", "fp32", False, True, 7, "x"),
        # backward of the training step's seam
        _seam("gradient layer", 8192, 4096, "bf16", "bf16", "bf16", True, False, 1, "x", op="gradient"),
        # backward with everything: a stream in 32 bits, a gate for each of five sequences whose lengths fill no tile
        _seam("gradient gated", 5 * 613, 2048, "bf16", "fp32", "fp32", True, True, 5, "x", op="gradient"),
        # adapters' or a small model's gradients, many short tensors one behind the other
        dict(name="clip small", op="clip", sizes=" ".join([SMALL_BLOCK] * 2), types="bf16", pad=1, in_place=False, clipped=True),
        # weight gradients of one block in 32 bits, as WGRAD leaves them, scaled
        dict(name="clip block", op="clip", sizes=BLOCK, types="fp32", pad=64, in_place=False, clipped=True),
        # a model of several blocks, vectors in 32 bits, within its largest norm: the gradients stay where they are
        dict(name="clip model", op="clip", sizes=" ".join([BLOCK] * 6), types="mixed", pad=64, in_place=True, clipped=False),
        # one token through eight of 64 experts of 1408: latency and the bytes of eight experts
        dict(name="moe one token", op="moe", tokens=1, top_k=8, experts=64, cols=2048, inner=1408, out="bf16", renormalize=True, masked=0.0),
        # sixteen sequences, six experts each: nearly all experts are read
        dict(name="moe batch", op="moe", tokens=16, top_k=6, experts=64, cols=2048, inner=1408, out="bf16", renormalize=True, masked=0.0),
        # thirty-two sequences, two of eight wide experts, some rows of the batch empty
        dict(name="moe wide", op="moe", tokens=32, top_k=2, experts=8, cols=4096, inner=14336, out="fp32", renormalize=False, masked=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["boundary", "boundary", "gradient", "gradient", "clip", "clip", "moe", "moe"])
    if op in ("boundary", "gradient"):
        block, stream = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
        out = rng.choice(["x", "x", "row", "both"]) if op == "boundary" else "x"
        params = stream if out != "x" else rng.choice(["bf16", "fp32"])
        cols = _log(rng, 17, 8192)
        rows = _log(rng, 1, 8192)
        if out != "x":
            cols, rows = max(32, cols // 32 * 32), max(32, rows // 32 * 32)
        rows = min(rows, max(32, (1 << (25 if block == stream == "bf16" else 23)) // cols // 32 * 32))
        gate = rng.random() < 0.5
        per_gate = -(-rows // (rng.choice([1, rng.randint(1, 9)]) if gate else 1))
        return _seam(None, rows, cols, block, stream, params, rng.random() < 0.7, gate, -(-rows // per_gate), out, op)
    if op == "clip":
        total, share = _log(rng, 1 << 10, 1 << 28), [rng.gammavariate(0.3, 1.0) + 1e-9 for _ in range(_log(rng, 1, 300))]
        sizes = [str(max(1, int(total * v / sum(share)))) for v in share]
        in_place = rng.random() < 0.3
        return dict(op=op, sizes=" ".join(sizes), types=rng.choice(["bf16", "fp32", "mixed"]), pad=rng.choice([1, 64]), in_place=in_place,
                    clipped=not in_place and rng.random() < 0.8)
    experts = rng.choice([4, 8, 16, 60, 64, 128, 256])
    cols = 32 * _log(rng, 4, 128)
    inner = 32 * min(_log(rng, 2, 256), max(2, (1 << 28) // (32 * experts * cols)))
    tokens = _log(rng, 1, 32)
    return dict(op=op, tokens=tokens, top_k=rng.randint(1, min(8, experts)), experts=experts, cols=cols, inner=inner, out=rng.choice(["bf16", "fp32"]),
                renormalize=rng.random() < 0.6, masked=0.1 if tokens > 8 and rng.random() < 0.4 else 0.0)


BYTES = {"bf16": 2, "fp32": 4}


def work(case):
    op = case["op"]
    if op == "clip":
        total = sum(n * BYTES[t] for n, t in _tensors(case))
        count = sum(n for n, _ in _tensors(case))
        return dict(bytes=total if case["in_place"] else 2 * total, flops=3 * count)
    if op == "moe":
        n, k, h, f = case["tokens"], case["top_k"], case["cols"], case["inner"]
        # experts that tokens choosing at random are expected to reach
        used = case["experts"] * (1 - (1 - k / case["experts"]) ** n)
        return dict(bytes=int(used * 3 * f * h * 17 / 32) + 2 * n * h + BYTES[case["out"]] * n * h + 4 * n * case["experts"], flops=6 * n * k * h * f)
    r, c, b, s, p = case["rows"], case["cols"], BYTES[case["block"]], BYTES[case["stream"]], BYTES[case["params"]]
    vectors = c * p * (1 + case["post"] + (case["gates"] if case["gate"] else 0))
    if op == "gradient":
        return dict(bytes=r * c * (3 * b + 3 * s) + 8 * r + vectors * (1 + 4 // p), flops=24 * r * c)
    converted = {"x": b * r * c, "row": r * c * 33 // 32, "both": r * c * 33 // 16}[case["out"]]
    return dict(bytes=r * c * (b + 2 * s) + converted + 8 * r + vectors, flops=12 * r * c)


# ---------------------------------------------------------------------------------- inputs

DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _numel(text):
    n = 1
    for part in text.split("x"):
        n *= int(part)
    return n


def _tensors(case):
    """(elements, type) of every gradient; with mixed types matrices are BF16 and vectors FP32 (sizes alone: by parity)."""
    out = []
    for text in case["sizes"].split():
        n = _numel(text)
        short = "x" not in text and (n % 2 == 0 or n < 64)
        out.append((n, case["types"] if case["types"] != "mixed" else ("fp32" if short else "bf16")))
    return out


def scale_bytes(mn, blocks):
    return (mn + 127) // 128 * ((blocks + 3) // 4) * 512


def _prepare_seam(case, st, g):
    r, c = case["rows"], case["cols"]
    block, stream, params = DTYPE[case["block"]], DTYPE[case["stream"]], DTYPE[case["params"]]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    # a residual stream has a few channels far above the others; rows of a block's output differ in size
    loud = 1 + 20 * (torch.rand(c, generator=g, device="cuda") < 0.005)
    st["h_in"] = (randn(r, c) * loud).to(stream)
    st["y"] = (0.5 * randn(r, c) * torch.exp(0.3 * randn(r, 1))).to(block)
    st["gamma_pre"] = (1 + 0.1 * randn(c)).to(params)
    st["gamma_post"] = (1 + 0.1 * randn(c)).to(params) if case["post"] else None
    st["gate"] = (0.5 * randn(case["gates"], c)).to(params) if case["gate"] else None
    st["rows_per_gate"] = (r + case["gates"] - 1) // case["gates"]
    st["residual_scale"], st["branch_scale"] = 1.0, 0.75
    st["rstd_post"] = torch.zeros(r, device="cuda") if case["post"] else None
    st["rstd_pre"] = torch.zeros(r, device="cuda")
    if case["op"] == "boundary":
        st["h"] = torch.zeros(r, c, dtype=stream, device="cuda")
        if case["out"] == "x":
            st["x"] = torch.zeros(r, c, dtype=block, device="cuda")
        else:
            for o, name, mn, blocks in ((ROW, "row", r, c // 32), (COL, "col", c, r // 32)):
                used = case["out"] == "both" or name == "row"
                st["q_" + name] = torch.zeros(r, c, dtype=torch.uint8, device="cuda") if used else None
                st["s_" + name] = torch.zeros(scale_bytes(mn, blocks), dtype=torch.uint8, device="cuda") if used else None
        return
    # what the forward pass keeps
    h, rp, rn = _plain_stream(st)
    st["h"], st["rstd_pre"] = h, rn.reshape(-1).contiguous()
    if case["post"]:
        st["rstd_post"] = rp.reshape(-1).contiguous()
    size = 1e-4 * torch.exp(randn(r, 1))
    st["dx"] = (size * randn(r, c)).to(block)
    st["dh"] = (size * randn(r, c)).to(stream)
    st["dy"], st["dh_in"] = torch.zeros(r, c, dtype=block, device="cuda"), torch.zeros(r, c, dtype=stream, device="cuda")
    st["d_gamma_pre"] = torch.zeros(c, device="cuda")
    st["d_gamma_post"] = torch.zeros(c, device="cuda") if case["post"] else None
    st["d_gate"] = torch.zeros(case["gates"], c, device="cuda") if case["gate"] else None


def _prepare_clip(case, st, g):
    at, places = {"bf16": 0, "fp32": 0}, []
    for n, t in _tensors(case):
        places.append((t, at[t], n))
        at[t] += (n + case["pad"] - 1) // case["pad"] * case["pad"]
    st["flat"] = {t: torch.randn(n, generator=g, device="cuda").mul_(1e-3).to(DTYPE[t]) for t, n in at.items() if n}
    size = torch.exp(0.5 * torch.randn(len(places), generator=g, device="cuda"))
    for i, (t, a, n) in enumerate(places):
        st["flat"][t][a:a + n] *= size[i]
        st["flat"][t][a + n:a + (n + case["pad"] - 1) // case["pad"] * case["pad"]] = 0        # between the tensors
    st["to"] = st["flat"] if case["in_place"] else {t: torch.zeros_like(v) for t, v in st["flat"].items()}
    st["grads"] = [st["flat"][t][a:a + n] for t, a, n in places]
    st["results"] = [st["to"][t][a:a + n] for t, a, n in places]
    # far below or far above the norm that such gradients have
    st["max_norm"] = 1e-3 * math.sqrt(sum(n for _, _, n in places)) * (0.1 if case["clipped"] else 300.0)
    st["norm"] = torch.zeros(2, device="cuda")


def _packed(g, matrices, rows, cols):
    """Random E2M1 matrices in the layout of the packed tiles: 16 rows x 128 columns, 1024 bytes of codes, 64 of scales."""
    shape = (matrices, (rows + 15) // 16, (cols + 127) // 128)
    code = torch.randint(0, 256, (*shape, 16, 64), generator=g, device="cuda", dtype=torch.uint8)
    byte = torch.randint(116, 121, (*shape, 16, 4), generator=g, device="cuda", dtype=torch.uint8)
    inside_r = (torch.arange(shape[1] * 16, device="cuda") < rows).reshape(-1, 1, 16, 1)
    inside_c = (torch.arange(shape[2] * 4, device="cuda") * 32 < cols).reshape(1, -1, 1, 4)
    inside = inside_r & inside_c
    code *= inside.repeat_interleave(16, dim=3)
    byte *= inside
    # [half, row % 8, quarter of a group, group] words of eight codes, then [row, group] scale bytes
    code = code.reshape(*shape, 2, 8, 4, 4, 4).permute(0, 1, 2, 3, 4, 6, 5, 7).reshape(*shape, 1024)
    return torch.cat([code, byte.reshape(*shape, 64)], dim=3).contiguous()


def _prepare_moe(case, st, g):
    n, e, h, f = case["tokens"], case["experts"], case["cols"], case["inner"]
    st["x"] = torch.randn(n, h, generator=g, device="cuda").to(torch.bfloat16)
    popularity = 0.5 * torch.randn(e, generator=g, device="cuda")
    logits = torch.randn(n, e, generator=g, device="cuda") + popularity
    # rows of the batch that hold no token: nothing may be chosen there
    st["logits"] = logits.masked_fill(torch.rand(n, 1, generator=g, device="cuda") < case["masked"], -math.inf)
    st["gate_up"] = _packed(g, e, 2 * f, h)
    st["down"] = _packed(g, e, h, f)
    st["y"] = torch.zeros(n, h, dtype=DTYPE[case["out"]], device="cuda")
    st["ids"] = torch.zeros(n, case["top_k"], dtype=torch.int32, device="cuda")
    st["weights"] = torch.zeros(n, case["top_k"], device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case=case)
    if case["op"] == "clip":
        _prepare_clip(case, st, g)
    elif case["op"] == "moe":
        _prepare_moe(case, st, g)
    else:
        _prepare_seam(case, st, g)
    return st


# ----------------------------------------------------------------------------- plain forms

def _rstd(v):
    return torch.rsqrt(v.square().mean(dim=1, keepdim=True) + EPS)


def _gate_rows(st, v):
    """The gate's row for every row of the stream."""
    return v if v is None or v.shape[0] == 1 else v.repeat_interleave(st["rows_per_gate"], dim=0)[:st["case"]["rows"]]


def _plain_stream(st):
    """The stream behind the block, in its type, and the two norms' statistics."""
    n, rp = st["y"].float(), None
    if st["gamma_post"] is not None:
        rp = _rstd(n)
        n = n * rp * st["gamma_post"].float()
    if st["gate"] is not None:
        n = n * _gate_rows(st, st["gate"]).float()
    h = (st["residual_scale"] * st["h_in"].float() + st["branch_scale"] * n).to(st["h_in"].dtype)
    return h, rp, _rstd(h.float())


def _swizzle(s):
    """[mn, blocks] scale bytes in atoms of 128 x 4: byte (mn % 32) * 16 + (mn % 128) / 32 * 4 + block % 4 of each."""
    mn, nb = s.shape
    s = torch.nn.functional.pad(s, (0, -nb % 4, 0, -mn % 128))
    return s.reshape(s.shape[0] // 128, 4, 32, s.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1)


def _plain_quantize(y, axis):
    """E4M3 codes and scales (rounded up to a power of two), 32 values along `axis` to a block."""
    blocks = y.unflatten(axis, (-1, 32))
    bits = blocks.abs().amax(dim=axis + 1).view(torch.int32)
    byte = torch.where(bits >> 23 == 0, 0, (bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(min=0)
    inverse = ((254 - byte) << 23).view(torch.float32)
    q = (blocks * inverse.unsqueeze(axis + 1)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).reshape(y.shape)
    byte = byte.to(torch.uint8)
    return q, _swizzle(byte if axis == 1 else byte.t()).view(torch.float8_e8m0fnu)


def _plain_boundary(st):
    h, rp, rn = _plain_stream(st)
    x = h.float() * rn * st["gamma_pre"].float()
    out = dict(h=h, rstd_pre=rn.reshape(-1))
    if rp is not None:
        out["rstd_post"] = rp.reshape(-1)
    if st["case"]["out"] == "x":
        out["x"] = x.to(DTYPE[st["case"]["block"]])
        return out
    x = x.to(h.dtype).float()                 # the conversion reads a tensor of the stream's type
    out["q_row"], out["s_row"] = _plain_quantize(x, 1)
    if st["case"]["out"] == "both":
        out["q_col"], out["s_col"] = _plain_quantize(x, 0)
    return out


def _per_gate(st, v):
    """Sums of v's rows that share a row of the gate."""
    gates, rows = st["gate"].shape[0], v.shape[0]
    v = torch.nn.functional.pad(v, (0, 0, 0, gates * st["rows_per_gate"] - rows))
    return v.reshape(gates, st["rows_per_gate"], -1).sum(dim=1)


def _plain_gradient(st):
    rn = st["rstd_pre"].unsqueeze(1)
    dx, hat = st["dx"].float(), st["h"].float() * rn
    t = dx * st["gamma_pre"].float()
    grad = st["dh"].float() + rn * (t - hat * (t * hat).mean(dim=1, keepdim=True))
    out = dict(dh_in=(st["residual_scale"] * grad).to(st["h"].dtype), d_gamma_pre=(dx * hat).sum(dim=0))
    branch = st["branch_scale"] * grad
    n = st["y"].float()
    if st["gamma_post"] is not None:
        rp, gamma = st["rstd_post"].unsqueeze(1), st["gamma_post"].float()
        yhat = n * rp
        n = yhat * gamma
    if st["gate"] is not None:
        out["d_gate"] = _per_gate(st, branch * n)
        branch = branch * _gate_rows(st, st["gate"]).float()
    if st["gamma_post"] is not None:
        out["d_gamma_post"] = (branch * yhat).sum(dim=0)
        u = branch * gamma
        branch = rp * (u - yhat * (u * yhat).mean(dim=1, keepdim=True))
    out["dy"] = branch.to(st["y"].dtype)
    return out


def _plain_clip(st):
    norm = torch.stack([v.float().square().sum() for v in st["flat"].values()]).sum().sqrt()
    factor = (st["max_norm"] / (norm + NORM_EPS)).clamp(max=1.0)
    factor = torch.where(torch.isfinite(norm), factor, torch.ones_like(factor))
    return dict(norm=torch.stack([norm, factor]), **{t: (v.float() * factor).to(v.dtype) for t, v in st["flat"].items()})


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


def _plain_choice(st):
    """Experts of every token (-1 where none is left) and their weights."""
    logits = st["logits"]
    top, ids = torch.sort(logits, dim=1, descending=True, stable=True)          # equal logits: the lowest expert first
    top, ids = top[:, :st["case"]["top_k"]], ids[:, :st["case"]["top_k"]]
    live = top > -math.inf
    first = torch.where(live[:, :1], top[:, :1], torch.zeros_like(top[:, :1]))
    e = torch.exp(top - first) * live
    total = e.sum(dim=1, keepdim=True) if st["case"]["renormalize"] else torch.exp(logits - first).sum(dim=1, keepdim=True)
    return torch.where(live, ids, -1).to(torch.int32), torch.where(live, e / total, torch.zeros_like(e))


def _plain_moe(st):
    case = st["case"]
    n, h, f = case["tokens"], case["cols"], case["inner"]
    ids, weights = _plain_choice(st)
    used, at = torch.unique(ids.long().clamp(min=0), return_inverse=True)       # each chosen expert is decoded once
    share = torch.zeros(n, used.numel(), device=ids.device).scatter_add_(1, at, weights)
    a = torch.matmul(st["x"].float(), _decoded(st["gate_up"][used], 2 * f, h).transpose(1, 2))
    m = a[..., :f] * torch.sigmoid(a[..., :f]) * a[..., f:]
    y = torch.bmm(m, _decoded(st["down"][used], h, f).transpose(1, 2))
    return dict(y=(y * share.t().unsqueeze(2)).sum(dim=0).to(DTYPE[case["out"]]), ids=ids, weights=weights)


def run(state):
    if own:
        return _own(state)
    return {"boundary": _plain_boundary, "gradient": _plain_gradient, "clip": _plain_clip, "moe": _plain_moe}[state["case"]["op"]](state)


def _own(st):
    """The calls that a user makes of the library."""
    from paper_2506_08027_b200 import binding as B
    case = st["case"]
    if case["op"] == "moe":
        B.mxfp8_e2m1_moe(st["x"], st["logits"], case["top_k"], st["gate_up"], st["down"], case["inner"], B.ACT_SILU, case["renormalize"], st["y"],
                         st["ids"], st["weights"], _once(st, "ws", lambda: torch.empty(B.mxfp8_e2m1_moe_ws_bytes(case["tokens"], case["top_k"], case["inner"]),
                                                                                       dtype=torch.uint8, device="cuda")))
        return dict(y=st["y"], ids=st["ids"], weights=st["weights"])
    if case["op"] == "clip":
        items = _once(st, "items", lambda: B.make_grad_items(st["grads"], st["results"]))
        ws = _once(st, "ws", lambda: torch.empty(B.mxfp8_grad_ws_bytes(items), dtype=torch.uint8, device="cuda"))
        B.mxfp8_grad_clip(items, st["max_norm"], st["norm"], ws)
        return dict(norm=st["norm"], **st["to"])
    seam = _once(st, "seam", lambda: B.make_seam(st["gamma_pre"], st["gamma_post"], st["gate"], st["rows_per_gate"], st["branch_scale"], st["residual_scale"], EPS))
    if case["op"] == "gradient":
        ws = _once(st, "ws", lambda: torch.empty(B.mxfp8_residual_rmsnorm_grad_ws_bytes(seam, case["rows"], case["cols"]), dtype=torch.uint8, device="cuda"))
        B.mxfp8_residual_rmsnorm_grad(seam, st["dx"], st["dh"], st["y"], st["h"], st["rstd_post"], st["rstd_pre"], st["dy"], st["dh_in"],
                                      st["d_gamma_pre"], st["d_gamma_post"], st["d_gate"], ws)
        return {k: st[k] for k in ("dy", "dh_in", "d_gamma_pre", "d_gamma_post", "d_gate") if st[k] is not None}
    out = dict(h=st["h"], rstd_pre=st["rstd_pre"])
    if case["post"]:
        out["rstd_post"] = st["rstd_post"]
    if case["out"] == "x":
        B.mxfp8_residual_rmsnorm(seam, st["y"], st["h_in"], st["h"], st["x"], st["rstd_post"], st["rstd_pre"])
        return dict(out, x=st["x"])
    B.mxfp8_residual_rmsnorm_quantize(seam, st["y"], st["h_in"], st["h"], st["rstd_post"], st["rstd_pre"], BOTH if case["out"] == "both" else ROW,
                                      B.RULE_PAPER, B.E4M3, st["q_row"], st["s_row"], st["q_col"], st["s_col"], B.SF_SWIZZLED)
    for name in ("row", "col") if case["out"] == "both" else ("row",):
        out["q_" + name], out["s_" + name] = st["q_" + name].view(torch.float8_e4m3fn), st["s_" + name].view(torch.float8_e8m0fnu)
    return out


def _once(st, name, make):
    """What a program makes once for its buffers and keeps beside them."""
    if name not in st:
        st[name] = make()
    return st[name]


# ------------------------------------------------------------------------------ in 64 bits

def _two(n):
    """2^n for whole numbers n of an ordinary exponent."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _exact_codes(v, axis):
    """Values of the E4M3 codes of v, 32 along `axis` to a block, scales ceil(log2(peak / 448))."""
    shape, blocks = v.shape, v.unflatten(axis, (-1, 32))
    peak = blocks.abs().amax(dim=axis + 1, keepdim=True)
    fraction, e = torch.frexp(peak / 448.0)
    exponent = torch.where(fraction == 0.5, e - 1, e)
    exponent = torch.where(peak == 0, torch.full_like(exponent, -127), exponent).clamp(-127, 127)
    v = blocks * _two(-exponent)
    _, e = torch.frexp(v)
    step = _two((e - 1).clamp(min=-6) - 3)
    return (torch.round(v / step) * step).clamp(-448.0, 448.0).reshape(shape)


def _gate_of(st):
    """One row of the gate per row of the stream, in 64 bits; ones without a gate."""
    r, c = st["case"]["rows"], st["case"]["cols"]
    if st["gate"] is None:
        return torch.ones(1, c, dtype=torch.float64, device="cuda")
    return st["gate"].double()[torch.arange(r, device="cuda") // st["rows_per_gate"]]


def _exact_boundary(st):
    y, out, c = st["y"].double(), {}, st["case"]["cols"]
    if st["gamma_post"] is not None:
        mean_square = torch.einsum("rc,rc->r", y, y) / c
        out["rstd_post"] = (mean_square + EPS) ** -0.5
        y = torch.einsum("rc,r,c->rc", y, out["rstd_post"], st["gamma_post"].double())
    h = torch.addcmul(st["residual_scale"] * st["h_in"].double(), y, _gate_of(st), value=st["branch_scale"])
    out["h"] = h
    h = h.to(st["h_in"].dtype).double()             # the norm reads the stream as it is stored
    out["rstd_pre"] = (torch.einsum("rc,rc->r", h, h) / c + EPS) ** -0.5
    x = torch.einsum("rc,r,c->rc", h, out["rstd_pre"], st["gamma_pre"].double())
    if st["case"]["out"] == "x":
        return dict(out, x=x)
    x = x.to(st["h_in"].dtype).double()
    out["q_row"], out["s_row"] = _exact_codes(x, 1), None
    if st["case"]["out"] == "both":
        out["q_col"], out["s_col"] = _exact_codes(x, 0), None
    return out


def _exact_gradient(st):
    """Through autograd of the forward formula in 64 bits, with the saved statistics' definitions in place."""
    leaf = {k: st[k].double().requires_grad_() for k in ("y", "gamma_pre", "gamma_post", "gate") if st[k] is not None}
    h = st["h"].double().requires_grad_()
    c = st["case"]["cols"]

    def normalised(v, gamma):
        return v / torch.sqrt(torch.linalg.vector_norm(v, dim=1, keepdim=True) ** 2 / c + EPS) * gamma

    # the norm before the next block: gradient of the stored stream
    torch.autograd.backward([normalised(h, leaf["gamma_pre"])], [st["dx"].double()])
    total = st["dh"].double() + h.grad
    n = normalised(leaf["y"], leaf["gamma_post"]) if "gamma_post" in leaf else leaf["y"]
    if "gate" in leaf:
        n = n * leaf["gate"][torch.arange(st["case"]["rows"], device="cuda") // st["rows_per_gate"]]
    torch.autograd.backward([st["branch_scale"] * n], [total])
    out = dict(dh_in=st["residual_scale"] * total, dy=leaf["y"].grad, d_gamma_pre=leaf["gamma_pre"].grad)
    for k in ("gamma_post", "gate"):
        if k in leaf:
            out["d_" + k] = leaf[k].grad
    return out


def _exact_clip(st):
    square = sum(torch.dot(p, p) for g in st["grads"] for p in (q.double() for q in g.split(1 << 24)))
    norm = float(square) ** 0.5
    factor = min(1.0, st["max_norm"] / (norm + NORM_EPS))
    return dict(norm=torch.tensor([norm, factor], dtype=torch.float64, device="cuda"), **{t: v.double() * factor for t, v in st["flat"].items()})


E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)       # by the three value bits


def _exact_matrix(flat, rows, cols):
    """One matrix of packed tiles, every element looked up at its place."""
    table = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
    row, col = torch.arange(rows, device="cuda").unsqueeze(1), torch.arange(cols, device="cuda").unsqueeze(0)
    tile = ((row // 16) * ((cols + 127) // 128) + col // 128) * 1088
    word = (tile + row % 16 // 8 * 512 + row % 8 * 64 + col % 32 // 8 * 16 + col % 128 // 32 * 4) // 4
    pair, high = col % 8 // 2, 16 * (col % 2)
    bits = flat.view(torch.int32)[word].long()
    value = table[(bits >> (torch.tensor(VALUE_BITS, device="cuda")[pair] + high)) & 7]
    sign = (bits >> (torch.tensor(SIGN_BIT, device="cuda")[pair] + high)) & 1
    del bits, word
    return value * (1 - 2 * sign) * _two(flat[tile + 1024 + row % 16 * 4 + col % 128 // 32].int() - 127)


def _exact_moe(st):
    case = st["case"]
    n, k, h, f = case["tokens"], case["top_k"], case["cols"], case["inner"]
    logits = st["logits"].double().tolist()
    weights = torch.zeros(n, k, dtype=torch.float64)
    pairs = {}
    for t, row in enumerate(logits):
        order = [e for e in sorted(range(len(row)), key=lambda e: (-row[e], e)) if row[e] > -math.inf][:k]
        top = max(row)
        total = sum(math.exp(row[e] - top) for e in (order if case["renormalize"] else range(len(row)))) if order else 1.0
        for j, e in enumerate(order):
            weights[t, j] = math.exp(row[e] - top) / total
            pairs.setdefault(e, []).append((t, j))
    y = torch.zeros(n, h, dtype=torch.float64, device="cuda")
    weights = weights.cuda()
    gate_up, down = st["gate_up"].reshape(case["experts"], -1), st["down"].reshape(case["experts"], -1)
    for e, chosen in pairs.items():
        t = torch.tensor([p[0] for p in chosen], device="cuda")
        j = torch.tensor([p[1] for p in chosen], device="cuda")
        a = st["x"].double()[t] @ _exact_matrix(gate_up[e], 2 * f, h).t()
        m = a[:, :f] / (1 + torch.exp(-a[:, :f])) * a[:, f:]
        y.index_add_(0, t, weights[t, j].unsqueeze(1) * (m @ _exact_matrix(down[e], h, f).t()))
    return dict(y=y, ids=None, weights=weights)


def exact(case, seed):
    st = prepare(case, seed)
    return {"boundary": _exact_boundary, "gradient": _exact_gradient, "clip": _exact_clip, "moe": _exact_moe}[case["op"]](st)
