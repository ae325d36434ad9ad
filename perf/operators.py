"""Operators on block-scaled 8-bit activations, as cases that can be timed: each is ONE pass through one operator.

A case is a dict of plain values; ``op`` names the operator and the rest its sizes and options:

* ``store``     a tensor into block-scaled 8 bits (an activation checkpoint, or the input of a quantized product)
* ``load``      the way back
* ``norm``      residual addition + root-mean-square norm, output in 8 bits; in training also the checkpoint of the sum and the
                reciprocal root mean squares that the backward pass reads
* ``norm_bwd``  gradient of the norm from the 8-bit checkpoint: of its input (with the residual path's gradient added) and of its weight
* ``swiglu``    gated activation silu(gate) * up, output in 8 bits; in training also the checkpoints of gate and up
* ``swiglu_bwd`` gradient of the gated activation from the two 8-bit checkpoints

A row of ``cols`` elements is cut into blocks of ``block`` (the last one may be short).  A block's scale is the smallest power of two,
from 2^-127, that maps its largest magnitude to at most the largest element value; elements are rounded to nearest even.
8-bit results are returned as float8 tensors and their scales as powers of two (float8_e8m0fnu): views of the bytes that are held.
"""
import torch

own = False

E8 = {"e4m3": (torch.float8_e4m3fn, 448.0), "e5m2": (torch.float8_e5m2, 57344.0)}
FLOAT = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-5


def listed():
    return [
        # a decoding step's activations in front of a quantized product
        {"name": "store_few_tokens", "op": "store", "rows": 4, "cols": 4096, "dtype": "bf16", "elem": "e4m3", "block": 32, "pad": 0},
        # the activation-shaped tensor of the benchmark configurations (8192 tokens, 1 % outlier channels)
        {"name": "store_activations", "op": "store", "rows": 8192, "cols": 4096, "dtype": "bf16", "elem": "e4m3", "block": 32, "pad": 0},
        # the checkpoint of an MLP's inner activations read back in the backward pass
        {"name": "load_activations", "op": "load", "rows": 8192, "cols": 14336, "dtype": "bf16", "elem": "e5m2", "block": 32, "pad": 0},
        # one new token
        {"name": "norm_one_token", "op": "norm", "rows": 1, "cols": 4096, "dtype": "bf16", "elem": "e4m3", "block": 32, "pad": 0, "residual": True, "keep": False},
        # a training step's norm, 8192 tokens
        {"name": "norm_train", "op": "norm", "rows": 8192, "cols": 4096, "dtype": "bf16", "elem": "e4m3", "block": 32, "pad": 0, "residual": True, "keep": True},
        # rows that no vector width divides, in fp32, the first norm of a model (nothing to add)
        {"name": "norm_ragged_f32", "op": "norm", "rows": 1021, "cols": 2501, "dtype": "f32", "elem": "e4m3", "block": 16, "pad": 0, "residual": False, "keep": True},
        {"name": "norm_bwd_train", "op": "norm_bwd", "rows": 8192, "cols": 4096, "dtype": "bf16", "elem": "e4m3", "block": 32, "pad": 0, "residual": True},
        # a short fp32 batch; the last norm of a model (no gradient beside it)
        {"name": "norm_bwd_short_f32", "op": "norm_bwd", "rows": 200, "cols": 1024, "dtype": "f32", "elem": "e4m3", "block": 16, "pad": 0, "residual": False},
        # a serving batch: gate and up are the halves of one product's result
        {"name": "swiglu_serve", "op": "swiglu", "rows": 16, "cols": 14336, "dtype": "bf16", "elem": "e4m3", "block": 32, "halves": True, "keep": False},
        {"name": "swiglu_train", "op": "swiglu", "rows": 8192, "cols": 14336, "dtype": "bf16", "elem": "e4m3", "block": 32, "halves": True, "keep": True},
        {"name": "swiglu_bwd_train", "op": "swiglu_bwd", "rows": 8192, "cols": 14336, "dtype": "bf16", "elem": "e4m3", "block": 32, "halves": True},
        # an inner width that neither a vector nor a block divides
        {"name": "swiglu_bwd_ragged", "op": "swiglu_bwd", "rows": 333, "cols": 2730, "dtype": "bf16", "elem": "e5m2", "block": 64, "halves": False},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["store", "load", "norm", "norm_bwd", "swiglu", "swiglu_bwd"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    wide = op.startswith("swiglu") or op == "load"
    cols = _spread(rng, 64, 16384)
    step = rng.choice([32, 32, 8, 8, 2, 1])   # mostly widths of models, some odd ones
    cols = max(step, cols // step * step)
    most = (8192 * 14336 if wide else 8192 * 4096) * 2 // SIZE[dtype]
    rows = _spread(rng, 1, max(1, min(16384, most // cols)))
    case = {"op": op, "rows": rows, "cols": cols, "dtype": dtype, "elem": rng.choice(["e4m3", "e4m3", "e5m2"]), "block": rng.choice([16, 32, 32, 64, 128])}
    if op in ("swiglu", "swiglu_bwd"):
        case["halves"] = rng.random() < 0.7
    else:
        case["pad"] = rng.choice([0, 0, 0, 8, 64])   # elements between the rows: a slice of a wider tensor
    if op in ("norm", "norm_bwd"):
        case["residual"] = rng.random() < 0.8
    if op in ("norm", "swiglu"):
        case["keep"] = rng.random() < 0.6
    return case


# ---- inputs --------------------------------------------------------------------------------------
def _activations(g, rows, cols, dtype, pad=0, gain=1.0):
    """N(0,1) rows, 1 % of the channels times 50, in rows of cols + pad."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    k = max(1, round(0.01 * cols))
    x[:, torch.randperm(cols, generator=g, device="cuda")[:k]] *= 50.0
    return _padded(x.mul_(gain), dtype, pad)


def _padded(x, dtype, pad):
    rows, cols = x.shape
    out = torch.zeros(rows, cols + pad, device="cuda", dtype=FLOAT[dtype])[:, :cols]
    out.copy_(x)
    return out


def _like(rows, cols, dtype, pad=0):
    return torch.empty(rows, cols + pad, device="cuda", dtype=FLOAT[dtype])[:, :cols]


def _bytes8(rows, cols, block):
    """Room for one 8-bit tensor: its codes and its scale bytes."""
    return (torch.empty(rows, cols, dtype=torch.uint8, device="cuda"), torch.empty(rows, -(-cols // block), dtype=torch.uint8, device="cuda"))


def _held(case, x):
    """x in 8 bits, as bytes."""
    c, s = _to8(x.float(), case)
    return c.view(torch.uint8), s.view(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, rows, cols, dtype, block = (case[k] for k in ("op", "rows", "cols", "dtype", "block"))
    pad = case.get("pad", 0)
    st = {"case": case}
    if op == "store":
        st["x"] = _activations(g, rows, cols, dtype, pad)
        st["out"] = _bytes8(rows, cols, block)
    elif op == "load":
        st["held"] = _held(case, _activations(g, rows, cols, dtype))
        st["out"] = _like(rows, cols, dtype, pad)
    elif op == "norm":
        st["x"] = _activations(g, rows, cols, dtype, pad, 0.25)
        st["residual"] = _activations(g, rows, cols, dtype, pad) if case["residual"] else None
        st["weight"] = (1 + 0.1 * torch.randn(cols, generator=g, device="cuda")).to(FLOAT[dtype])
        st["sum"] = _like(rows, cols, dtype, pad) if case["residual"] else None
        st["out"] = _bytes8(rows, cols, block)
        st["kept"] = _bytes8(rows, cols, block) if case["keep"] else (None, None)
        st["rstd"] = torch.empty(rows, device="cuda") if case["keep"] else None
    elif op == "norm_bwd":
        h = _activations(g, rows, cols, dtype)
        st["held"] = _held(case, h)
        st["rstd"] = h.float().square().mean(1).add(EPS).rsqrt()
        st["weight"] = (1 + 0.1 * torch.randn(cols, generator=g, device="cuda")).to(FLOAT[dtype])
        st["dy"] = _padded(torch.randn(rows, cols, generator=g, device="cuda") * 1e-3, dtype, pad)
        st["dsum"] = _padded(torch.randn(rows, cols, generator=g, device="cuda") * 1e-3, dtype, pad) if case["residual"] else None
        st["dx"] = _like(rows, cols, dtype, pad)
        st["dweight"] = torch.empty(cols, device="cuda")
        # one row of partial sums for each of at most 1024 groups of rows
        st["workspace"] = torch.empty(min(rows, 1024) * cols, device="cuda")
    else:
        if op == "swiglu":
            both = torch.randn(rows, 2 * cols, generator=g, device="cuda").mul_(2.0).to(FLOAT[dtype])
            st["gate"], st["up"] = (both[:, :cols], both[:, cols:]) if case["halves"] else (both[:, :cols].contiguous(), both[:, cols:].contiguous())
            st["out"] = _bytes8(rows, cols, block)
            st["kept"] = _bytes8(rows, cols, block) + _bytes8(rows, cols, block) if case["keep"] else (None,) * 4
        else:
            st["gate"] = _held(case, (torch.randn(rows, cols, generator=g, device="cuda") * 2.0).to(FLOAT[dtype]))
            st["up"] = _held(case, (torch.randn(rows, cols, generator=g, device="cuda") * 2.0).to(FLOAT[dtype]))
            st["dy"] = _padded(torch.randn(rows, cols, generator=g, device="cuda") * 1e-3, dtype, 0)
            both = _like(rows, 2 * cols, dtype)
            st["dgate"], st["dup"] = (both[:, :cols], both[:, cols:]) if case["halves"] else (_like(rows, cols, dtype), _like(rows, cols, dtype))
    return st


# ---- the plain forms -----------------------------------------------------------------------------
def _blocks(x, block):
    """rows x cols as rows x blocks x block, with zeros behind the end of a row."""
    rows, cols = x.shape
    nb = -(-cols // block)
    if nb * block != cols:
        x = torch.nn.functional.pad(x, (0, nb * block - cols))
    return x.view(rows, nb, block)


def _to8(v, case):
    """fp32 values in block-scaled 8 bits: (float8 codes, float8_e8m0fnu scales)."""
    kind, top = E8[case["elem"]]
    b = _blocks(v, case["block"])
    m, e = torch.frexp(b.abs().amax(2))                 # amax = m 2^e, 1/2 <= m < 1; top = 7/8 2^t
    t = 9 if case["elem"] == "e4m3" else 16
    byte = torch.where(m == 0, 0, (e - t + (m > 0.875) + 127).clamp_(min=0))
    scale = torch.where(byte == 0, 0x00400000, byte << 23).to(torch.int32).view(torch.float32)
    codes = (b / scale.unsqueeze(2)).to(kind).view(v.shape[0], -1)[:, : v.shape[1]].contiguous()
    return codes, byte.to(torch.uint8).view(torch.float8_e8m0fnu)


def _from8(held, case):
    """The fp32 values that 8-bit codes and their scales stand for."""
    codes, scales = held
    kind, _ = E8[case["elem"]]
    v = _blocks(codes.view(kind).float(), case["block"]) * scales.view(torch.float8_e8m0fnu).float().unsqueeze(2)
    return v.view(codes.shape[0], -1)[:, : codes.shape[1]]


def _views(case, held):
    return held[0].view(E8[case["elem"]][0]), held[1].view(torch.float8_e8m0fnu)


def run(st):
    case = st["case"]
    if own:
        return _run_own(st)
    op, dtype = case["op"], FLOAT[case["dtype"]]
    if op == "store":
        return {"held": _to8(st["x"].float(), case)}
    if op == "load":
        return {"x": _from8(st["held"], case).to(dtype)}
    if op == "norm":
        x = st["x"].float()
        out = {}
        if case["residual"]:
            out["sum"] = (x + st["residual"].float()).to(dtype)
            x = out["sum"].float()
        rstd = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
        out["held"] = _to8(x * rstd.unsqueeze(1) * st["weight"].float(), case)
        if case["keep"]:
            out["kept"], out["rstd"] = _to8(x, case), rstd
        return out
    if op == "norm_bwd":
        xh = _from8(st["held"], case) * st["rstd"].unsqueeze(1)
        dy = st["dy"].float()
        wd = dy * st["weight"].float()
        dx = (wd - xh * (wd * xh).mean(1, keepdim=True)) * st["rstd"].unsqueeze(1)
        if case["residual"]:
            dx = dx + st["dsum"].float()
        return {"dx": dx.to(dtype), "dweight": (dy * xh).sum(0)}
    if op == "swiglu":
        g, u = st["gate"].float(), st["up"].float()
        out = {"held": _to8(g / (1.0 + torch.exp(-g)) * u, case)}
        if case["keep"]:
            out["gate"], out["up"] = _to8(g, case), _to8(u, case)
        return out
    g, u, dy = _from8(st["gate"], case), _from8(st["up"], case), st["dy"].float()
    s = 1.0 / (1.0 + torch.exp(-g))
    return {"dgate": (dy * u * s * (1.0 + g * (1.0 - s))).to(dtype), "dup": (dy * g * s).to(dtype)}


# ---- the framework's calls -----------------------------------------------------------------------
def _run_own(st):
    from paper_2605_08565_b200 import binding as mxq
    case = st["case"]
    op, block = case["op"], case["block"]
    elem = mxq.MXQ_E4M3 if case["elem"] == "e4m3" else mxq.MXQ_E5M2
    if op == "store":
        mxq.mxq_quantize8(st["x"], block, elem, *st["out"])
        return {"held": _views(case, st["out"])}
    if op == "load":
        mxq.mxq_dequantize8(*st["held"], block, elem, st["out"])
        return {"x": st["out"]}
    if op == "norm":
        mxq.mxq_add_rmsnorm8(st["x"], st["residual"], st["weight"], EPS, block, elem, st["sum"], *st["out"], *st["kept"], st["rstd"])
        out = {"held": _views(case, st["out"])}
        if case["residual"]:
            out["sum"] = st["sum"]
        if case["keep"]:
            out["kept"], out["rstd"] = _views(case, st["kept"]), st["rstd"]
        return out
    if op == "norm_bwd":
        mxq.mxq_add_rmsnorm8_backward(st["dy"], st["dsum"], st["weight"], *st["held"], st["rstd"], block, elem, st["dx"], st["dweight"], st["workspace"])
        return {"dx": st["dx"], "dweight": st["dweight"]}
    if op == "swiglu":
        mxq.mxq_swiglu8(st["gate"], st["up"], block, elem, *st["out"], *st["kept"])
        out = {"held": _views(case, st["out"])}
        if case["keep"]:
            out["gate"], out["up"] = _views(case, st["kept"][:2]), _views(case, st["kept"][2:])
        return out
    mxq.mxq_swiglu8_backward(st["dy"], *st["gate"], *st["up"], block, elem, st["dgate"], st["dup"])
    return {"dgate": st["dgate"], "dup": st["dup"]}


# ---- what a pass cannot do without ---------------------------------------------------------------
def work(case):
    op, rows, cols, size = case["op"], case["rows"], case["cols"], SIZE[case["dtype"]]
    wide = rows * cols * size                                       # a tensor as it is computed with
    held = rows * cols + rows * -(-cols // case["block"])           # the same in 8 bits
    n = rows * cols
    if op in ("store", "load"):
        return {"bytes": wide + held, "flops": 2 * n}
    if op == "norm":
        return {"bytes": wide * (3 if case["residual"] else 1) + held * (2 if case["keep"] else 1) + cols * size + (4 * rows if case["keep"] else 0),
                "flops": 8 * n}
    if op == "norm_bwd":
        return {"bytes": wide * (3 if case["residual"] else 2) + held + cols * (size + 4) + 4 * rows, "flops": 10 * n}
    if op == "swiglu":
        return {"bytes": 2 * wide + held * (3 if case["keep"] else 1), "flops": 8 * n}
    return {"bytes": 3 * wide + 2 * held, "flops": 12 * n}


# ---- the definitions in 64 bits ------------------------------------------------------------------
def _exact8(v, case, known=True):
    """8-bit codes and scales of v.  Where v is the very tensor that is held (`known`) its codes have one right value.  Where v was
    computed on the way, the value before the rounding to 8 bits is given, as for outputs in other types (for e5m2, whose steps are a
    quarter of the value, None)."""
    top, mant, least = (448.0, 3, -6) if case["elem"] == "e4m3" else (57344.0, 2, -14)
    rows, cols = v.shape
    nb = -(-cols // case["block"])
    of = torch.arange(cols, device=v.device) // case["block"]
    amax = torch.zeros(rows, nb, dtype=torch.float64, device=v.device).scatter_reduce_(1, of.expand(rows, cols), v.abs(), "amax")
    scale = torch.exp2(torch.round(torch.log2(amax / top)).clamp(min=-127.0))   # right, or twice or half of it
    scale = torch.where(amax > top * scale, 2 * scale, scale)
    scale = torch.where((2 * amax <= top * scale) & (scale > 2.0 ** -127), scale / 2, scale)
    q = v / scale[:, of]
    if known:
        step = torch.exp2((torch.frexp(q)[1].double() - 1).clamp(min=least) - mant)
        q = torch.round(q / step) * step
    return (q if known or case["elem"] == "e4m3" else None), scale


def _exact_held(held, case):
    """8-bit tensors by their definition, from the bits."""
    codes, scales = held
    mant, bias = (3, 7) if case["elem"] == "e4m3" else (2, 15)
    c = codes.long()
    e, m = (c & 127) >> mant, (c & ((1 << mant) - 1)).double() / (1 << mant)
    v = torch.where(e == 0, m * 2.0 ** (1 - bias), (1 + m) * torch.exp2((e - bias).double())) * (1 - 2 * (c >> 7)).double()
    of = torch.arange(codes.shape[1], device=codes.device) // case["block"]
    return v * torch.exp2(scales.double() - 127)[:, of]


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "store":
        return {"held": _exact8(st["x"].double(), case)}
    if op == "load":
        return {"x": _exact_held(st["held"], case)}
    if op == "norm":
        h, out = st["x"].double(), {}
        if case["residual"]:   # the sum is rounded to binary32 and then to the tensors' type, and that is what the norm is of
            h = (h + st["residual"].double()).float().to(FLOAT[case["dtype"]]).double()
            out["sum"] = h
        rstd = (h.square().mean(1) + EPS).pow(-0.5)
        out["held"] = _exact8(h * rstd[:, None] * st["weight"].double(), case, False)
        if case["keep"]:
            out["kept"], out["rstd"] = _exact8(h, case), rstd
        return out
    if op == "norm_bwd":
        rstd, dy, w = st["rstd"].double()[:, None], st["dy"].double(), st["weight"].double()
        xh = _exact_held(st["held"], case) * rstd
        dx = rstd * (dy * w - xh * (dy * w * xh).sum(1, keepdim=True) / case["cols"])
        if case["residual"]:
            dx += st["dsum"].double()
        return {"dx": dx, "dweight": torch.einsum("rc,rc->c", dy, xh)}
    if op == "swiglu":
        g, u = st["gate"].double(), st["up"].double()
        out = {"held": _exact8(g * torch.sigmoid(g) * u, case, False)}
        if case["keep"]:
            out["gate"], out["up"] = _exact8(g, case), _exact8(u, case)
        return out
    g, u, dy = _exact_held(st["gate"], case), _exact_held(st["up"], case), st["dy"].double()
    s = torch.sigmoid(g)
    return {"dgate": dy * u * (s + g * s * (1 - s)), "dup": dy * g * s}
