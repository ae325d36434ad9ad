"""Operators on block-scaled 8-bit activations against their definitions in binary64 (tests/act8_ref.py).

Quantization of a given tensor and de-quantization are exact: byte for byte.  What is computed first is allowed the rounding errors of
its binary32 operations, u = 2^-24 each, counted in the comments below, and half a step of the type that it is stored in."""
import numpy as np
import pytest
import torch

import act8_ref as ref
from act8_ref import U
from paper_2605_08565_b200 import binding as mxq

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
HALF = {t: torch.finfo(t).eps / 2 for t in (BF16, F32)}      # half a step, relative to the value: bf16 has 8 significant bits, 2^-8
GUARD = 0x5B


@pytest.fixture(params=["native", "ctypes"])
def route(request, monkeypatch):
    """Both ways through the binding."""
    mxq.load_library()
    if request.param == "ctypes":
        monkeypatch.setattr(mxq, "_native", mxq._CtypesOnly())


def np64(t):
    return t.detach().double().cpu().numpy()


class Guarded:
    """A tensor inside a buffer whose other bytes have to stay as they are: rows `pad` elements apart, `shift` elements behind a
    16-byte boundary."""

    def __init__(self, rows, cols, dtype, pad=0, shift=0):
        size = torch.empty(0, dtype=dtype).element_size()
        n = rows * (cols + pad)
        self.raw = torch.full(((shift + n) * size + 64,), GUARD, dtype=torch.uint8, device="cuda")
        flat = self.raw[: (shift + n) * size].view(dtype)[shift:]
        self.t = torch.as_strided(flat, (rows, cols), (cols + pad, 1), flat.storage_offset())

    def fill(self, x):
        self.t.copy_(x)
        self.keep = self.raw.clone()
        return self.t

    def untouched(self):
        """After a call that writes every element of .t: the rest holds GUARD."""
        r = self.raw.clone()
        size = self.t.element_size()
        mask = torch.zeros_like(r, dtype=torch.bool)
        off = self.t.storage_offset() * size
        m = torch.as_strided(mask, (self.t.shape[0], self.t.shape[1] * size), (self.t.stride(0) * size, 1), off)
        m.fill_(True)
        return bool((r[~mask] == GUARD).all())


def held_out(rows, cols, B):
    return Guarded(1, rows * cols, torch.uint8), Guarded(1, rows * (-(-cols // B)), torch.uint8)


def mixed(rows, cols, seed, dtype, special=True):
    """Values over the whole range: blocks of zeros, of short mantissas (ties), tiny and huge ones; infinities and NaN in a few places."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-12, 12, (rows, 1)))
    kind = rng.integers(0, 8, (rows, -(-cols // 16))).repeat(16, 1)[:, :cols]
    x[kind == 0] = 0
    x = np.where(kind == 1, np.round(x * 8) / 8, x)
    x = np.where(kind == 2, rng.integers(-448, 449, (rows, cols)) * 2.0 ** -3, x)
    x = np.where(kind == 3, x * 2.0 ** -140, x)
    x = np.where(kind == 4, np.clip(x * 2.0 ** 124, -3.3e38, 3.3e38), x)
    t = torch.from_numpy(x).to(F32).to(dtype)
    t[t == 0] *= torch.where(torch.rand(int((t == 0).sum()), generator=torch.Generator().manual_seed(seed)) < 0.5, 1.0, -1.0).to(dtype)
    if special and cols > 40:
        f = t.view(-1)
        for k, v in enumerate((float("inf"), -float("inf"), float("nan"))):
            f[int(rng.integers(0, f.numel()))] = v
    return t


def check_exact(c, s, x, B, fmt, cols):
    wc, ws = ref.quantize(x, B, fmt)
    rows = x.shape[0]
    assert np.array_equal(s.t.cpu().numpy().reshape(rows, -1), ws)
    assert np.array_equal(c.t.cpu().numpy().reshape(rows, cols), wc)
    assert c.untouched() and s.untouched()


SHAPES = [(1, 1, 0, 0), (1, 16, 0, 0), (3, 40, 0, 0), (5, 129, 0, 0), (2, 4096, 0, 0), (7, 1000, 8, 0), (33, 264, 3, 0), (300, 72, 0, 1), (1, 70001, 0, 0), (513, 8, 0, 8), (9, 132, 4, 0),
          (5, 2052, 0, 4)]


@pytest.mark.parametrize("B", [16, 32, 64, 128])
@pytest.mark.parametrize("fmt", [ref.E4M3, ref.E5M2])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,pad,shift", SHAPES)
def test_quantize8_is_exact(rows, cols, pad, shift, dtype, fmt, B):
    x = Guarded(rows, cols, dtype, pad, shift).fill(mixed(rows, cols, rows + cols + B, dtype))
    c, s = held_out(rows, cols, B)
    mxq.mxq_quantize8(x, B, fmt, c.t, s.t)
    check_exact(c, s, np64(x), B, fmt, cols)


@pytest.mark.parametrize("B", [16, 32, 64, 128])
@pytest.mark.parametrize("fmt", [ref.E4M3, ref.E5M2])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,pad,shift", SHAPES)
def test_dequantize8_is_exact(rows, cols, pad, shift, dtype, fmt, B):
    """Any code under any scale byte, the ones that mean NaN and infinity among them."""
    rng = np.random.default_rng(rows * cols + B)
    codes = rng.integers(0, 256, (rows, cols)).astype(np.uint8)
    nb = -(-cols // B)
    scales = rng.choice([0, 1, 7, 8, 100, 127, 128, 240, 247, 254, 255], (rows, nb)).astype(np.uint8)
    out = Guarded(rows, cols, dtype, pad, shift)
    mxq.mxq_dequantize8(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), B, fmt, out.t)
    with np.errstate(over="ignore"):
        want = torch.from_numpy(ref.dequantize(codes, scales, B, fmt).astype(np.float32)).to(dtype)
    got = out.t.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got, nan=1.0, posinf=float("inf"), neginf=-float("inf")),
                       torch.nan_to_num(want, nan=1.0, posinf=float("inf"), neginf=-float("inf")))
    assert out.untouched()


# Rows of one and of several vectors a thread, of whole and short blocks, on and off the 16-byte grid; more rows than resident CTAs.
NORM_SHAPES = [(1, 1, 0, 0), (1, 4096, 0, 0), (3, 40, 0, 0), (5, 129, 0, 0), (7, 1000, 8, 0), (33, 264, 3, 0), (700, 72, 0, 0), (1300, 520, 0, 1), (3, 5120, 0, 0),
               (2, 8200, 0, 0), (2, 16392, 8, 0), (2, 32768, 0, 0), (2, 16385, 0, 0), (2, 32767, 1, 0), (3, 2052, 0, 0), (2, 6144, 0, 0), (2, 8192, 16, 0), (2, 16384, 0, 0), (2500, 544, 0, 0), (200, 8224, 0, 0)]


def rel_of_norm(cols):
    """y = (h rstd) w against binary64: a thread adds up to 32 squares and 10 partial sums follow, all of one sign, so the sum is off by
    43 u at most (32 fused steps, 10 additions, and the warps' sums are 10 more levels); mean and eps: 2 u.  rstd takes half of that, the
    reciprocal square root is 2 ulp = 4 u off, and two products follow (2 u): below 32 u."""
    return 32 * U


def norm_inputs(rows, cols, pad, shift, dtype, wdtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-6, 7, (rows, 1), generator=g))
    r = torch.randn(rows, cols, generator=g)
    x[:, :: 50] *= 50
    if rows > 2:
        x[1], r[1] = 0, 0                      # a row of nothing
    w = (1 + 0.2 * torch.randn(cols, generator=g)).to(wdtype)
    mk = lambda v: Guarded(rows, cols, dtype, pad, shift).fill(v.to(dtype))  # noqa: E731
    return mk(x), mk(r), w.cuda()


@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("fmt,B", [(ref.E4M3, 32), (ref.E5M2, 128), (ref.E4M3, 16)])
@pytest.mark.parametrize("rows,cols,pad,shift", NORM_SHAPES)
@pytest.mark.parametrize("with_residual", [True, False])
def test_add_rmsnorm8(rows, cols, pad, shift, fmt, B, dtype, wdtype, with_residual):
    eps = 1e-5
    x, r, w = norm_inputs(rows, cols, pad, shift, dtype, wdtype, cols + rows)
    if not with_residual:
        r = None
    total = Guarded(rows, cols, dtype, pad, shift) if with_residual else None
    (c, s), (kc, ks) = held_out(rows, cols, B), held_out(rows, cols, B)
    rstd = Guarded(1, rows, F32)
    mxq.mxq_add_rmsnorm8(x, r, w, eps, B, fmt, total.t if total else None, c.t, s.t, kc.t, ks.t, rstd.t)
    h = np64(x)
    if with_residual:
        want = (x.float() + r.float()).to(dtype)
        assert torch.equal(total.t, want) and total.untouched()
        h = np64(want)
    check_exact(kc, ks, h, B, fmt, cols)
    y, wr = ref.rmsnorm(h, np64(w), np.float64(np.float32(eps)))
    assert (np.abs(np64(rstd.t)[0] - wr) <= 30 * U * wr).all() and rstd.untouched()
    ref.check_held(c.t.cpu().numpy().reshape(rows, cols), s.t.cpu().numpy().reshape(rows, -1), y, rel_of_norm(cols), B, fmt)
    assert c.untouched() and s.untouched()
    # without the checkpoint and rstd: the same output
    c2, s2 = held_out(rows, cols, B)
    mxq.mxq_add_rmsnorm8(x, r, w, eps, B, fmt, total.t if total else None, c2.t, s2.t)
    assert torch.equal(c2.t, c.t) and torch.equal(s2.t, s.t)


def test_norms_of_more_rows_than_the_device_holds():
    """Every CTA comes to several rows of 4096 elements, forward and backward."""
    rows, cols, B = 1000, 4096, 32
    x, r, w = norm_inputs(rows, cols, 0, 0, BF16, BF16, 1)
    total = torch.empty_like(x)
    (c, s), (kc, ks) = held_out(rows, cols, B), held_out(rows, cols, B)
    rstd = torch.empty(rows, device="cuda")
    mxq.mxq_add_rmsnorm8(x, r, w, 1e-5, B, ref.E4M3, total, c.t, s.t, kc.t, ks.t, rstd)
    h = np64(total)
    assert torch.equal(total, (x.float() + r.float()).to(BF16))
    check_exact(kc, ks, h, B, ref.E4M3, cols)
    y = ref.rmsnorm(h, np64(w), np.float64(np.float32(1e-5)))[0]
    ref.check_held(c.t.cpu().numpy().reshape(rows, cols), s.t.cpu().numpy().reshape(rows, -1), y, rel_of_norm(cols), B, ref.E4M3)
    dy = Guarded(rows, cols, BF16).fill((torch.randn(rows, cols, generator=torch.Generator().manual_seed(2)) * 1e-3).to(BF16))
    dx, dw = Guarded(rows, cols, BF16), Guarded(1, cols, F32)
    mxq.mxq_add_rmsnorm8_backward(dy, r, w, kc.t.view(rows, cols), ks.t.view(rows, -1), rstd, B, ref.E4M3, dx.t, dw.t, workspace(rows, cols))
    held = ref.dequantize(kc.t.cpu().numpy().reshape(rows, cols), ks.t.cpu().numpy().reshape(rows, -1), B, ref.E4M3)
    wx, ww, size, wsize = ref.rmsnorm_backward(np64(dy), np64(w), held, np64(rstd), np64(r))
    assert (np.abs(np64(dx.t) - wx) <= HALF[BF16] * np.abs(wx) + 65 * U * size).all()
    assert (np.abs(np64(dw.t)[0] - ww) <= (rows + 3) * U * wsize).all()
    assert dx.untouched() and dw.untouched()


def test_add_rmsnorm8_in_place():
    """The sum may be written over either summand."""
    for over in ("x", "residual"):
        x, r, w = norm_inputs(9, 520, 8, 0, BF16, BF16, 4)
        want = (x.float() + r.float()).to(BF16)
        (c, s), (c2, s2) = held_out(9, 520, 32), held_out(9, 520, 32)
        mxq.mxq_add_rmsnorm8(x, r, w, 1e-5, 32, ref.E4M3, torch.empty_like(want), c.t, s.t)
        out = x if over == "x" else r
        mxq.mxq_add_rmsnorm8(x, r, w, 1e-5, 32, ref.E4M3, out, c2.t, s2.t)
        assert torch.equal(out, want) and torch.equal(c.t, c2.t) and torch.equal(s.t, s2.t)


def test_values_that_are_not_finite_stay_visible():
    """A NaN in a row makes the whole row NaN, an infinity makes it zeros and a NaN block; other rows are not touched by it."""
    x = torch.randn(6, 256, device="cuda").to(BF16)
    y = x.clone()
    y[1, 5], y[3, 200], y[4, 100] = float("nan"), float("inf"), -float("inf")
    w = torch.ones(256, device="cuda", dtype=BF16)
    a, b = held_out(6, 256, 32), held_out(6, 256, 32)
    for v, o in ((x, a), (y, b)):
        mxq.mxq_add_rmsnorm8(v, None, w, 1e-5, 32, ref.E4M3, None, o[0].t, o[1].t)
    ca, cb, sa, sb = (t.t.cpu().numpy().reshape(6, -1) for t in (a[0], b[0], a[1], b[1]))
    for row in (0, 2, 5):
        assert np.array_equal(ca[row], cb[row]) and np.array_equal(sa[row], sb[row])
    assert (sb[1] == 255).all() and (cb[1] == 0x7F).all()
    for row, block in ((3, 6), (4, 3)):
        assert sb[row, block] == 255 and (cb[row, block * 32: block * 32 + 32] == 0x7F).all()
        rest = np.delete(np.arange(8), block)
        assert (sb[row, rest] == 0).all() and ((cb[row].reshape(8, 32)[rest] & 0x7F) == 0).all()


def backward_inputs(rows, cols, pad, shift, dtype, wdtype, fmt, B, seed):
    x, r, w = norm_inputs(rows, cols, pad, shift, dtype, wdtype, seed)
    h = np64(x)
    codes, scales = ref.quantize(h, B, fmt)
    rstd = torch.from_numpy(ref.rmsnorm(h, np64(w), 1e-5)[1]).float().cuda()
    dy = Guarded(rows, cols, dtype, pad, shift).fill((torch.randn(rows, cols, generator=torch.Generator().manual_seed(seed + 1)) * 1e-3).to(dtype))
    return dy, r, w, torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), rstd


def workspace(rows, cols):
    return torch.full((mxq.mxq_add_rmsnorm8_workspace_bytes(rows, cols) // 4,), float("nan"), device="cuda")


@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("fmt,B", [(ref.E4M3, 32), (ref.E5M2, 128), (ref.E4M3, 16)])
@pytest.mark.parametrize("rows,cols,pad,shift", NORM_SHAPES)
@pytest.mark.parametrize("with_dsum", [True, False])
def test_add_rmsnorm8_backward(rows, cols, pad, shift, fmt, B, dtype, wdtype, with_dsum):
    dy, ds, w, codes, scales, rstd = backward_inputs(rows, cols, pad, shift, dtype, wdtype, fmt, B, rows + cols)
    ds = ds if with_dsum else None
    dx, dw = Guarded(rows, cols, dtype, pad, shift), Guarded(1, cols, F32)
    mxq.mxq_add_rmsnorm8_backward(dy, ds, w, codes, scales, rstd, B, fmt, dx.t, dw.t, workspace(rows, cols))
    h = ref.dequantize(codes.cpu().numpy(), scales.cpu().numpy(), B, fmt)
    wx, ww, size, wsize = ref.rmsnorm_backward(np64(dy), np64(w), h, np64(rstd), np64(ds) if with_dsum else None)
    # the dot product of a row: 2 roundings a term, 32 terms of a thread and 10 levels above: 45 u of the terms' sizes, and 8 more steps
    assert (np.abs(np64(dx.t) - wx) <= HALF[dtype] * np.abs(wx) + 65 * U * size).all()
    # at most `rows` additions in some order, and 3 roundings a term
    assert (np.abs(np64(dw.t)[0] - ww) <= (rows + 3) * U * wsize).all()
    assert dx.untouched() and dw.untouched()
    # without the weight's gradient: the same dx, no workspace
    dx2 = Guarded(rows, cols, dtype, pad, shift)
    mxq.mxq_add_rmsnorm8_backward(dy, ds, w, codes, scales, rstd, B, fmt, dx2.t)
    assert torch.equal(dx2.t, dx.t)


def test_add_rmsnorm8_backward_in_place_and_repeatable():
    dy, ds, w, codes, scales, rstd = backward_inputs(1000, 1024, 0, 0, BF16, BF16, ref.E4M3, 32, 8)
    got = []
    for over in (None, None, "dy", "dsum"):
        y, s = dy.clone(), ds.clone()
        out = {None: torch.empty_like(y), "dy": y, "dsum": s}[over]
        dw = torch.empty(1024, device="cuda")
        mxq.mxq_add_rmsnorm8_backward(y, s, w, codes, scales, rstd, 32, ref.E4M3, out, dw, workspace(1000, 1024))
        got.append((out, dw))
    for out, dw in got[1:]:
        assert torch.equal(out, got[0][0]) and torch.equal(dw, got[0][1])


def gated_inputs(rows, cols, dtype, halves, seed, pad=0, shift=0):
    g = torch.Generator().manual_seed(seed)
    both = torch.randn(rows, 2 * cols, generator=g) * 3
    both.view(-1)[:: 37] *= 30                    # sigmoids of 0 and 1
    both = both.to(dtype).cuda()
    if halves:
        return both[:, :cols], both[:, cols:]
    return Guarded(rows, cols, dtype, pad, shift).fill(both[:, :cols]), Guarded(rows, cols, dtype, 2 * pad, shift).fill(both[:, cols:])


GATED_SHAPES = [(1, 1, False, 0, 0), (1, 14336, True, 0, 0), (3, 40, True, 0, 0), (5, 129, True, 0, 0), (7, 1000, False, 8, 0), (33, 264, False, 3, 0), (300, 72, True, 0, 0),
                (65, 2730, False, 0, 0), (9, 2048, False, 0, 1), (9, 132, True, 0, 0), (5, 2052, False, 4, 0)]


def off_of_sigmoid(g, dtype):
    """Relative error of s = 1 / (1 + e), e = exp(-g).  The sum is rounded (1 u) and the reciprocal is off by an ulp (2 u).  e is off by
    2 ulp = 4 u; in bf16 it is 2^t with t = -g log2 e, whose constant is off by less than 0.25 u and whose product by 1 u of |t|: |g| 1.25 u in
    e, which is at most |t| ln 2 = |g| times that.  An error of e counts in s as e / (1 + e) <= 1, which for g > 0 is below exp(-g): there
    |g| exp(-g) <= 0.37."""
    grows = np.where(g < 0, np.abs(g), 0.37) * 1.25 if dtype == BF16 else 0.0
    return (grows + 4 + 3) * U


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt,B", [(ref.E4M3, 32), (ref.E5M2, 128), (ref.E4M3, 64), (ref.E5M2, 16)])
@pytest.mark.parametrize("rows,cols,halves,pad,shift", GATED_SHAPES)
def test_swiglu8(rows, cols, halves, pad, shift, fmt, B, dtype):
    gate, up = gated_inputs(rows, cols, dtype, halves, rows * cols, pad, shift)
    (c, s), (gc, gs), (uc, us) = (held_out(rows, cols, B) for _ in range(3))
    mxq.mxq_swiglu8(gate, up, B, fmt, c.t, s.t, gc.t, gs.t, uc.t, us.t)
    g, u = np64(gate), np64(up)
    check_exact(gc, gs, g, B, fmt, cols)
    check_exact(uc, us, u, B, fmt, cols)
    # the sigmoid, two products 2 u; one u for what is left out here.  A sigmoid below 2^-126 counts as zero.
    ref.check_held(c.t.cpu().numpy().reshape(rows, cols), s.t.cpu().numpy().reshape(rows, -1), ref.swiglu(g, u), off_of_sigmoid(g, dtype) + 3 * U, B, fmt,
                   2.0 ** -126 * np.abs(g * u))
    assert c.untouched() and s.untouched()
    c2, s2 = held_out(rows, cols, B)
    mxq.mxq_swiglu8(gate, up, B, fmt, c2.t, s2.t)
    assert torch.equal(c2.t, c.t) and torch.equal(s2.t, s.t)


def check_gated_gradients(dg, du, d, g, u, dtype):
    """The sigmoid is off_of_sigmoid() off, 1 - s by so much of s and a rounding; three products, a fused one and the slope's sum follow: 6 u of
    each part of dg, 3 u of du.  Below 2^-126 the sigmoid counts as zero."""
    wg, wu = ref.swiglu_backward(d, g, u)
    s = ref.sigmoid(g)
    tiny = 2.0 ** -126 * np.abs(d) * (1 + np.abs(u) * (1 + np.abs(g)) + np.abs(g)) + 2.0 ** -133
    near = off_of_sigmoid(g, dtype)
    off = np.abs(d * u * s) * ((near + 6 * U) * np.abs(1 + g * (1 - s)) + np.abs(g) * (near * s + 2 * U * (1 - s)))
    assert (np.abs(dg - wg) <= HALF[dtype] * np.abs(wg) + (1 + HALF[dtype]) * off + tiny).all()
    assert (np.abs(du - wu) <= (HALF[dtype] + (1 + HALF[dtype]) * (near + 3 * U)) * np.abs(wu) + tiny).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt,B", [(ref.E4M3, 32), (ref.E5M2, 128), (ref.E4M3, 64), (ref.E5M2, 16)])
@pytest.mark.parametrize("rows,cols,halves,pad,shift", GATED_SHAPES)
def test_swiglu8_backward(rows, cols, halves, pad, shift, fmt, B, dtype):
    gate, up = gated_inputs(rows, cols, dtype, False, rows * cols)
    (gc, gs), (uc, us) = ref.quantize(np64(gate), B, fmt), ref.quantize(np64(up), B, fmt)
    dev = [torch.from_numpy(v).cuda() for v in (gc, gs, uc, us)]
    dy = Guarded(rows, cols, dtype, pad, shift).fill((torch.randn(rows, cols, generator=torch.Generator().manual_seed(1)) * 1e-2).to(dtype))
    if halves:
        both = torch.empty(rows, 2 * cols, device="cuda", dtype=dtype)
        dg, du = both[:, :cols], both[:, cols:]
    else:
        o = Guarded(rows, cols, dtype, pad, shift), Guarded(rows, cols, dtype, 2 * pad, shift)
        dg, du = o[0].t, o[1].t
    mxq.mxq_swiglu8_backward(dy, *dev, B, fmt, dg, du)
    g, u, d = ref.dequantize(gc, gs, B, fmt), ref.dequantize(uc, us, B, fmt), np64(dy)
    check_gated_gradients(np64(dg), np64(du), d, g, u, dtype)
    if not halves:
        assert o[0].untouched() and o[1].untouched()
        for k in (0, 1):                          # over dy itself
            y = Guarded(rows, cols, dtype, pad, shift).fill(dy)
            other = torch.empty(rows, cols, device="cuda", dtype=dtype)
            a, b = (y, other) if k == 0 else (other, y)
            mxq.mxq_swiglu8_backward(y, *dev, B, fmt, a, b)
            assert torch.equal(a, dg) and torch.equal(b, du)


def test_both_routes_take_the_same_tensors(route):
    """Leading dimensions, float8 and byte buffers, a slice of a wider tensor, a row on its own; with the extension module and without."""
    for fmt, kind in ((ref.E4M3, torch.float8_e4m3fn), (ref.E5M2, torch.float8_e5m2)):
        x = torch.randn(3, 5, 200, device="cuda").to(BF16)
        c, s = mxq.quantize8(x, 64, fmt)
        assert c.dtype == kind and s.dtype == torch.float8_e8m0fnu and c.shape == (15, 200) and s.shape == (15, 4)
        wc, ws = ref.quantize(np64(x).reshape(15, 200), 64, fmt)
        assert np.array_equal(c.view(torch.uint8).cpu().numpy(), wc) and np.array_equal(s.view(torch.uint8).cpu().numpy(), ws)
        y = torch.empty(3, 5, 256, device="cuda", dtype=F32)[..., :200]
        mxq.mxq_dequantize8(c, s.view(torch.uint8), 64, fmt, y)
        assert np.array_equal(np64(y).reshape(15, 200), ref.dequantize(wc, ws, 64, fmt))
        row = x[1, 2]
        c1, s1 = mxq.quantize8(row, 64, fmt)
        assert np.array_equal(c1.view(torch.uint8).cpu().numpy()[0], wc[7]) and np.array_equal(s1.view(torch.uint8).cpu().numpy()[0], ws[7])


def test_binding_refuses_tensors_that_do_not_fit(route):
    x = torch.zeros(4, 64, device="cuda", dtype=BF16)
    u8 = lambda *n: torch.zeros(*n, device="cuda", dtype=torch.uint8)  # noqa: E731
    c, s, w, f = u8(4, 64), u8(4, 2), torch.ones(64, device="cuda"), torch.ones(4, device="cuda")
    q = lambda x=x, B=32, e=0, c=c, s=s: mxq.mxq_quantize8(x, B, e, c, s)  # noqa: E731
    n = lambda x=x, r=None, w=w, eps=1e-5, o=None, k=None, ks=None, rs=None: mxq.mxq_add_rmsnorm8(x, r, w, eps, 32, 0, o, c, s, k, ks, rs)  # noqa: E731
    q(), n()
    for f_, text in ((lambda: q(x.half()), "unsupported dtype"), (lambda: q(x.t()), "contiguous"), (lambda: q(x[:, ::2]), "contiguous"),
                     (lambda: q(x[:0]), "at least one"), (lambda: q(x[:, :0]), "at least one"), (lambda: q(x[0, 0]), "scalar"), (lambda: q(B=8), "block_size"),
                     (lambda: q(B=16), "expected"), (lambda: q(e=2), "status 2"), (lambda: q(c=u8(4, 63)), "expected"), (lambda: q(c=c.cpu()), "CUDA tensors only"),
                     (lambda: q(c=c.view(torch.float8_e5m2)), "dtype"), (lambda: q(c=c.view(torch.int16)), "dtype"), (lambda: q(s=u8(4, 4)[:, ::2]), "contiguous"),
                     (lambda: q(x[:1].expand(4, 64)), "status 3"), (lambda: q(x.view(2, 2, 64).transpose(0, 1)), "evenly spaced|expected"),
                     (lambda: n(r=x), "status 1"), (lambda: n(r=x.float(), o=x), "bfloat16|float32"), (lambda: n(r=x[:2], o=x), "expected"), (lambda: n(w=w[:32]), "expected"),
                     (lambda: n(w=w.half()), "unsupported dtype"), (lambda: n(eps=0.0), "status 5"), (lambda: n(k=c), "CUDA tensors only|status 1"),
                     (lambda: n(rs=f.double()), "float32"), (lambda: n(rs=f[:3]), "expected"),
                     (lambda: mxq.mxq_add_rmsnorm8_backward(x, None, w, c, s, f, 32, 0, x.clone(), w.clone()), "status 6"),
                     (lambda: mxq.mxq_add_rmsnorm8_backward(x, None, w, c, s, f, 32, 0, x.clone(), w.clone(), w), "status 6"),
                     (lambda: mxq.mxq_swiglu8(x, x.float(), 32, 0, c, s), "bfloat16|float32"), (lambda: mxq.mxq_swiglu8(x, x, 32, 0, c, s, c, s), "status 1"),
                     (lambda: mxq.mxq_swiglu8_backward(x, c, s, c, s, 32, 0, x, x), "status 3")):
        with pytest.raises(mxq.MxqError, match=text):
            f_()


class Block:
    """Norm, up and gate products, gated activation, down product, and their gradients, with the 8-bit tensors between them."""

    def __init__(self, rows, d, inner, B, fmt, seed):
        g = torch.Generator().manual_seed(seed)
        t = lambda *n: (torch.randn(*n, generator=g)).to(BF16).cuda()  # noqa: E731
        self.B, self.fmt = B, fmt
        self.x, self.res, self.w, self.dout = t(rows, d), t(rows, d), 1 + 0.1 * t(d), t(rows, d)
        self.w1, self.w2 = t(d, 2 * inner) / d ** 0.5, t(inner, d) / inner ** 0.5
        e = lambda *n, dtype=BF16: torch.empty(*n, dtype=dtype, device="cuda")  # noqa: E731
        held = lambda c: mxq.alloc_outputs8(rows, c, B, fmt, "cuda")  # noqa: E731
        self.sum, self.y8, self.k8, self.rstd = e(rows, d), held(d), held(d), e(rows, dtype=F32)
        self.y, self.gu, self.a8, self.g8, self.u8, self.a, self.out = e(rows, d), e(rows, 2 * inner), held(inner), held(inner), held(inner), e(rows, inner), e(rows, d)
        self.da, self.dgu, self.dy, self.dx, self.dw = e(rows, inner), e(rows, 2 * inner), e(rows, d), e(rows, d), e(d, dtype=F32)
        self.ws = e(mxq.mxq_add_rmsnorm8_workspace_bytes(rows, d) // 4, dtype=F32)
        self.inner = inner

    def step(self):
        B, f, i = self.B, self.fmt, self.inner
        mxq.mxq_add_rmsnorm8(self.x, self.res, self.w, 1e-5, B, f, self.sum, *self.y8, *self.k8, self.rstd)
        mxq.mxq_dequantize8(*self.y8, B, f, self.y)
        torch.matmul(self.y, self.w1, out=self.gu)
        mxq.mxq_swiglu8(self.gu[:, :i], self.gu[:, i:], B, f, *self.a8, *self.g8, *self.u8)
        mxq.mxq_dequantize8(*self.a8, B, f, self.a)
        torch.matmul(self.a, self.w2, out=self.out)
        torch.matmul(self.dout, self.w2.t(), out=self.da)
        mxq.mxq_swiglu8_backward(self.da, *self.g8, *self.u8, B, f, self.dgu[:, :i], self.dgu[:, i:])
        torch.matmul(self.dgu, self.w1.t(), out=self.dy)
        mxq.mxq_add_rmsnorm8_backward(self.dy, self.dout, self.w, *self.k8, self.rstd, B, f, self.dx, self.dw, self.ws)
        return {k: v.clone() for k, v in (("sum", self.sum), ("y", self.y), ("a", self.a), ("out", self.out), ("dgu", self.dgu), ("dx", self.dx), ("dw", self.dw))}

    def check(self, got):
        """Each operator's result from the tensors that it was given."""
        B, f, i = self.B, self.fmt, self.inner
        n8 = lambda h: (h[0].view(torch.uint8).cpu().numpy(), h[1].view(torch.uint8).cpu().numpy())  # noqa: E731
        h = np64((self.x.float() + self.res.float()).to(BF16))
        assert np.array_equal(np64(got["sum"]), h)
        y, rstd = ref.rmsnorm(h, np64(self.w), 1e-5)
        ref.check_held(*n8(self.y8), y, rel_of_norm(h.shape[1]), B, f)
        assert np.array_equal(np64(got["y"]), ref.dequantize(*n8(self.y8), B, f))
        gu = np64(self.gu)
        ref.check_held(*n8(self.a8), ref.swiglu(gu[:, :i], gu[:, i:]), off_of_sigmoid(gu[:, :i], BF16) + 3 * U, B, f)
        for held, v in ((self.k8, h), (self.g8, gu[:, :i]), (self.u8, gu[:, i:])):
            c, s = ref.quantize(v, B, f)
            assert np.array_equal(n8(held)[0], c) and np.array_equal(n8(held)[1], s)
        dgu = np64(got["dgu"])
        check_gated_gradients(dgu[:, :i], dgu[:, i:], np64(self.da), ref.dequantize(*n8(self.g8), B, f), ref.dequantize(*n8(self.u8), B, f), BF16)
        dx, dw, size, wsize = ref.rmsnorm_backward(np64(self.dy), np64(self.w), ref.dequantize(*n8(self.k8), B, f), np64(self.rstd), np64(self.dout))
        assert (np.abs(np64(got["dx"]) - dx) <= HALF[BF16] * np.abs(dx) + 65 * U * size).all()
        assert (np.abs(np64(got["dw"]) - dw) <= (h.shape[0] + 3) * U * wsize).all()


@pytest.mark.parametrize("rows,d,inner,B,fmt", [(37, 256, 712, 32, ref.E4M3), (130, 512, 1024, 64, ref.E5M2)])
def test_a_block_forward_and_backward(rows, d, inner, B, fmt):
    b = Block(rows, d, inner, B, fmt, 5)
    b.check(b.step())


def test_a_captured_block_replays_with_new_inputs():
    """Captured on a stream of its own, replayed twice with other inputs, beside an eager step of another block with its own workspace."""
    b, other = Block(37, 256, 712, 32, ref.E4M3, 5), Block(37, 256, 712, 32, ref.E4M3, 6)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b.step()                                   # library handles and occupancies
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = b.step()
    for seed in (11, 12):
        n = Block(37, 256, 712, 32, ref.E4M3, seed)
        for k in ("x", "res", "w", "dout", "w1", "w2"):
            getattr(b, k).copy_(getattr(n, k))
        torch.cuda.synchronize()
        graph.replay()
        want_other = other.step()
        torch.cuda.synchronize()
        b.check(got)
        other.check(want_other)


@pytest.mark.parametrize("rows,cols", [(200001, 3), (70000, 16), (9, 4096), (5, 1000)])
@pytest.mark.parametrize("shift", [0, 1, 2, 3])
def test_vectors_and_scales_that_start_anywhere(rows, cols, shift):
    """Scale bytes at any address, weight, rstd, dweight at any element, the workspace at any 16 bytes; many short rows."""
    B, fmt = 32, ref.E4M3
    nb = -(-cols // B)
    x, r, w = norm_inputs(rows, cols, 0, 0, BF16, BF16, 7)
    w = Guarded(1, cols, BF16, 0, shift).fill(w).view(-1)
    u8 = lambda n: torch.full((n + 64,), GUARD, dtype=torch.uint8, device="cuda")  # noqa: E731
    c, kc = u8(rows * cols)[: rows * cols], u8(rows * cols)[: rows * cols]
    sb, kb = u8(rows * nb), u8(rows * nb)
    s, ks = sb[shift: shift + rows * nb], kb[shift: shift + rows * nb]
    total, rstd = torch.empty_like(x), torch.empty(rows + 4, device="cuda")[shift: shift + rows]
    mxq.mxq_add_rmsnorm8(x, r, w, 1e-5, B, fmt, total, c, s, kc, ks, rstd)
    h = np64(total)
    wc, ws = ref.quantize(h, B, fmt)
    assert np.array_equal(kc.cpu().numpy().reshape(rows, cols), wc) and np.array_equal(ks.cpu().numpy().reshape(rows, nb), ws)
    for b in (sb, kb):
        assert bool((b[:shift] == GUARD).all()) and bool((b[shift + rows * nb:] == GUARD).all())
    y, wr = ref.rmsnorm(h, np64(w), np.float64(np.float32(1e-5)))
    ref.check_held(c.cpu().numpy().reshape(rows, cols), s.cpu().numpy().reshape(rows, nb), y, rel_of_norm(cols), B, fmt)
    dy = torch.randn(rows, cols, generator=torch.Generator().manual_seed(3)).to(BF16).cuda()
    dx, dw = torch.empty_like(dy), torch.full((cols + 8,), -1.0, device="cuda")
    space = torch.empty(mxq.mxq_add_rmsnorm8_workspace_bytes(rows, cols) // 4 + 16, device="cuda")[4 * shift:]
    mxq.mxq_add_rmsnorm8_backward(dy, dy, w, kc, ks, rstd, B, fmt, dx, dw[shift: shift + cols], space)
    wx, ww, size, wsize = ref.rmsnorm_backward(np64(dy), np64(w), ref.dequantize(wc, ws, B, fmt), np64(rstd), np64(dy))
    assert (np.abs(np64(dx) - wx) <= HALF[BF16] * np.abs(wx) + 65 * U * size).all()
    assert (np.abs(np64(dw)[shift: shift + cols] - ww) <= (rows + 3) * U * wsize).all()
    assert bool((dw[:shift] == -1).all()) and bool((dw[shift + cols:] == -1).all())
    out = torch.empty_like(dx)
    mxq.mxq_dequantize8(kc, ks, B, fmt, out)
    assert np.array_equal(np64(out), np64(torch.from_numpy(ref.dequantize(wc, ws, B, fmt)).float().to(BF16)))
    # the gradient over both of its inputs at once
    mxq.mxq_add_rmsnorm8_backward(dy, dy, w, kc, ks, rstd, B, fmt, dy)
    assert torch.equal(dy, dx)


def test_first_calls_of_a_process_may_be_captured(tmp_path):
    """What the first call of a kernel asks of the driver (its limits, how many CTAs fit) may be asked while a stream is captured."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2605_08565_b200 import binding as mxq
x = torch.randn(700, 2048, device="cuda").to(torch.bfloat16)
w, rstd = torch.ones(2048, device="cuda"), torch.empty(700, device="cuda")
h, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(2048, device="cuda")
q, k, a = (mxq.alloc_outputs8(700, 2048, 32, mxq.MXQ_E4M3, "cuda") for _ in range(3))
ws = torch.empty(mxq.mxq_add_rmsnorm8_workspace_bytes(700, 2048) // 4, device="cuda")
def step():
    mxq.mxq_add_rmsnorm8(x, x, w, 1e-5, 32, mxq.MXQ_E4M3, h, *q, *k, rstd)
    mxq.mxq_add_rmsnorm8_backward(x, h, w, *k, rstd, 32, mxq.MXQ_E4M3, dx, dw, ws)
    mxq.mxq_swiglu8(x, h, 32, mxq.MXQ_E4M3, *a)
    return [t.clone() for t in (h, dx, dw, q[0].view(torch.uint8), a[0].view(torch.uint8))]
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    got = step()
g.replay()
torch.cuda.synchronize()
want = step()
assert all(torch.equal(a, b) for a, b in zip(got, want))
print("captured")
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


def test_four_host_threads_at_once():
    """Each with its own stream, block and workspace, sixteen steps over: the results of a quiet run."""
    import threading
    blocks = [Block(130, 544, 1024, 32, ref.E4M3, 40 + i) for i in range(4)]
    want = [b.step() for b in blocks]
    torch.cuda.synchronize()
    errors = []

    def worker(b, w):
        try:
            torch.cuda.set_device(0)
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(16):
                    got = b.step()
            torch.cuda.synchronize()
            for k in ("sum", "y", "dx", "dw"):
                if not torch.equal(got[k], w[k]):
                    errors.append(k)
        except Exception as e:   # a thread's exception would be lost
            errors.append(repr(e))

    threads = [threading.Thread(target=worker, args=a) for a in zip(blocks, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors


def test_a_stream_given_explicitly_is_the_one_that_is_used():
    rows, cols = 64, 4096
    src = torch.randn(rows, cols, device="cuda").to(BF16)
    x = torch.zeros_like(src)
    c, s = mxq.alloc_outputs8(rows, cols, 32, ref.E4M3, "cuda")
    back, w = torch.empty_like(src), torch.ones(cols, device="cuda")
    n = mxq.alloc_outputs8(rows, cols, 32, ref.E4M3, "cuda")
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(a):
        torch.cuda._sleep(40_000_000)
        x.copy_(src)
    b.wait_stream(a)
    mxq.mxq_quantize8(x, 32, ref.E4M3, c, s, stream=b)
    mxq.mxq_dequantize8(c, s, 32, ref.E4M3, back, stream=b)
    mxq.mxq_add_rmsnorm8(back, None, w, 1e-5, 32, ref.E4M3, None, *n, stream=b)
    b.synchronize()
    wc, ws = ref.quantize(np64(src), 32, ref.E4M3)
    assert np.array_equal(c.view(torch.uint8).cpu().numpy(), wc) and np.array_equal(s.view(torch.uint8).cpu().numpy(), ws)
    y = ref.rmsnorm(ref.dequantize(wc, ws, 32, ref.E4M3), np.ones(cols), 1e-5)[0]
    ref.check_held(n[0].view(torch.uint8).cpu().numpy(), n[1].view(torch.uint8).cpu().numpy(), y, rel_of_norm(cols), 32, ref.E4M3)


def test_offsets_past_32_bits():
    """Rows that lie more than 2^32 elements from the first one: only those are looked at on the host."""
    rows, cols, stride = 5, 1 << 10, (1 << 30) + 8
    need = (rows - 1) * stride + cols
    if torch.cuda.mem_get_info()[0] < 2 * need + (4 << 30):
        pytest.skip("not enough free memory")
    buf = torch.empty(need, dtype=BF16, device="cuda")
    x = torch.as_strided(buf, (rows, cols), (stride, 1))
    src = mixed(rows, cols, 3, BF16, special=False)
    x.copy_(src)
    c, s = mxq.alloc_outputs8(rows, cols, 32, ref.E4M3, "cuda")
    mxq.mxq_quantize8(x, 32, ref.E4M3, c, s)
    wc, ws = ref.quantize(np64(src), 32, ref.E4M3)
    assert np.array_equal(c.view(torch.uint8).cpu().numpy(), wc) and np.array_equal(s.view(torch.uint8).cpu().numpy(), ws)
    x.zero_()
    mxq.mxq_dequantize8(c, s, 32, ref.E4M3, x)
    assert np.array_equal(np64(x), ref.dequantize(wc, ws, 32, ref.E4M3).astype(np.float32).astype(np.float64)) or \
        torch.equal(x.cpu(), torch.from_numpy(ref.dequantize(wc, ws, 32, ref.E4M3)).float().to(BF16))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols,pad,shift", [(1024, 0, 0), (4096, 0, 0), (8192, 0, 0), (16384, 0, 0), (32768, 0, 0), (4104, 0, 0), (1000, 3, 1), (128, 0, 0)])
def test_the_workspace_changes_no_bit_of_the_gradients(cols, pad, shift, dtype):
    """On 32, 16 bytes, or not there: the kernels of whole, halved and shifted rows, one row of each and several."""
    rows = 400
    dy, ds, w, codes, scales, rstd = backward_inputs(rows, cols, pad, shift, dtype, F32, ref.E4M3, 32, cols)
    got = []
    for at in (None, 0, 4, 12):
        dx, dw = Guarded(rows, cols, dtype, pad, shift), Guarded(1, cols, F32)
        room = mxq.mxq_add_rmsnorm8_workspace_bytes(rows, cols) // 4
        ws = Guarded(1, room, F32, 0, at or 0)
        if at is None:
            mxq.mxq_add_rmsnorm8_backward(dy, ds, w, codes, scales, rstd, 32, ref.E4M3, dx.t)
        else:
            mxq.mxq_add_rmsnorm8_backward(dy, ds, w, codes, scales, rstd, 32, ref.E4M3, dx.t, dw.t, ws.t.view(-1))
        assert dx.untouched() and dw.untouched() and ws.untouched()
        got.append((dx.t, dw.t))
    for dx, dw in got[1:]:
        assert torch.equal(dx, got[0][0]) and torch.equal(dw, got[1][1])


def dequantize64(codes, scales, B, fmt):
    """The values of 8-bit codes (bytes), in binary64 on the device."""
    table = torch.from_numpy(ref.value_of(np.arange(256, dtype=np.uint8), fmt)).cuda()
    s = torch.exp2(scales.double() - 127).repeat_interleave(B, 1)[:, : codes.shape[1]]
    return table[codes.long()] * s


# Every kernel of the gradient with more rows (or groups of rows) than it has CTAs: rows that share a warp; whole, halved and shifted rows of CTAs of
# 256, 512 and 1024 threads; the streaming kernels; two and four vectors a thread.
MANY_ROWS = [(F32, 200001, 3, 0, 0), (BF16, 200001, 3, 0, 0), (BF16, 70000, 16, 0, 0), (BF16, 90001, 24, 0, 0), (F32, 40000, 200, 0, 0), (BF16, 30000, 500, 1, 1),
             (F32, 1500, 1001, 1, 1), (BF16, 1500, 1001, 0, 0), (BF16, 1500, 1000, 8, 0), (F32, 900, 2501, 0, 0), (BF16, 900, 5001, 0, 1), (BF16, 900, 4104, 0, 0),
             (F32, 400, 5001, 0, 0), (BF16, 400, 9001, 3, 0), (BF16, 400, 8200, 0, 0), (F32, 400, 9001, 0, 0), (BF16, 400, 16389, 0, 0), (BF16, 400, 20008, 0, 0),
             (BF16, 400, 32768, 0, 0), (F32, 400, 17001, 0, 1), (F32, 400, 20004, 0, 0), (F32, 400, 32768, 0, 0), (F32, 400, 16384, 0, 0), (BF16, 900, 1024, 0, 0),
             (BF16, 900, 5120, 0, 0), (BF16, 900, 6144, 0, 0), (BF16, 900, 8192, 0, 0), (BF16, 400, 16384, 0, 0), (F32, 900, 2048, 0, 0), (F32, 900, 8192, 0, 0)]


@pytest.mark.parametrize("with_dsum", [True, False])
@pytest.mark.parametrize("dtype,rows,cols,pad,shift", MANY_ROWS)
def test_gradient_of_the_weight_counts_every_row(dtype, rows, cols, pad, shift, with_dsum):
    """dy has the sign of h, so that every row adds to dweight, and the bound counts the additions that are made: what a CTA takes in one turn is far above it."""
    B, fmt = 16, ref.E4M3
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    codes, scales = (t.view(torch.uint8) for t in mxq.quantize8(rand(rows, cols), B, fmt))
    h = dequantize64(codes, scales, B, fmt)
    rstd = (h.square().mean(1) + 1e-5).rsqrt().float()
    dy = Guarded(rows, cols, dtype, pad, shift).fill((1 + rand(rows, cols).abs()) * torch.where(h < 0, -1.0, 1.0).float())
    ds = Guarded(rows, cols, dtype, pad, shift).fill(rand(rows, cols)) if with_dsum else None
    w = 1 + 0.2 * rand(cols)
    dx, dw = Guarded(rows, cols, dtype, pad, shift), Guarded(1, cols, F32)
    mxq.mxq_add_rmsnorm8_backward(dy, ds, w, codes, scales, rstd, B, fmt, dx.t, dw.t, workspace(rows, cols))
    assert dx.untouched() and dw.untouched()
    r, n = rstd.double()[:, None], h * rstd.double()[:, None]
    wd = w.double() * dy.double()
    mean, size_of_mean = (wd * n).mean(1, keepdim=True), (wd * n).abs().mean(1, keepdim=True)
    want, size = r * (wd - n * mean), r * (wd.abs() + n.abs() * size_of_mean)
    if with_dsum:
        want, size = want + ds.double(), size + ds.double().abs()
    assert bool(((dx.t.double() - want).abs() <= HALF[dtype] * want.abs() + 65 * U * size).all())    # as in test_add_rmsnorm8_backward
    # dweight: the rounding of n; a turn each of a thread, of which a CTA has the fewer the more CTAs there are (one an SM at least); the groups of
    # rows of a CTA, one after the other; at most 1024 parts, every 32nd by a warp, and a tree over the warps
    vectors = -(-cols // B) * (B // (8 if dtype == F32 else 16))
    group = 1 << max(0, (vectors - 1).bit_length()) if vectors <= 32 else 0
    rows_cta = 256 // group if group else 1
    work = -(-rows // rows_cta)
    turns = -(-work // min(work, torch.cuda.get_device_properties(0).multi_processor_count))
    terms = dy.double() * n
    total = terms.sum(0)
    bound = (1 + turns + (rows_cta if group else 0) + min(work, 1024) // 32 + 1 + 5) * U * terms.abs().sum(0)
    assert bool(((dw.t[0].double() - total).abs() <= bound).all())
    # without what one CTA adds in one turn the check would fail, whichever turn it is
    parts = torch.nn.functional.pad(terms, (0, 0, 0, work * rows_cta - rows)).view(work, rows_cta, cols).sum(1)
    assert bool((parts.abs() > 2 * bound).any(1).all())


@pytest.mark.parametrize("dtype,rows,cols,pad,shift", [(BF16, 9, 1001, 3, 1), (F32, 9, 1001, 0, 1), (BF16, 40, 2501, 0, 0), (F32, 40, 2502, 0, 2), (BF16, 7, 8193, 0, 3), (F32, 5, 8190, 0, 0),
                                                       (BF16, 3, 20001, 1, 0), (F32, 3, 20001, 0, 0), (BF16, 300, 77, 0, 0), (BF16, 6, 4104, 0, 0)])
def test_norm_and_gradient_in_place_on_shifted_rows(dtype, rows, cols, pad, shift):
    """Over either summand, over dy and over dsum, where neighbouring rows, warps and vectors of a thread share 16-byte pieces."""
    x, r, w = norm_inputs(rows, cols, pad, shift, dtype, F32, cols)
    got = []
    for over in (None, "x", "residual"):
        a, b = Guarded(rows, cols, dtype, pad, shift), Guarded(rows, cols, dtype, pad, shift)
        a.fill(x), b.fill(r)
        out = {None: Guarded(rows, cols, dtype, pad, shift), "x": a, "residual": b}[over]
        held, kept, rstd = held_out(rows, cols, 16), held_out(rows, cols, 16), torch.empty(rows, device="cuda")
        mxq.mxq_add_rmsnorm8(a.t, b.t, w, 1e-5, 16, ref.E4M3, out.t, held[0].t, held[1].t, kept[0].t, kept[1].t, rstd)
        assert out.untouched() and all(t.untouched() for t in held + kept)
        got.append([out.t, rstd] + [t.t for t in held + kept])
    assert torch.equal(got[0][0], (x.float() + r.float()).to(dtype))
    for other in got[1:]:
        assert all(torch.equal(p, q) for p, q in zip(other, got[0]))
    rstd, kept = got[0][1], [got[0][4].view(rows, cols), got[0][5].view(rows, -1)]
    got = []
    for over in (None, "dy", "dsum", "both"):
        a, b = Guarded(rows, cols, dtype, pad, shift), Guarded(rows, cols, dtype, pad, shift)
        a.fill(x), b.fill(x if over == "both" else r)
        out = {None: Guarded(rows, cols, dtype, pad, shift), "dy": a, "dsum": b, "both": a}[over]
        dw = torch.empty(cols, device="cuda")
        mxq.mxq_add_rmsnorm8_backward(a.t, a.t if over == "both" else b.t, w, *kept, rstd, 16, ref.E4M3, out.t, dw, workspace(rows, cols))
        assert out.untouched()
        if over == "both":
            plain = Guarded(rows, cols, dtype, pad, shift)
            mxq.mxq_add_rmsnorm8_backward(b.t, b.t, w, *kept, rstd, 16, ref.E4M3, plain.t)
            assert torch.equal(out.t, plain.t)
        else:
            got.append((out.t, dw))
    for dx, dw in got[1:]:
        assert torch.equal(dx, got[0][0]) and torch.equal(dw, got[0][1])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,B", [(33, 256, 32), (5, 4096, 16), (3, 9216, 128), (2, 20480, 64)])
def test_where_rows_start_changes_no_bit_that_is_elementwise(rows, cols, B, dtype):
    """Whole, halved and shifted rows of the same values: sums, codes of given tensors, the gated activation and its gradient are the same bits."""
    x, r, w = norm_inputs(rows, cols, 0, 0, dtype, F32, cols)
    first = None
    for pad, shift in ((0, 0), (0, 16 // x.element_size()), (3, 1), (8, 5)):
        put = lambda v: Guarded(rows, cols, dtype, pad, shift).fill(v)  # noqa: E731
        a, b = put(x), put(r)
        wide = [Guarded(rows, cols, dtype, pad, shift) for _ in range(4)]
        y, kept, q, act, gk, uk = (held_out(rows, cols, B) for _ in range(6))
        mxq.mxq_add_rmsnorm8(a, b, w, 1e-5, B, ref.E4M3, wide[0].t, y[0].t, y[1].t, kept[0].t, kept[1].t)
        mxq.mxq_quantize8(a, B, ref.E4M3, q[0].t, q[1].t)
        mxq.mxq_dequantize8(q[0].t, q[1].t, B, ref.E4M3, wide[1].t)
        mxq.mxq_swiglu8(a, b, B, ref.E4M3, act[0].t, act[1].t, gk[0].t, gk[1].t, uk[0].t, uk[1].t)
        mxq.mxq_swiglu8_backward(b, gk[0].t, gk[1].t, uk[0].t, uk[1].t, B, ref.E4M3, wide[2].t, wide[3].t)
        assert all(t.untouched() for t in wide)
        out = [t.t.clone() for t in wide] + [t.t.clone() for pair in (kept, q, act, gk, uk) for t in pair]
        first = first or out
        assert all(torch.equal(p, o) for p, o in zip(first, out))


@pytest.mark.parametrize("fmt,first", [(ref.E4M3, 1.9375), (ref.E5M2, 1.875)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_upper_end_of_the_format(fmt, first, dtype):
    """Finite magnitudes that a code rounds to 2^128 read back as infinities, the next smaller ones do not; neighbours in the block keep their values."""
    below = first - (2.0 ** -7 if dtype == BF16 else 2.0 ** -23)
    x = torch.zeros(4, 32, dtype=torch.float64)
    for row, m in enumerate((first, below, -first, torch.finfo(dtype).max / 2.0 ** 127)):
        x[row, 5], x[row, 6] = m * 2.0 ** 127, 2.0 ** 126
    x = x.to(dtype).cuda()
    c, s = mxq.quantize8(x, 32, fmt)
    wc, ws = ref.quantize(np64(x), 32, fmt)
    assert np.array_equal(c.view(torch.uint8).cpu().numpy(), wc) and np.array_equal(s.view(torch.uint8).cpu().numpy(), ws)
    back = torch.empty_like(x)
    mxq.mxq_dequantize8(c, s, 32, fmt, back)
    inf = float("inf")
    assert back[0, 5] == inf and torch.isfinite(back[1, 5]) and back[2, 5] == -inf and back[3, 5] == inf
    assert bool((back[:, 6] == 2.0 ** 126).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", [64, 1001, 2048])
def test_a_sum_of_squares_past_binary32_gives_zeros(cols, dtype):
    x = torch.randn(3, cols, device="cuda").to(dtype)
    x[1] = 2.0 ** 64
    w, rstd = torch.ones(cols, device="cuda"), torch.empty(3, device="cuda")
    c, s = mxq.alloc_outputs8(3, cols, 16, ref.E4M3, "cuda")
    mxq.mxq_add_rmsnorm8(x, None, w, 1e-5, 16, ref.E4M3, None, c, s, None, None, rstd)
    c = c.view(torch.uint8)
    assert rstd[1] == 0 and bool(((c[1] & 0x7F) == 0).all()) and bool((s.view(torch.uint8)[1] == 0).all())
    assert bool((rstd[[0, 2]] > 0).all()) and bool(((c[[0, 2]] & 0x7F) != 0).any(1).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sigmoids_at_the_lower_end_of_binary32(dtype):
    """Zero below 2^-126, in the forward pass and in both gradients, and no NaN there."""
    gate = torch.tensor([-80.0, -87.0, -87.5, -88.0, -89.0, -1000.0, -3e38, 0.0] * 4, device="cuda").to(dtype).view(2, 16)
    up = torch.full_like(gate, 2.0 ** 100)
    (c, s), g, u = (mxq.alloc_outputs8(2, 16, 16, ref.E4M3, "cuda") for _ in range(3))
    mxq.mxq_swiglu8(gate, up, 16, ref.E4M3, c, s, *g, *u)
    held = torch.empty_like(gate)
    mxq.mxq_dequantize8(c, s, 16, ref.E4M3, held)
    far = gate < -87.4
    assert bool((held[far] == 0).all()) and bool((held[gate == -80.0] < 0).all())
    # the gradients of such gates, each in a block of its own scale so that the codes hold them
    for v in (-88.0, -1000.0, -3e38):
        (gc, gs), (uc, us) = mxq.quantize8(torch.full((1, 16), v, device="cuda"), 16, ref.E4M3), mxq.quantize8(torch.ones(1, 16, device="cuda"), 16, ref.E4M3)
        dy, dg, du = torch.ones(1, 16, device="cuda", dtype=dtype), torch.empty(1, 16, device="cuda", dtype=dtype), torch.empty(1, 16, device="cuda", dtype=dtype)
        mxq.mxq_swiglu8_backward(dy, gc, gs, uc, us, 16, ref.E4M3, dg, du)
        assert bool((dg == 0).all()) and bool((du == 0).all()), v


def test_helpers_and_workspaces_that_do_not_fit_are_refused(route):
    x = torch.zeros(4, 64, device="cuda", dtype=BF16)
    u8 = lambda *n: torch.zeros(*n, device="cuda", dtype=torch.uint8)  # noqa: E731
    c, s, w, f = u8(4, 64), u8(4, 2), torch.ones(64, device="cuda"), torch.ones(4, device="cuda")
    back = lambda ws: mxq.mxq_add_rmsnorm8_backward(x, None, w, c, s, f, 32, 0, x.clone(), w.clone(), ws)  # noqa: E731
    back(torch.empty(256, device="cuda"))
    for f_, text in ((lambda: mxq.quantize8(x, 0), "block_size"), (lambda: mxq.quantize8(x, 24), "block_size"), (lambda: mxq.quantize8(x, 32, 2), "elem_fmt"),
                     (lambda: mxq.quantize8(x[0, 0]), "scalar"), (lambda: mxq.quantize8(x[:, :0]), "at least one"), (lambda: mxq.quantize8(x[:0]), "at least one"),
                     (lambda: back(torch.empty(256)), "CUDA tensors only"), (lambda: back(4096), "CUDA tensors only"),
                     (lambda: back(torch.empty(512, device="cuda")[::2]), "contiguous"), (lambda: back(torch.empty(255, device="cuda")), "status 6"),
                     (lambda: back(torch.empty(300, device="cuda")[1:]), "status 4")):
        with pytest.raises(mxq.MxqError, match=text):
            f_()


@pytest.fixture
def memory_given_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("cols", [4096, 4097])
def test_tensors_of_more_than_32_bits_of_elements(cols, memory_given_back):
    """2^32 elements and some rows: the first and the last rows are the bits that calls on those rows alone give."""
    rows, B, fmt, few = (1 << 20) + 70, 32, ref.E4M3, 64
    if torch.cuda.mem_get_info()[0] < (60 << 30):
        pytest.skip("not enough free memory")
    x, r = (torch.empty(rows, cols, dtype=BF16, device="cuda").normal_() for _ in range(2))
    x0, r0 = ([t[:few].clone(), t[-few:].clone()] for t in (x, r))
    w = torch.linspace(0.5, 1.5, cols, device="cuda")
    y, kept, rstd = mxq.alloc_outputs8(rows, cols, B, fmt, "cuda"), mxq.alloc_outputs8(rows, cols, B, fmt, "cuda"), torch.empty(rows, device="cuda")
    ends = lambda *ts: [[t[:few].clone().view(torch.uint8) if t.element_size() == 1 else t[:few].clone() for t in ts],  # noqa: E731
                        [t[-few:].clone().view(torch.uint8) if t.element_size() == 1 else t[-few:].clone() for t in ts]]

    def same(got, want):
        assert all(torch.equal(a, b) for a, b in zip(got, want))

    mxq.mxq_add_rmsnorm8(x, r, w, 1e-5, B, fmt, r, *y, *kept, rstd)
    got = ends(r, *y, *kept, rstd)
    for k in (0, 1):
        y1, k1, s1, h1 = mxq.alloc_outputs8(few, cols, B, fmt, "cuda"), mxq.alloc_outputs8(few, cols, B, fmt, "cuda"), torch.empty(few, device="cuda"), torch.empty_like(x0[k])
        mxq.mxq_add_rmsnorm8(x0[k], r0[k], w, 1e-5, B, fmt, h1, *y1, *k1, s1)
        same(got[k], [h1] + [t.view(torch.uint8) for t in (*y1, *k1)] + [s1])
    # the gradient with x as dy and the sum as dsum, over x
    r1 = [got[k][0] for k in (0, 1)]
    mxq.mxq_add_rmsnorm8_backward(x, r, w, *kept, rstd, B, fmt, x)
    got = ends(x)
    for k in (0, 1):
        k1 = [(t[:few] if k == 0 else t[-few:]).clone() for t in kept]
        s1, d1 = (rstd[:few] if k == 0 else rstd[-few:]).clone(), torch.empty_like(x0[k])
        mxq.mxq_add_rmsnorm8_backward(x0[k], r1[k], w, *k1, s1, B, fmt, d1)
        same(got[k], [d1])
    x1 = [got[k][0] for k in (0, 1)]
    # the gated activation of (x, r) with its gradient, store and load
    mxq.mxq_swiglu8(x, r, B, fmt, *y, *kept, *(u := mxq.alloc_outputs8(rows, cols, B, fmt, "cuda")))
    got = ends(*y, *kept, *u)
    held = []
    for k in (0, 1):
        a = [mxq.alloc_outputs8(few, cols, B, fmt, "cuda") for _ in range(3)]
        mxq.mxq_swiglu8(x1[k], r1[k], B, fmt, *a[0], *a[1], *a[2])
        same(got[k], [t.view(torch.uint8) for p in a for t in p])
        held.append(a)
    other = torch.empty_like(x)
    mxq.mxq_swiglu8_backward(x, *kept, *u, B, fmt, x, other)
    got = ends(x, other)
    for k in (0, 1):
        dg, du = torch.empty_like(x1[k]), torch.empty_like(x1[k])
        mxq.mxq_swiglu8_backward(x1[k], *held[k][1], *held[k][2], B, fmt, dg, du)
        same(got[k], [dg, du])
    mxq.mxq_quantize8(r, B, fmt, *y)
    mxq.mxq_dequantize8(*y, B, fmt, other)
    got = ends(*y, other)
    for k in (0, 1):
        c1, s1 = mxq.quantize8(r1[k], B, fmt)
        back = torch.empty_like(r1[k])
        mxq.mxq_dequantize8(c1, s1, B, fmt, back)
        same(got[k], [c1.view(torch.uint8), s1.view(torch.uint8), back])


def test_rows_times_lanes_past_32_bits(memory_given_back):
    """Rows of one element in blocks of 128: 2^32 vectors and some, most of them behind the ends of the rows."""
    rows, few = (1 << 29) + 7, 1000
    x = torch.empty(rows, 1, dtype=BF16, device="cuda").normal_()
    c, s = mxq.quantize8(x, 128, ref.E5M2)
    back = torch.empty_like(x)
    mxq.mxq_dequantize8(c, s, 128, ref.E5M2, back)
    for part in (slice(0, few), slice(rows // 2, rows // 2 + few), slice(rows - few, rows)):
        wc, ws = ref.quantize(np64(x[part]), 128, ref.E5M2)
        assert np.array_equal(c[part].view(torch.uint8).cpu().numpy(), wc) and np.array_equal(s[part].view(torch.uint8).cpu().numpy(), ws)
        assert np.array_equal(np64(back[part]), ref.dequantize(wc, ws, 128, ref.E5M2))
