"""The operators on block-scaled 8-bit activations from their definitions, in numpy and binary64: test infrastructure only.

Nothing here is shared with the library: formats are value tables made from their bit fields, roundings are searches for the
nearest value in them."""
import numpy as np

E4M3, E5M2 = 0, 1
TOP = {E4M3: 448.0, E5M2: 57344.0}
U = 2.0 ** -24          # half a unit in the last place of a binary32 value, relative


def _table(fmt):
    mant, bias, last = (3, 7, 0x7E) if fmt == E4M3 else (2, 15, 0x7B)
    v = []
    for c in range(last + 1):
        e, m = c >> mant, (c & ((1 << mant) - 1)) / (1 << mant)
        v.append(m * 2.0 ** (1 - bias) if e == 0 else (1 + m) * 2.0 ** (e - bias))
    return np.array(v)


TABLE = {f: _table(f) for f in (E4M3, E5M2)}


def value_of(codes, fmt):
    """Codes (uint8) -> binary64; NaN and infinity codes as the formats have them."""
    t = np.full(128, np.nan)
    t[: len(TABLE[fmt])] = TABLE[fmt]
    if fmt == E5M2:
        t[0x7C] = np.inf
    return np.where(codes >> 7, -1.0, 1.0) * t[codes & 127]


def scale_of(bytes_):
    return np.where(bytes_ == 255, np.nan, 2.0 ** (bytes_.astype(np.float64) - 127))


def scale_bytes(v, B, fmt):
    """Smallest power of two >= 2^-127 with amax <= TOP * S; 255 for a block that is not finite."""
    rows, cols = v.shape
    nb = -(-cols // B)
    p = np.zeros((rows, nb * B))
    p[:, :cols] = v
    a = np.abs(p.reshape(rows, nb, B)).max(2)      # NaN wins
    out = np.full((rows, nb), 255, np.uint8)
    s = 2.0 ** (np.arange(255) - 127.0)
    ok = np.isfinite(a)
    out[ok] = np.searchsorted(TOP[fmt] * s, a[ok], side="left")
    return out


def over_blocks(per_block, cols, B):
    return np.repeat(per_block, B, axis=1)[:, :cols]


def nearest(q, fmt):
    """Codes nearest to |q| <= TOP, ties to the even code, with q's sign bit."""
    t = TABLE[fmt]
    a = np.abs(q)
    hi = np.searchsorted(t, a, side="left").clip(0, len(t) - 1)
    lo = (hi - 1).clip(0)
    dl, dh = a - t[lo], t[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (c | (np.signbit(q).astype(np.int64) << 7)).astype(np.uint8)


def quantize(v, B, fmt):
    """(codes, scale bytes) of a matrix."""
    b = scale_bytes(v, B, fmt)
    s = over_blocks(scale_of(b), v.shape[1], B)
    with np.errstate(invalid="ignore"):
        q = v / s
    codes = nearest(np.where(np.isfinite(q), q, 0.0), fmt)
    codes[~np.isfinite(s)] = 0x7F
    return codes, b


def dequantize(codes, b, B, fmt):
    return value_of(codes, fmt) * over_blocks(scale_of(b), codes.shape[1], B)


def half_step(q, fmt):
    """Half the distance between neighbouring values at |q|."""
    mant, least = (3, -6) if fmt == E4M3 else (2, -14)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.maximum(np.abs(q), 2.0 ** least)))
    return 2.0 ** (np.maximum(e, least) - mant - 1)


def check_held(codes, b, v, rel, B, fmt, absolute=0.0):
    """Codes and scale bytes are those of SOME matrix that is `rel` relative (and `absolute`) from v at most."""
    rows, cols = v.shape
    finite = np.isfinite(v)
    near = rel * np.abs(np.where(finite, v, 0)) + absolute
    big = np.where(finite, np.abs(v) + near, v)
    small = np.where(finite, np.maximum(np.abs(v) - near, 0), v)
    lo, hi = scale_bytes(small, B, fmt), scale_bytes(big, B, fmt)
    assert ((b >= lo) & (b <= hi)).all(), "scale bytes"
    s = over_blocks(scale_of(b), cols, B)
    bad = ~np.isfinite(s)
    assert (codes[bad] == 0x7F).all()
    got = value_of(codes, fmt) * s
    with np.errstate(invalid="ignore"):
        # past the largest element value by rounding, a value saturates: by `rel` at most, which `near` holds
        off = np.abs(got - v) - (half_step(np.abs(v) / s + near / s, fmt) * s + near)
    assert (off[~bad] <= 0).all(), float(np.nanmax(off[~bad]))


# ---- operators -----------------------------------------------------------------------------------
def rmsnorm(h, w, eps):
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    return h * rstd[:, None] * w, rstd


def rmsnorm_backward(dy, w, h, rstd, dsum=None):
    """(dx, dweight) and, per element, what the rounding errors of dx scale with."""
    n = h * rstd[:, None]
    wd = w * dy
    dx = rstd[:, None] * (wd - n * (wd * n).mean(1, keepdims=True))
    size = rstd[:, None] * (np.abs(wd) + np.abs(n) * np.abs(wd * n).mean(1, keepdims=True))
    if dsum is not None:
        dx, size = dx + dsum, size + np.abs(dsum)
    return dx, (dy * n).sum(0), size, np.abs(dy * n).sum(0)


def sigmoid(g):
    e = np.exp(-np.abs(g))
    return np.where(g >= 0, 1 / (1 + e), e / (1 + e))


def swiglu(g, u):
    return g * sigmoid(g) * u


def swiglu_backward(dy, g, u):
    s = sigmoid(g)
    return dy * u * s * (1 + g * (1 - s)), dy * g * s
