"""Host-only checks of the operators on block-scaled 8-bit activations: what they refuse, before anything is launched, and the
reference that the GPU tests compare with against torch's float8 casts."""
import numpy as np
import pytest
import torch

import act8_ref as ref

# fake, 16-byte aligned "device" addresses
A, B_, C, D, E, F, G, H = (0x10000 * k for k in range(1, 9))


@pytest.fixture(scope="module")
def lib():
    from paper_2605_08565_b200 import binding, build
    build.build()
    return binding.load_library()


def caller(f, names, **good):
    def call(**kw):
        assert set(kw) <= set(good)
        return f(*[{**good, **kw}[n] for n in names.split()])
    return call


COMMON = [(dict(dtype=2), 2), (dict(dtype=-1), 2), (dict(elem=2), 2), (dict(elem=-1), 2), (dict(block=8), 3), (dict(block=0), 3), (dict(block=-32), 3),
          (dict(block=256), 3), (dict(rows=0), 3), (dict(cols=0), 3), (dict(rows=1 << 31), 8), (dict(rows=2 ** 64 - 1, cols=2 ** 64 - 1), 8)]


def check(call, cases):
    for kw, status in COMMON + cases:
        assert call(**kw) == status, (kw, status)


def test_quantize8_and_dequantize8_refuse(lib):
    q = caller(lib.mxq_quantize8, "x dtype rows cols stride block elem codes scales stream", x=A, dtype=0, rows=4, cols=64, stride=64, block=32, elem=0, codes=B_,
               scales=C, stream=0)
    check(q, [(dict(x=0), 1), (dict(codes=0), 1), (dict(scales=0), 1), (dict(stride=63), 3), (dict(x=A + 2), 4), (dict(x=A + 1, dtype=1), 4), (dict(codes=B_ + 8), 4),
              (dict(rows=1 << 30, cols=1 << 12, stride=1 << 12), 8), (dict(cols=2 ** 63, stride=2 ** 63), 8)])
    d = caller(lib.mxq_dequantize8, "codes scales rows cols block elem out dtype stride stream", codes=A, scales=B_, rows=4, cols=64, block=32, elem=0, out=C, dtype=0,
               stride=64, stream=0)
    check(d, [(dict(codes=0), 1), (dict(scales=0), 1), (dict(out=0), 1), (dict(stride=63), 3), (dict(out=C + 2), 4), (dict(codes=A + 4), 4)])


def test_add_rmsnorm8_refuses(lib):
    n = caller(lib.mxq_add_rmsnorm8, "x residual weight dtype wtype rows cols sx sr eps block elem sum ss codes scales kcodes kscales rstd stream", x=A, residual=B_,
               weight=C, dtype=0, wtype=0, rows=4, cols=64, sx=64, sr=64, eps=1e-5, block=32, elem=0, sum=D, ss=64, codes=E, scales=F, kcodes=G, kscales=H, rstd=0,
               stream=0)
    check(n, [(dict(x=0), 1), (dict(residual=0), 1), (dict(sum=0), 1), (dict(weight=0), 1), (dict(codes=0), 1), (dict(scales=0), 1), (dict(kcodes=0), 1),
              (dict(kscales=0), 1), (dict(wtype=2), 2), (dict(sx=60), 3), (dict(sr=60), 3), (dict(ss=60), 3), (dict(eps=0.0), 5), (dict(eps=-1.0), 5),
              (dict(eps=float("inf")), 5), (dict(eps=float("nan")), 5), (dict(cols=32769, sx=40000, sr=40000, ss=40000), 8), (dict(sum=A, sx=72), 3),
              (dict(sum=B_, sr=72), 3), (dict(weight=C + 2), 4), (dict(rstd=2), 4), (dict(codes=E + 8), 4), (dict(kcodes=G + 8), 4), (dict(residual=B_ + 1), 4)])


def test_add_rmsnorm8_backward_refuses(lib):
    names = "dy dsum weight dtype wtype rows cols sy ss kcodes kscales rstd block elem dx sx dweight ws ws_bytes stream"
    n = caller(lib.mxq_add_rmsnorm8_backward, names, dy=A, dsum=B_, weight=C, dtype=0, wtype=0, rows=4, cols=64, sy=64, ss=64, kcodes=D, kscales=E, rstd=F, block=32,
               elem=0, dx=G, sx=64, dweight=H, ws=0x90000, ws_bytes=4 * 64 * 4, stream=0)
    check(n, [(dict(dy=0), 1), (dict(weight=0), 1), (dict(kcodes=0), 1), (dict(kscales=0), 1), (dict(rstd=0), 1), (dict(dx=0), 1), (dict(wtype=-1), 2), (dict(sy=60), 3),
              (dict(ss=60), 3), (dict(sx=60), 3), (dict(dx=A, sy=72), 3), (dict(dx=B_, ss=72), 3), (dict(cols=32769, sx=40000, sy=40000, ss=40000), 8), (dict(ws=0), 6),
              (dict(ws_bytes=4 * 64 * 4 - 1), 6), (dict(ws=0x90008), 4), (dict(rstd=F + 2), 4), (dict(dweight=H + 2), 4), (dict(dx=G + 2), 4)])
    assert lib.mxq_add_rmsnorm8_workspace_bytes(4, 64) == 4 * 64 * 4
    assert lib.mxq_add_rmsnorm8_workspace_bytes(1 << 20, 4096) <= 1024 * 4096 * 4


def test_swiglu8_refuses(lib):
    f = caller(lib.mxq_swiglu8, "gate up dtype rows cols sg su block elem codes scales gc gs uc us stream", gate=A, up=B_, dtype=0, rows=4, cols=64, sg=64, su=64, block=32,
               elem=0, codes=C, scales=D, gc=E, gs=F, uc=G, us=H, stream=0)
    check(f, [(dict(gate=0), 1), (dict(up=0), 1), (dict(codes=0), 1), (dict(scales=0), 1), (dict(gc=0), 1), (dict(gs=0), 1), (dict(uc=0), 1), (dict(us=0), 1),
              (dict(gc=0, gs=0, uc=0), 1), (dict(sg=60), 3), (dict(su=60), 3), (dict(up=B_ + 2), 4), (dict(uc=G + 8), 4)])
    b = caller(lib.mxq_swiglu8_backward, "dy dtype rows cols sy gc gs uc us block elem dgate sg dup su stream", dy=A, dtype=0, rows=4, cols=64, sy=64, gc=B_, gs=C, uc=D, us=E,
               block=32, elem=0, dgate=F, sg=64, dup=G, su=64, stream=0)
    check(b, [(dict(dy=0), 1), (dict(gc=0), 1), (dict(gs=0), 1), (dict(uc=0), 1), (dict(us=0), 1), (dict(dgate=0), 1), (dict(dup=0), 1), (dict(sy=60), 3), (dict(sg=60), 3),
              (dict(su=60), 3), (dict(dgate=G), 3), (dict(dgate=A, sg=72), 3), (dict(dup=A, su=72), 3), (dict(dup=G + 2), 4)])


@pytest.mark.parametrize("rows,cols", [(1 << 30, 1 << 34), (1 << 30, (1 << 34) + 128), (1 << 27, 1 << 37), ((1 << 31) - 1, 1 << 33), (1 << 24, 1 << 41), (1 << 15, (1 << 26) + 1)])
def test_sizes_whose_product_passes_64_bits_are_too_large(lib, rows, cols):
    """Four products of rows and padded cols are small modulo 2^64, one comes close to it, and the last one is past the limit by its padding alone."""
    assert rows * -(-cols // 128) * 128 > 1 << 41
    assert lib.mxq_quantize8(A, 0, rows, cols, cols, 32, 0, B_, C, 0) == 8
    assert lib.mxq_dequantize8(A, B_, rows, cols, 32, 0, C, 0, cols, 0) == 8
    assert lib.mxq_swiglu8(A, B_, 0, rows, cols, cols, cols, 32, 0, C, D, 0, 0, 0, 0, 0) == 8
    assert lib.mxq_swiglu8_backward(A, 0, rows, cols, cols, B_, C, D, E, 32, 0, F, cols, G, cols, 0) == 8
    assert lib.mxq_add_rmsnorm8(A, 0, C, 0, 0, rows, cols, cols, 0, 1e-5, 32, 0, 0, 0, E, F, 0, 0, 0, 0) == 8
    assert lib.mxq_add_rmsnorm8_backward(A, 0, C, 0, 0, rows, cols, cols, 0, D, E, F, 32, 0, G, cols, 0, 0, 0, 0) == 8


def test_binding_refuses_what_is_not_on_a_gpu(lib):
    from paper_2605_08565_b200 import binding as mxq
    x, c, s = torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)
    for f in (lambda: mxq.mxq_quantize8(x, 32, mxq.MXQ_E4M3, c, s), lambda: mxq.mxq_dequantize8(c, s, 32, mxq.MXQ_E4M3, x),
              lambda: mxq.mxq_add_rmsnorm8(x, None, x[0], 1e-5, 32, mxq.MXQ_E4M3, None, c, s),
              lambda: mxq.mxq_add_rmsnorm8_backward(x, None, x[0], c, s, x[:, 0], 32, mxq.MXQ_E4M3, x),
              lambda: mxq.mxq_swiglu8(x, x, 32, mxq.MXQ_E4M3, c, s), lambda: mxq.mxq_swiglu8_backward(x, c, s, c, s, 32, mxq.MXQ_E4M3, x, x),
              lambda: mxq.quantize8(x)):
        with pytest.raises(mxq.MxqError, match="CUDA tensors only"):
            f()


def test_helpers_refuse_options_that_there_are_not(lib):
    from paper_2605_08565_b200 import binding as mxq
    for B in (0, 8, 24, -32, 32.0, True, None):
        with pytest.raises(mxq.MxqError, match="block_size"):
            mxq.alloc_outputs8(4, 64, B, mxq.MXQ_E4M3, "cpu")
    for fmt in (2, -1, None):
        with pytest.raises(mxq.MxqError, match="elem_fmt"):
            mxq.alloc_outputs8(4, 64, 32, fmt, "cpu")
    for x in (torch.tensor(1.0), None, 3):
        with pytest.raises(mxq.MxqError, match="CUDA tensors only"):
            mxq.quantize8(x)


@pytest.mark.parametrize("fmt,kind", [(ref.E4M3, torch.float8_e4m3fn), (ref.E5M2, torch.float8_e5m2)])
def test_reference_formats_and_rounding_are_torch_s(fmt, kind):
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(kind).double().numpy()
    assert np.array_equal(ref.value_of(codes, fmt), want, equal_nan=True)
    t = ref.TABLE[fmt]
    q = np.concatenate([t, (t[1:] + t[:-1]) / 2, np.nextafter(np.float32((t[1:] + t[:-1]) / 2), np.float32(0)).astype(float),
                        np.random.default_rng(1).uniform(0, ref.TOP[fmt], 5000).astype(np.float32).astype(float)])
    q = np.concatenate([q, -q])
    assert np.array_equal(ref.nearest(q, fmt), torch.from_numpy(q.astype(np.float32)).to(kind).view(torch.uint8).numpy())


@pytest.mark.parametrize("fmt", [ref.E4M3, ref.E5M2])
def test_reference_scale_rule(fmt):
    """One block each: the scale maps the largest magnitude into (TOP / 2, TOP], ends of the range apart."""
    top = ref.TOP[fmt]
    for a, want in ((top, 127), (np.nextafter(top, 1e9), 128), (top / 2, 126), (0.0, 0), (2.0 ** -149, 0), (top * 2.0 ** -127, 0), (np.inf, 255), (np.nan, 255)):
        assert ref.scale_bytes(np.array([[0.0, a]]), 16, fmt)[0, 0] == want


def test_reference_gradients_are_those_of_the_reference_operators():
    """The gradient formulas against central differences in binary64 (step 1e-6: truncation 1e-12, rounding 1e-10)."""
    rng = np.random.default_rng(3)
    h, w, dy = rng.standard_normal((3, 9)), rng.standard_normal(9), rng.standard_normal((3, 9))
    eps, d = 1e-5, 1e-6
    loss = lambda h, w: (ref.rmsnorm(h, w, eps)[0] * dy).sum()  # noqa: E731
    dx, dw = ref.rmsnorm_backward(dy, w, h, ref.rmsnorm(h, w, eps)[1])[:2]
    for i in np.ndindex(3, 9):
        p = np.zeros((3, 9))
        p[i] = d
        assert abs((loss(h + p, w) - loss(h - p, w)) / (2 * d) - dx[i]) < 1e-7
    for j in range(9):
        p = np.zeros(9)
        p[j] = d
        assert abs((loss(h, w + p) - loss(h, w - p)) / (2 * d) - dw[j]) < 1e-7
    g, u = 3 * rng.standard_normal((3, 9)), rng.standard_normal((3, 9))
    dg, du = ref.swiglu_backward(dy, g, u)
    assert np.abs((ref.swiglu(g + d, u) - ref.swiglu(g - d, u)) / (2 * d) * dy - dg).max() < 1e-7
    assert np.abs((ref.swiglu(g, u + d) - ref.swiglu(g, u - d)) / (2 * d) * dy - du).max() < 1e-7
