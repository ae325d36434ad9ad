// Element-wise operators on block-scaled 8-bit activations: quantize, de-quantize, gated activation and its gradient.
#include "mxq_act8.cuh"

namespace mxq {

// Vectors are numbered row by row, each row padded to whole blocks; a thread takes one.  Two or four of them a thread, with all loads first,
// cost resident threads and were slower: store 8192 x 4096 16.2 us with one, 17.1 with two, 16.8 with four, load 8192 x 14336 53.1, 66.2, 71.9.
struct Rows8 {
    size_t rows, cols, blocks;   // blocks: per row
    size_t vectors;              // per row, padded to whole blocks
    int lanes_log2;

    template <int V>
    __device__ __forceinline__ Place at(size_t slot) const {
        Place t;
        if (rows == 1) {
            t.row = 0, t.vec = slot;
        } else if (((slot | vectors) >> 32) == 0) {
            t.row = (uint32_t)slot / (uint32_t)vectors;
            t.vec = (uint32_t)slot - (uint32_t)t.row * (uint32_t)vectors;
        } else {
            t.row = slot / vectors, t.vec = slot % vectors;
        }
        t.left = t.row < rows ? left_of(cols, t.vec * V) : 0;
        return t;
    }
};

static Rows8 rows8(size_t rows, size_t cols, int B, int dtype, bool flat) {
    Rows8 r;
    if (flat) {
        cols *= rows;
        rows = 1;
    }
    r.rows = rows, r.cols = cols;
    r.blocks = (cols + B - 1) / B;
    r.lanes_log2 = lanes_log2_of(B, dtype);
    r.vectors = r.blocks << r.lanes_log2;
    return r;
}

static unsigned grid_of(const Rows8& r) { return (unsigned)((r.rows * r.vectors + kThreads - 1) / kThreads); }

template <int DT, int FMT, int FIT>
__global__ void __launch_bounds__(kThreads) k_quantize8(const void* x, size_t stride, Rows8 r, Held8 out) {
    constexpr int V = vec_elems(DT);
    wait_for_prior_grid();
    release_dependents();
    const Place t = r.at<V>((size_t)blockIdx.x * kThreads + threadIdx.x);
    float v[V];
    load_wide<DT, FIT>(x, t.row * stride + t.vec * V, t.left, v);
    put_held<FMT, FIT>(out, v, t, r.cols, r.blocks, r.lanes_log2);
}

template <int DT, int FMT, int FIT>
__global__ void __launch_bounds__(kThreads) k_dequantize8(Held8 in, Rows8 r, void* out, size_t stride) {
    constexpr int V = vec_elems(DT);
    wait_for_prior_grid();
    release_dependents();
    const Place t = r.at<V>((size_t)blockIdx.x * kThreads + threadIdx.x);
    float v[V];
    get_held<FMT, FIT>(in, v, t, r.cols, r.blocks, r.lanes_log2);
    store_wide<DT, FIT>(out, t.row * stride + t.vec * V, t, v);
}

// 1 / (1 + exp(-g)) of two values.  The reciprocal's argument is 1 at least; where exp(-g) passes 2^126 (g < -87.3) the sigmoid is taken
// as zero.  In fp32 exp() is expf().  bf16 tensors, whose results are rounded to 8 significant bits at most, take 2^(-g log2 e) with the
// exponent rounded to binary32: off by (1.3 |g| + 4) 2^-24 relative where g is negative and by less where it is positive, 1e-6 at
// g = -16; a third fewer instructions in kernels that the issue slots bound.
template <int DT>
__device__ __forceinline__ float2 sigmoid2(float2 g) {
    float2 e, r;
    if constexpr (DT == kBF16) {
        const float2 t = mul2(g, make_float2(-1.4426950408889634f, -1.4426950408889634f));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(t.x));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(t.y));
    } else {
        e = make_float2(expf(-g.x), expf(-g.y));
    }
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(1.0f + e.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(1.0f + e.y));
    return r;
}

// Registers for five (six) CTAs an SM: 8192 x 14336 with the checkpoints 129 us (four 132, six 140), without 93 with five or six (four 100), in a few passes
// one after the other, like the figures below; a tenth of a second of them meets the power limit and takes 139 and 103.  Shifted bf16 rows, 8192 x 3075: with
// the checkpoints four, 55 (one 63, five 60), without six, 32 (one 38, five 35).
template <int DT, int FMT, int FIT, bool KEEP>
__global__ void __launch_bounds__(kThreads, KEEP ? (FIT == kAny ? 4 : 5) : 6) k_swiglu8(const void* gate, size_t gate_stride, const void* up, size_t up_stride, Rows8 r, Held8 out, Held8 out_gate, Held8 out_up) {
    constexpr int V = vec_elems(DT);
    wait_for_prior_grid();
    release_dependents();
    const Place t = r.at<V>((size_t)blockIdx.x * kThreads + threadIdx.x);
    float g[V], p[V];
    load_wide<DT, FIT>(gate, t.row * gate_stride + t.vec * V, t.left, g);
    load_wide<DT, FIT>(up, t.row * up_stride + t.vec * V, t.left, p);
    if constexpr (KEEP) {
        put_held<FMT, FIT>(out_gate, g, t, r.cols, r.blocks, r.lanes_log2);
        put_held<FMT, FIT>(out_up, p, t, r.cols, r.blocks, r.lanes_log2);
    }
#pragma unroll
    for (int j = 0; j < V; j += 2) {
        const float2 gg = make_float2(g[j], g[j + 1]);
        const float2 a = mul2(mul2(gg, sigmoid2<DT>(gg)), make_float2(p[j], p[j + 1]));
        g[j] = a.x, g[j + 1] = a.y;
    }
    put_held<FMT, FIT>(out, g, t, r.cols, r.blocks, r.lanes_log2);
}

// Six CTAs an SM: 8192 x 14336 150 us (five 154, four 175; 163 under the power limit); shifted rows, 8192 x 3075: of bf16 five, 58 (one 75, four 64), of
// fp32 six, 89 (five 98).
template <int DT, int FMT, int FIT>
__global__ void __launch_bounds__(kThreads, FIT == kAny && DT == kBF16 ? 5 : 6) k_swiglu8_backward(const void* dy, size_t dy_stride, Held8 gate, Held8 up, Rows8 r, void* dgate, size_t dgate_stride, void* dup, size_t dup_stride) {
    constexpr int V = vec_elems(DT);
    wait_for_prior_grid();
    release_dependents();
    const Place t = r.at<V>((size_t)blockIdx.x * kThreads + threadIdx.x);
    float d[V], g[V], p[V];
    load_wide<DT, FIT>(dy, t.row * dy_stride + t.vec * V, t.left, d);
    get_held<FMT, FIT>(gate, g, t, r.cols, r.blocks, r.lanes_log2);
    get_held<FMT, FIT>(up, p, t, r.cols, r.blocks, r.lanes_log2);
#pragma unroll
    for (int j = 0; j < V; j += 2) {
        const float2 gg = make_float2(g[j], g[j + 1]), s = sigmoid2<DT>(gg);
        const float2 ds = mul2(make_float2(d[j], d[j + 1]), s);
        const float2 du = mul2(ds, gg);
        const float2 slope = fma2(gg, make_float2(1.0f - s.x, 1.0f - s.y), make_float2(1.0f, 1.0f));
        const float2 dg = mul2(mul2(ds, make_float2(p[j], p[j + 1])), slope);
        d[j] = du.x, d[j + 1] = du.y;
        g[j] = dg.x, g[j + 1] = dg.y;
    }
    store_wide<DT, FIT>(dgate, t.row * dgate_stride + t.vec * V, t, g);
    store_wide<DT, FIT>(dup, t.row * dup_stride + t.vec * V, t, d);
}

template <typename F>
static cudaError_t pick(int dtype, int fmt, int fit, F f) {
    using std::integral_constant;
    auto by_fit = [&](auto dt, auto fm) {
        return fit == kWhole  ? f(dt, fm, integral_constant<int, kWhole>{})
               : fit == kHalf ? f(dt, fm, integral_constant<int, kHalf>{})
                              : f(dt, fm, integral_constant<int, kAny>{});
    };
    auto by_fmt = [&](auto dt) { return fmt == kE4M3 ? by_fit(dt, integral_constant<int, kE4M3>{}) : by_fit(dt, integral_constant<int, kE5M2>{}); };
    return dtype == kBF16 ? by_fmt(integral_constant<int, kBF16>{}) : by_fmt(integral_constant<int, kF32>{});
}

cudaError_t launch_quantize8(const Wide8& x, size_t rows, size_t cols, int B, int dtype, int fmt, const Held8& out, cudaStream_t s) {
    const Rows8 r = rows8(rows, cols, B, dtype, x.stride == cols && cols % B == 0);
    return pick(dtype, fmt, fit_of(x, cols, dtype), [&](auto dt, auto fm, auto fit) {
        count_launch();
        return launch_pdl(k_quantize8<dt(), fm(), fit()>, grid_of(r), kThreads, 0, s, (const void*)x.p, x.stride, r, out);
    });
}

cudaError_t launch_dequantize8(const Held8& in, size_t rows, size_t cols, int B, int dtype, int fmt, const Wide8& out, cudaStream_t s) {
    const Rows8 r = rows8(rows, cols, B, dtype, out.stride == cols && cols % B == 0);
    return pick(dtype, fmt, fit_of(out, cols, dtype), [&](auto dt, auto fm, auto fit) {
        count_launch();
        return launch_pdl(k_dequantize8<dt(), fm(), fit()>, grid_of(r), kThreads, 0, s, in, r, out.p, out.stride);
    });
}

cudaError_t launch_swiglu8(const Wide8& gate, const Wide8& up, size_t rows, size_t cols, int B, int dtype, int fmt, const Held8& out, const Held8& out_gate,
                           const Held8& out_up, cudaStream_t s) {
    const Rows8 r = rows8(rows, cols, B, dtype, gate.stride == cols && up.stride == cols && cols % B == 0);
    return pick(dtype, fmt, worst_fit(fit_of(gate, cols, dtype), fit_of(up, cols, dtype)), [&](auto dt, auto fm, auto fit) {
        count_launch();
        auto kernel = out_gate.codes ? k_swiglu8<dt(), fm(), fit(), true> : k_swiglu8<dt(), fm(), fit(), false>;
        return launch_pdl(kernel, grid_of(r), kThreads, 0, s, (const void*)gate.p, gate.stride, (const void*)up.p, up.stride, r, out, out_gate, out_up);
    });
}

cudaError_t launch_swiglu8_backward(const Wide8& dy, const Held8& gate, const Held8& up, size_t rows, size_t cols, int B, int dtype, int fmt, const Wide8& dgate,
                                    const Wide8& dup, cudaStream_t s) {
    const Rows8 r = rows8(rows, cols, B, dtype, dy.stride == cols && dgate.stride == cols && dup.stride == cols && cols % B == 0);
    return pick(dtype, fmt, worst_fit(fit_of(dy, cols, dtype), worst_fit(fit_of(dgate, cols, dtype), fit_of(dup, cols, dtype))), [&](auto dt, auto fm, auto fit) {
        count_launch();
        return launch_pdl(k_swiglu8_backward<dt(), fm(), fit()>, grid_of(r), kThreads, 0, s, (const void*)dy.p, dy.stride, gate, up, r, dgate.p, dgate.stride, dup.p,
                          dup.stride);
    });
}

}  // namespace mxq
