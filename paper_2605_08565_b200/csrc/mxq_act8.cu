// Element-wise operators on block-scaled 8-bit activations: quantize, de-quantize, gated activation and its gradient.
#include "mxq_act8.cuh"

namespace mxq {

// Where a thread's vectors lie.  Vectors are numbered row by row, each row padded to whole blocks; a CTA takes U * 256 consecutive
// ones, a thread every 256th of them.
struct Walk {
    size_t row, vec;
};
struct Rows8 {
    size_t rows, cols, blocks;   // blocks: per row
    size_t vectors;              // per row, padded to whole blocks
    size_t step_rows, step_vecs; // 256 vectors further on
    int lanes, lanes_log2;

    __device__ __forceinline__ Walk at(size_t slot) const {
        if (rows == 1) return {0, slot};
        if (((slot | vectors) >> 32) == 0) {
            const uint32_t r = (uint32_t)slot / (uint32_t)vectors;
            return {r, (uint32_t)slot - r * (uint32_t)vectors};
        }
        return {slot / vectors, slot % vectors};
    }
    __device__ __forceinline__ void advance(Walk& w) const {
        w.row += step_rows;
        w.vec += step_vecs;
        if (w.vec >= vectors && rows != 1) {
            w.vec -= vectors;
            ++w.row;
        }
    }
    // Elements from the vector's first one to the end of its row; <= 0: nothing there.
    __device__ __forceinline__ int left(const Walk& w) const {
        if (w.row >= rows || w.vec * kVec >= cols) return 0;
        const size_t n = cols - w.vec * kVec;
        return n < (size_t)kVec ? (int)n : kVec;
    }
};

static Rows8 rows8(size_t rows, size_t cols, int B, bool flat) {
    Rows8 r;
    if (flat) {
        cols *= rows;
        rows = 1;
    }
    r.rows = rows, r.cols = cols;
    r.blocks = (cols + B - 1) / B;
    r.lanes = B / kVec;
    r.lanes_log2 = r.lanes == 2 ? 1 : r.lanes == 4 ? 2 : r.lanes == 8 ? 3 : 4;
    r.vectors = r.blocks * r.lanes;
    r.step_rows = rows == 1 ? 0 : kThreads / r.vectors;
    r.step_vecs = rows == 1 ? kThreads : kThreads % r.vectors;
    return r;
}

template <int U>
static unsigned grid_of(const Rows8& r) {
    const size_t per_cta = (size_t)U * kThreads;
    return (unsigned)((r.rows * r.vectors + per_cta - 1) / per_cta);
}

template <int DT, int FMT, bool VEC, int U>
__global__ void __launch_bounds__(kThreads) k_quantize8(const void* x, size_t stride, Rows8 r, Held8 out) {
    wait_for_prior_grid();
    release_dependents();
    Walk w = r.at((size_t)blockIdx.x * (U * kThreads) + threadIdx.x);
    float v[U][kVec];
    Walk at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        at[u] = w;
        load8<DT, VEC>(x, w.row * stride + w.vec * kVec, r.left(w), v[u]);
        r.advance(w);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) put_held8<FMT, VEC>(out, v[u], at[u].row, at[u].vec, r.cols, r.blocks, r.lanes, r.lanes_log2, r.left(at[u]));
}

template <int DT, int FMT, bool VEC, int U>
__global__ void __launch_bounds__(kThreads) k_dequantize8(Held8 in, Rows8 r, void* out, size_t stride) {
    wait_for_prior_grid();
    release_dependents();
    Walk w = r.at((size_t)blockIdx.x * (U * kThreads) + threadIdx.x);
    float v[U][kVec];
    Walk at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        at[u] = w;
        get_held8<FMT, VEC>(in, v[u], w.row, w.vec, r.cols, r.blocks, r.lanes_log2, r.left(w));
        r.advance(w);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) store8<DT, VEC>(out, at[u].row * stride + at[u].vec * kVec, r.left(at[u]), v[u]);
}

// 1 / (1 + exp(-g)); exp(-g) overflows to infinity for g < -88.7, where the sigmoid is below 2^-126: zero.
__device__ __forceinline__ float sigmoid(float g) { return __fdividef(1.0f, 1.0f + expf(-g)); }

template <int DT, int FMT, bool VEC, bool KEEP, int U>
__global__ void __launch_bounds__(kThreads) k_swiglu8(const void* gate, size_t gate_stride, const void* up, size_t up_stride, Rows8 r, Held8 out, Held8 out_gate, Held8 out_up) {
    wait_for_prior_grid();
    release_dependents();
    Walk w = r.at((size_t)blockIdx.x * (U * kThreads) + threadIdx.x);
    float g[U][kVec], p[U][kVec];
    Walk at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        at[u] = w;
        load8<DT, VEC>(gate, w.row * gate_stride + w.vec * kVec, r.left(w), g[u]);
        load8<DT, VEC>(up, w.row * up_stride + w.vec * kVec, r.left(w), p[u]);
        r.advance(w);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int left = r.left(at[u]);
        if constexpr (KEEP) {
            put_held8<FMT, VEC>(out_gate, g[u], at[u].row, at[u].vec, r.cols, r.blocks, r.lanes, r.lanes_log2, left);
            put_held8<FMT, VEC>(out_up, p[u], at[u].row, at[u].vec, r.cols, r.blocks, r.lanes, r.lanes_log2, left);
        }
        float a[kVec];
#pragma unroll
        for (int j = 0; j < kVec; ++j) a[j] = g[u][j] * sigmoid(g[u][j]) * p[u][j];
        put_held8<FMT, VEC>(out, a, at[u].row, at[u].vec, r.cols, r.blocks, r.lanes, r.lanes_log2, left);
    }
}

template <int DT, int FMT, bool VEC, int U>
__global__ void __launch_bounds__(kThreads) k_swiglu8_backward(const void* dy, size_t dy_stride, Held8 gate, Held8 up, Rows8 r, void* dgate, size_t dgate_stride, void* dup, size_t dup_stride) {
    wait_for_prior_grid();
    release_dependents();
    Walk w = r.at((size_t)blockIdx.x * (U * kThreads) + threadIdx.x);
    float d[U][kVec], g[U][kVec], p[U][kVec];
    Walk at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int left = r.left(w);
        at[u] = w;
        load8<DT, VEC>(dy, w.row * dy_stride + w.vec * kVec, left, d[u]);
        get_held8<FMT, VEC>(gate, g[u], w.row, w.vec, r.cols, r.blocks, r.lanes_log2, left);
        get_held8<FMT, VEC>(up, p[u], w.row, w.vec, r.cols, r.blocks, r.lanes_log2, left);
        r.advance(w);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int left = r.left(at[u]);
        float dg[kVec], du[kVec];
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            const float s = sigmoid(g[u][j]), ds = d[u][j] * s;
            dg[j] = ds * p[u][j] * __fmaf_rn(g[u][j], 1.0f - s, 1.0f);
            du[j] = ds * g[u][j];
        }
        store8<DT, VEC>(dgate, at[u].row * dgate_stride + at[u].vec * kVec, left, dg);
        store8<DT, VEC>(dup, at[u].row * dup_stride + at[u].vec * kVec, left, du);
    }
}

template <typename F>
static cudaError_t pick(int dtype, int fmt, bool vec, F f) {
    using std::integral_constant;
    auto by_vec = [&](auto dt, auto fm) { return vec ? f(dt, fm, integral_constant<bool, true>{}) : f(dt, fm, integral_constant<bool, false>{}); };
    auto by_fmt = [&](auto dt) { return fmt == kE4M3 ? by_vec(dt, integral_constant<int, kE4M3>{}) : by_vec(dt, integral_constant<int, kE5M2>{}); };
    return dtype == kBF16 ? by_fmt(integral_constant<int, kBF16>{}) : by_fmt(integral_constant<int, kF32>{});
}

cudaError_t launch_quantize8(const Wide8& x, size_t rows, size_t cols, int B, int dtype, int fmt, const Held8& out, cudaStream_t s) {
    constexpr int U = 2;
    const Rows8 r = rows8(rows, cols, B, x.stride == cols && cols % B == 0);
    return pick(dtype, fmt, wide_vec(x, cols, dtype), [&](auto dt, auto fm, auto vec) {
        count_launch();
        return launch_pdl(k_quantize8<dt(), fm(), vec(), U>, grid_of<U>(r), kThreads, 0, s, (const void*)x.p, x.stride, r, out);
    });
}

cudaError_t launch_dequantize8(const Held8& in, size_t rows, size_t cols, int B, int dtype, int fmt, const Wide8& out, cudaStream_t s) {
    constexpr int U = 2;
    const Rows8 r = rows8(rows, cols, B, out.stride == cols && cols % B == 0);
    return pick(dtype, fmt, wide_vec(out, cols, dtype), [&](auto dt, auto fm, auto vec) {
        count_launch();
        return launch_pdl(k_dequantize8<dt(), fm(), vec(), U>, grid_of<U>(r), kThreads, 0, s, in, r, out.p, out.stride);
    });
}

cudaError_t launch_swiglu8(const Wide8& gate, const Wide8& up, size_t rows, size_t cols, int B, int dtype, int fmt, const Held8& out, const Held8& out_gate,
                           const Held8& out_up, cudaStream_t s) {
    constexpr int U = 1;
    const Rows8 r = rows8(rows, cols, B, gate.stride == cols && up.stride == cols && cols % B == 0);
    return pick(dtype, fmt, wide_vec(gate, cols, dtype) && wide_vec(up, cols, dtype), [&](auto dt, auto fm, auto vec) {
        count_launch();
        auto kernel = out_gate.codes ? k_swiglu8<dt(), fm(), vec(), true, U> : k_swiglu8<dt(), fm(), vec(), false, U>;
        return launch_pdl(kernel, grid_of<U>(r), kThreads, 0, s, (const void*)gate.p, gate.stride, (const void*)up.p, up.stride, r, out, out_gate, out_up);
    });
}

cudaError_t launch_swiglu8_backward(const Wide8& dy, const Held8& gate, const Held8& up, size_t rows, size_t cols, int B, int dtype, int fmt, const Wide8& dgate,
                                    const Wide8& dup, cudaStream_t s) {
    constexpr int U = 1;
    const Rows8 r = rows8(rows, cols, B, dy.stride == cols && dgate.stride == cols && dup.stride == cols && cols % B == 0);
    return pick(dtype, fmt, wide_vec(dy, cols, dtype) && wide_vec(dgate, cols, dtype) && wide_vec(dup, cols, dtype), [&](auto dt, auto fm, auto vec) {
        count_launch();
        return launch_pdl(k_swiglu8_backward<dt(), fm(), vec(), U>, grid_of<U>(r), kThreads, 0, s, (const void*)dy.p, dy.stride, gate, up, r, dgate.p, dgate.stride, dup.p,
                          dup.stride);
    });
}

}  // namespace mxq
