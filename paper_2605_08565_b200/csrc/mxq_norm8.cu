// Root-mean-square norm of rows with the residual's addition and an output in block-scaled 8 bits, and its gradient from the 8-bit
// checkpoint of the sum.
#include "mxq_act8.cuh"

namespace mxq {

// How rows are laid over threads.
//   group > 0: a row's vectors fit a warp.  Every `group` lanes (a power of two) hold a row, a CTA 256 / group rows.
//   group = 0: a CTA holds a row, a thread K vectors of it, blockDim.x apart.
struct NormShape {
    size_t rows, cols, blocks;
    int lanes_log2, group;
};

// Sum over the threads that hold a row, the same bits in all of them: a shuffle tree in each warp, then one over the warps' sums.
// scratch: 32 floats that nothing else uses between the barrier inside and the next one.
template <bool SMALL>
__device__ __forceinline__ float row_sum(float v, int group, float* scratch) {
    if constexpr (SMALL) {
        for (int o = group >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
        return v;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return v;
    const int top = 32 - __clz(warps - 1);   // log2 of the warps, rounded up
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    const int i = threadIdx.x & ((1 << top) - 1);
    v = i < warps ? scratch[i] : 0.0f;
    for (int o = 1 << (top - 1); o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}

template <int V, bool SMALL>
__device__ __forceinline__ Place place_of(const NormShape& n, size_t row, int k) {
    Place t;
    t.row = row;
    t.vec = SMALL ? threadIdx.x & (n.group - 1) : (size_t)k * blockDim.x + threadIdx.x;
    t.left = row < n.rows ? (long long)n.cols - (long long)(t.vec * V) : 0;
    return t;
}

template <bool VEC, int V>
__device__ __forceinline__ void load_weight(const void* weight, int weight_dtype, const Place& t, float (&w)[V]) {
    if (weight_dtype == kBF16) load_wide<kBF16, VEC>(weight, t.vec * V, t.left, w);
    else load_wide<kF32, VEC>(weight, t.vec * V, t.left, w);
}

template <int DT, int FMT, bool VEC, int K, bool SMALL>
__global__ void __launch_bounds__(SMALL ? 256 : 1024) k_add_rmsnorm8(const void* x, size_t x_stride, const void* residual, size_t r_stride, const void* weight, int weight_dtype,
                                                                     float eps, NormShape n, void* out_sum, size_t s_stride, Held8 out, Held8 kept, float* out_rstd) {
    constexpr int V = vec_elems(DT);
    __shared__ float scratch[32];
    wait_for_prior_grid();
    release_dependents();
    const size_t row = SMALL ? (size_t)blockIdx.x * (256 / n.group) + threadIdx.x / n.group : blockIdx.x;
    float h[K][V];
    float sq = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const Place t = place_of<V, SMALL>(n, row, k);
        load_wide<DT, VEC>(x, row * x_stride + t.vec * V, t.left, h[k]);
        if (residual) {
            float r[V];
            load_wide<DT, VEC>(residual, row * r_stride + t.vec * V, t.left, r);
#pragma unroll
            for (int j = 0; j < V; ++j) h[k][j] += r[j];
            uint32_t w[V * elem_bytes(DT) / 4];
            pack<DT, V>(h[k], w);
            unpack<DT, V>(w, h[k]);
            store_wide<DT, VEC>(out_sum, row * s_stride + t.vec * V, t, h[k]);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) sq = __fmaf_rn(h[k][j], h[k][j], sq);
        if (kept.codes) put_held<FMT, VEC>(kept, h[k], t, n.cols, n.blocks, n.lanes_log2);
    }
    sq = row_sum<SMALL>(sq, n.group, scratch);
    const float rstd = 1.0f / sqrtf(sq / (float)n.cols + eps);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const Place t = place_of<V, SMALL>(n, row, k);
        if (out_rstd && t.vec == 0 && row < n.rows) out_rstd[row] = rstd;
        float w[V];
        load_weight<VEC, V>(weight, weight_dtype, t, w);
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const float2 y = mul2(mul2(make_float2(h[k][j], h[k][j + 1]), make_float2(rstd, rstd)), make_float2(w[j], w[j + 1]));
            w[j] = y.x, w[j + 1] = y.y;
        }
        put_held<FMT, VEC>(out, w, t, n.cols, n.blocks, n.lanes_log2);
    }
}

// A CTA takes every gridDim.x-th row (or group of rows); a thread holds the same K vectors of each and adds up its columns' part of the
// weight's gradient.
template <int DT, int FMT, bool VEC, int K, bool SMALL>
__global__ void __launch_bounds__(SMALL ? 256 : 1024) k_add_rmsnorm8_backward(const void* dy, size_t dy_stride, const void* dsum, size_t ds_stride, const void* weight,
                                                                              int weight_dtype, Held8 kept, const float* rstd, NormShape n, void* dx, size_t dx_stride,
                                                                              float* parts) {
    constexpr int V = vec_elems(DT);
    __shared__ float scratch[2][32];
    __shared__ float by_group[SMALL ? 256 * V : 1];
    wait_for_prior_grid();
    release_dependents();
    float dw[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) dw[k][j] = 0.0f;
    const size_t rows_cta = SMALL ? 256 / n.group : 1;
    int turn = 0;
    for (size_t first = blockIdx.x * rows_cta; first < n.rows; first += gridDim.x * rows_cta, turn ^= 1) {
        const size_t row = SMALL ? first + threadIdx.x / n.group : first;
        const float rs = row < n.rows ? rstd[row] : 0.0f;
        float wd[K][V], xh[K][V];
        float dot = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const Place t = place_of<V, SMALL>(n, row, k);
            load_wide<DT, VEC>(dy, row * dy_stride + t.vec * V, t.left, wd[k]);
            get_held<FMT, VEC>(kept, xh[k], t, n.cols, n.blocks, n.lanes_log2);
            float w[V];
            load_weight<VEC, V>(weight, weight_dtype, t, w);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                xh[k][j] *= rs;
                dw[k][j] = __fmaf_rn(wd[k][j], xh[k][j], dw[k][j]);
                wd[k][j] *= w[j];
                dot = __fmaf_rn(wd[k][j], xh[k][j], dot);
            }
        }
        const float c = row_sum<SMALL>(dot, n.group, scratch[turn]) / (float)n.cols;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const Place t = place_of<V, SMALL>(n, row, k);
            float ds[V];
            if (dsum) load_wide<DT, VEC>(dsum, row * ds_stride + t.vec * V, t.left, ds);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float e = __fmaf_rn(-xh[k][j], c, wd[k][j]);
                wd[k][j] = dsum ? __fmaf_rn(e, rs, ds[j]) : e * rs;
            }
            store_wide<DT, VEC>(dx, row * dx_stride + t.vec * V, t, wd[k]);
        }
    }
    if (!parts) return;
    if constexpr (SMALL) {   // the groups' sums in order
#pragma unroll
        for (int j = 0; j < V; ++j) by_group[(threadIdx.x / n.group * V + j) * n.group + (threadIdx.x & (n.group - 1))] = dw[0][j];
        __syncthreads();
        for (unsigned i = threadIdx.x; i < (unsigned)n.group * V; i += 256) {
            const unsigned vec = i / V, j = i % V;
            if (i >= n.cols) continue;
            float s = 0.0f;
            for (int g = 0; g < 256 / n.group; ++g) s += by_group[(g * V + j) * n.group + vec];
            parts[blockIdx.x * n.cols + i] = s;
        }
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const Place t = place_of<V, SMALL>(n, 0, k);
            store_wide<kF32, VEC>(parts, blockIdx.x * n.cols + t.vec * V, t, dw[k]);
        }
    }
}

// dweight[c] = sum over the parts, in a fixed order: each of 8 warps every eighth part, then the warps' sums in order.
__global__ void __launch_bounds__(256) k_rmsnorm8_dweight(const float* parts, int n_parts, size_t cols, float* dweight) {
    __shared__ float sums[8][32];
    wait_for_prior_grid();
    release_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const size_t col = (size_t)blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (col < cols)
        for (int p = warp; p < n_parts; p += 8) s += parts[(size_t)p * cols + col];
    sums[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && col < cols) {
#pragma unroll
        for (int w = 1; w < 8; ++w) s += sums[w][lane];
        dweight[col] = s;
    }
}

// Shape, threads of a CTA and vectors of a thread for rows of this kind.
struct NormLaunch {
    NormShape n;
    unsigned threads;
    int K;
    size_t rows_cta;
};
static NormLaunch norm_launch(size_t rows, size_t cols, int B, int dtype) {
    NormLaunch l;
    l.n.rows = rows, l.n.cols = cols, l.n.blocks = (cols + B - 1) / B;
    l.n.lanes_log2 = lanes_log2_of(B, dtype);
    const size_t vectors = l.n.blocks << l.n.lanes_log2;
    l.n.group = 0;
    l.K = 1;
    l.rows_cta = 1;
    if (vectors <= 32) {
        l.n.group = 1;
        while ((size_t)l.n.group < vectors) l.n.group *= 2;
        l.threads = 256;
        l.rows_cta = 256 / l.n.group;
    } else {
        while (vectors > (size_t)l.K * 1024) l.K *= 2;
        l.threads = (unsigned)(((vectors + l.K - 1) / l.K + 31) / 32 * 32);
    }
    return l;
}

template <typename F>
static cudaError_t pick(int dtype, int fmt, bool vec, const NormLaunch& l, F f) {
    using std::integral_constant;
    using Yes = integral_constant<bool, true>;
    using No = integral_constant<bool, false>;
    auto by_k = [&](auto dt, auto fm, auto v) {
        if (l.n.group) return f(dt, fm, v, integral_constant<int, 1>{}, Yes{});
        return l.K == 1   ? f(dt, fm, v, integral_constant<int, 1>{}, No{})
               : l.K == 2 ? f(dt, fm, v, integral_constant<int, 2>{}, No{})
                          : f(dt, fm, v, integral_constant<int, 4>{}, No{});
    };
    auto by_vec = [&](auto dt, auto fm) { return vec ? by_k(dt, fm, Yes{}) : by_k(dt, fm, No{}); };
    auto by_fmt = [&](auto dt) { return fmt == kE4M3 ? by_vec(dt, integral_constant<int, kE4M3>{}) : by_vec(dt, integral_constant<int, kE5M2>{}); };
    return dtype == kBF16 ? by_fmt(integral_constant<int, kBF16>{}) : by_fmt(integral_constant<int, kF32>{});
}

cudaError_t launch_add_rmsnorm8(const Wide8& x, const Wide8& residual, const void* weight, int weight_dtype, size_t rows, size_t cols, float eps, int B, int dtype, int fmt,
                                const Wide8& out_sum, const Held8& out, const Held8& kept, float* out_rstd, cudaStream_t s) {
    const NormLaunch l = norm_launch(rows, cols, B, dtype);
    const bool vec = wide_vec(x, cols, dtype) && (!residual.p || (wide_vec(residual, cols, dtype) && wide_vec(out_sum, cols, dtype))) && ((uintptr_t)weight & 31) == 0;
    return pick(dtype, fmt, vec, l, [&](auto dt, auto fm, auto v, auto k, auto small) {
        count_launch();
        return launch_pdl(k_add_rmsnorm8<dt(), fm(), v(), k(), small()>, (unsigned)((rows + l.rows_cta - 1) / l.rows_cta), l.threads, 0, s, (const void*)x.p, x.stride,
                          (const void*)residual.p, residual.stride, weight, weight_dtype, eps, l.n, out_sum.p, out_sum.stride, out, kept, out_rstd);
    });
}

cudaError_t launch_add_rmsnorm8_backward(const Wide8& dy, const Wide8& dsum, const void* weight, int weight_dtype, const Held8& kept, const float* rstd, size_t rows, size_t cols,
                                         int B, int dtype, int fmt, const Wide8& dx, float* dweight, float* parts, cudaStream_t s) {
    const NormLaunch l = norm_launch(rows, cols, B, dtype);
    const bool vec = wide_vec(dy, cols, dtype) && (!dsum.p || wide_vec(dsum, cols, dtype)) && wide_vec(dx, cols, dtype) && ((uintptr_t)weight & 31) == 0 &&
                     (!dweight || ((uintptr_t)parts & 31) == 0);
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    size_t ctas = (size_t)sm_count(dev) * 2;
    if (ctas > (rows + l.rows_cta - 1) / l.rows_cta) ctas = (rows + l.rows_cta - 1) / l.rows_cta;
    if (ctas > (size_t)kNorm8Parts) ctas = kNorm8Parts;
    err = pick(dtype, fmt, vec, l, [&](auto dt, auto fm, auto v, auto k, auto small) {
        count_launch();
        return launch_pdl(k_add_rmsnorm8_backward<dt(), fm(), v(), k(), small()>, (unsigned)ctas, l.threads, 0, s, (const void*)dy.p, dy.stride, (const void*)dsum.p, dsum.stride,
                          weight, weight_dtype, kept, rstd, l.n, dx.p, dx.stride, dweight ? parts : (float*)nullptr);
    });
    if (err != cudaSuccess || !dweight) return err;
    count_launch();
    return launch_pdl(k_rmsnorm8_dweight, (unsigned)((cols + 31) / 32), 256, 0, s, (const float*)parts, (int)ctas, cols, dweight);
}

}  // namespace mxq
