// Root-mean-square norm of rows with the residual's addition and an output in block-scaled 8 bits, and its gradient from the 8-bit
// checkpoint of the sum.
#include "mxq_act8.cuh"

namespace mxq {

// Sum over a CTA of up to 1024 threads, the same bits in every thread: a shuffle tree in each warp, then the warps' sums in order.
// scratch: 32 floats that nothing else uses between the barrier inside and the next one.
__device__ __forceinline__ float cta_sum(float v, float* scratch) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return v;
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < warps ? scratch[threadIdx.x & 31] : 0.0f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

struct NormShape {
    size_t rows, cols, blocks;
    int lanes, lanes_log2;
};

__device__ __forceinline__ int left_of(size_t cols, size_t vec) {
    if (vec * kVec >= cols) return 0;
    const size_t n = cols - vec * kVec;
    return n < (size_t)kVec ? (int)n : kVec;
}

// One CTA a row; a thread holds K vectors of it.
template <int DT, int FMT, bool VEC, int K>
__global__ void __launch_bounds__(1024) k_add_rmsnorm8(const void* x, size_t x_stride, const void* residual, size_t r_stride, const void* weight, int weight_dtype, float eps,
                                                       NormShape n, void* out_sum, size_t s_stride, Held8 out, Held8 kept, float* out_rstd) {
    __shared__ float scratch[32];
    wait_for_prior_grid();
    release_dependents();
    const size_t row = blockIdx.x;
    float h[K][kVec];
    float sq = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const size_t vec = (size_t)k * blockDim.x + threadIdx.x;
        const int left = left_of(n.cols, vec);
        load8<DT, VEC>(x, row * x_stride + vec * kVec, left, h[k]);
        if (residual) {
            float r[kVec];
            load8<DT, VEC>(residual, row * r_stride + vec * kVec, left, r);
#pragma unroll
            for (int j = 0; j < kVec; ++j) h[k][j] += r[j];
            round8<DT>(h[k]);
            store8<DT, VEC>(out_sum, row * s_stride + vec * kVec, left, h[k]);
        }
#pragma unroll
        for (int j = 0; j < kVec; ++j) sq = __fmaf_rn(h[k][j], h[k][j], sq);
        if (kept.codes) put_held8<FMT, VEC>(kept, h[k], row, vec, n.cols, n.blocks, n.lanes, n.lanes_log2, left);
    }
    sq = cta_sum(sq, scratch);
    const float rstd = 1.0f / sqrtf(sq / (float)n.cols + eps);
    if (out_rstd && threadIdx.x == 0) out_rstd[row] = rstd;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const size_t vec = (size_t)k * blockDim.x + threadIdx.x;
        const int left = left_of(n.cols, vec);
        float w[kVec];
        if (weight_dtype == kBF16) load8<kBF16, VEC>(weight, vec * kVec, left, w);
        else load8<kF32, VEC>(weight, vec * kVec, left, w);
#pragma unroll
        for (int j = 0; j < kVec; ++j) w[j] *= h[k][j] * rstd;
        put_held8<FMT, VEC>(out, w, row, vec, n.cols, n.blocks, n.lanes, n.lanes_log2, left);
    }
}

// A CTA takes every gridDim.x-th row; a thread holds the same K vectors of each and adds up its columns' part of the weight's gradient.
template <int DT, int FMT, bool VEC, int K>
__global__ void __launch_bounds__(1024) k_add_rmsnorm8_backward(const void* dy, size_t dy_stride, const void* dsum, size_t ds_stride, const void* weight, int weight_dtype,
                                                                Held8 kept, const float* rstd, NormShape n, void* dx, size_t dx_stride, float* parts) {
    __shared__ float scratch[2][32];
    wait_for_prior_grid();
    release_dependents();
    float dw[K][kVec];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < kVec; ++j) dw[k][j] = 0.0f;
    int turn = 0;
    for (size_t row = blockIdx.x; row < n.rows; row += gridDim.x, turn ^= 1) {
        const float rs = rstd[row];
        float wd[K][kVec], xh[K][kVec];
        float dot = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const size_t vec = (size_t)k * blockDim.x + threadIdx.x;
            const int left = left_of(n.cols, vec);
            load8<DT, VEC>(dy, row * dy_stride + vec * kVec, left, wd[k]);
            get_held8<FMT, VEC>(kept, xh[k], row, vec, n.cols, n.blocks, n.lanes_log2, left);
            float w[kVec];
            if (weight_dtype == kBF16) load8<kBF16, VEC>(weight, vec * kVec, left, w);
            else load8<kF32, VEC>(weight, vec * kVec, left, w);
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                xh[k][j] *= rs;
                dw[k][j] = __fmaf_rn(wd[k][j], xh[k][j], dw[k][j]);
                wd[k][j] *= w[j];
                dot = __fmaf_rn(wd[k][j], xh[k][j], dot);
            }
        }
        const float c = cta_sum(dot, scratch[turn]) / (float)n.cols;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const size_t vec = (size_t)k * blockDim.x + threadIdx.x;
            const int left = left_of(n.cols, vec);
            float ds[kVec];
            if (dsum) load8<DT, VEC>(dsum, row * ds_stride + vec * kVec, left, ds);
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                const float t = __fmaf_rn(-xh[k][j], c, wd[k][j]);
                wd[k][j] = dsum ? __fmaf_rn(t, rs, ds[j]) : t * rs;
            }
            store8<DT, VEC>(dx, row * dx_stride + vec * kVec, left, wd[k]);
        }
    }
    if (parts) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const size_t vec = (size_t)k * blockDim.x + threadIdx.x;
            store8<kF32, VEC>(parts, blockIdx.x * n.cols + vec * kVec, left_of(n.cols, vec), dw[k]);
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

// Threads and vectors a thread for rows of `vectors` vectors (padded to whole blocks): as few vectors as 1024 threads allow.
static void split_row(size_t vectors, unsigned& threads, int& K) {
    K = vectors <= 1024 ? 1 : vectors <= 2048 ? 2 : 4;
    threads = (unsigned)(((vectors + K - 1) / K + 31) / 32 * 32);
}

static NormShape norm_shape(size_t rows, size_t cols, int B) {
    NormShape n;
    n.rows = rows, n.cols = cols, n.blocks = (cols + B - 1) / B;
    n.lanes = B / kVec;
    n.lanes_log2 = n.lanes == 2 ? 1 : n.lanes == 4 ? 2 : n.lanes == 8 ? 3 : 4;
    return n;
}

template <typename F>
static cudaError_t pick(int dtype, int fmt, bool vec, int K, F f) {
    using std::integral_constant;
    auto by_k = [&](auto dt, auto fm, auto v) {
        return K == 1 ? f(dt, fm, v, integral_constant<int, 1>{}) : K == 2 ? f(dt, fm, v, integral_constant<int, 2>{}) : f(dt, fm, v, integral_constant<int, 4>{});
    };
    auto by_vec = [&](auto dt, auto fm) { return vec ? by_k(dt, fm, integral_constant<bool, true>{}) : by_k(dt, fm, integral_constant<bool, false>{}); };
    auto by_fmt = [&](auto dt) { return fmt == kE4M3 ? by_vec(dt, integral_constant<int, kE4M3>{}) : by_vec(dt, integral_constant<int, kE5M2>{}); };
    return dtype == kBF16 ? by_fmt(integral_constant<int, kBF16>{}) : by_fmt(integral_constant<int, kF32>{});
}

cudaError_t launch_add_rmsnorm8(const Wide8& x, const Wide8& residual, const void* weight, int weight_dtype, size_t rows, size_t cols, float eps, int B, int dtype, int fmt,
                                const Wide8& out_sum, const Held8& out, const Held8& kept, float* out_rstd, cudaStream_t s) {
    const NormShape n = norm_shape(rows, cols, B);
    unsigned threads;
    int K;
    split_row(n.blocks * n.lanes, threads, K);
    const bool vec = wide_vec(x, cols, dtype) && (!residual.p || (wide_vec(residual, cols, dtype) && wide_vec(out_sum, cols, dtype))) && ((uintptr_t)weight & 15) == 0;
    return pick(dtype, fmt, vec, K, [&](auto dt, auto fm, auto v, auto k) {
        count_launch();
        return launch_pdl(k_add_rmsnorm8<dt(), fm(), v(), k()>, (unsigned)rows, threads, 0, s, (const void*)x.p, x.stride, (const void*)residual.p, residual.stride, weight,
                          weight_dtype, eps, n, out_sum.p, out_sum.stride, out, kept, out_rstd);
    });
}

cudaError_t launch_add_rmsnorm8_backward(const Wide8& dy, const Wide8& dsum, const void* weight, int weight_dtype, const Held8& kept, const float* rstd, size_t rows, size_t cols,
                                         int B, int dtype, int fmt, const Wide8& dx, float* dweight, float* parts, cudaStream_t s) {
    const NormShape n = norm_shape(rows, cols, B);
    unsigned threads;
    int K;
    split_row(n.blocks * n.lanes, threads, K);
    const bool vec = wide_vec(dy, cols, dtype) && (!dsum.p || wide_vec(dsum, cols, dtype)) && wide_vec(dx, cols, dtype) && ((uintptr_t)weight & 15) == 0;
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    size_t ctas = (size_t)sm_count(dev) * 2;
    if (ctas > rows) ctas = rows;
    if (ctas > (size_t)kNorm8Parts) ctas = kNorm8Parts;
    err = pick(dtype, fmt, vec, K, [&](auto dt, auto fm, auto v, auto k) {
        count_launch();
        return launch_pdl(k_add_rmsnorm8_backward<dt(), fm(), v(), k()>, (unsigned)ctas, threads, 0, s, (const void*)dy.p, dy.stride, (const void*)dsum.p, dsum.stride, weight,
                          weight_dtype, kept, rstd, n, dx.p, dx.stride, dweight ? parts : (float*)nullptr);
    });
    if (err != cudaSuccess || !dweight) return err;
    count_launch();
    return launch_pdl(k_rmsnorm8_dweight, (unsigned)((cols + 31) / 32), 256, 0, s, (const float*)parts, (int)ctas, cols, dweight);
}

}  // namespace mxq
