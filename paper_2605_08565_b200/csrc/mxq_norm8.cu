// Root-mean-square norm of rows with the residual's addition and an output in block-scaled 8 bits, and its gradient from the 8-bit
// checkpoint of the sum.
#include <atomic>

#include "mxq_act8.cuh"

namespace mxq {

// How rows are laid over threads.
//   group > 0: a row's vectors fit a warp.  Every `group` lanes (a power of two) hold a row, a CTA 256 / group rows.
//   group = 0: a CTA holds a row, a thread K vectors of it, blockDim.x apart.
struct NormShape {
    size_t rows, cols, blocks;
    int lanes_log2, group;
};

// A vector's part of the weight's gradient, in the kernels that stream rows of whole vectors: 32 bytes at a time where the workspace starts on 32 bytes, else 16
// (8192 x 4096 bf16 42.3 us, and 43.1 with 16 throughout).
template <int V>
__device__ __forceinline__ void store_parts(float* parts, size_t at, const Place& t, const float (&v)[V]) {
    if ((reinterpret_cast<uintptr_t>(parts) & 31u) == 0) store_wide<kF32, kWhole>(parts, at, t, v);
    else store_wide<kF32, kHalf>(parts, at, t, v);
}

// Sum over the CTA, the same bits in every thread.  sums: T / 32 floats, those of warps that the CTA does not have zeros, which nothing else
// uses between the barrier inside and the next one.
template <int T>
__device__ __forceinline__ float cta_sum(float v, float* sums) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = v;
    __syncthreads();
    float4 t = reinterpret_cast<const float4*>(sums)[0];
#pragma unroll
    for (int i = 1; i < (T + 127) / 128; ++i) {
        const float4 u = reinterpret_cast<const float4*>(sums)[i];
        t.x += u.x, t.y += u.y, t.z += u.z, t.w += u.w;
    }
    return (t.x + t.y) + (t.z + t.w);
}

// Sum over the `group` lanes (a power of two) that hold a row.
__device__ __forceinline__ float group_sum(float v, int group) {
    for (int o = group >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}

template <int V, bool SMALL>
__device__ __forceinline__ Place place_of(const NormShape& n, size_t row, int k) {
    Place t;
    t.row = row;
    t.vec = SMALL ? threadIdx.x & (n.group - 1) : (size_t)k * blockDim.x + threadIdx.x;
    t.left = row < n.rows ? left_of(n.cols, t.vec * V) : 0;
    return t;
}

template <int FIT, int V>
__device__ __forceinline__ void load_weight(const void* weight, int weight_dtype, const Place& t, float (&w)[V]) {
    if (weight_dtype == kBF16) load_wide<kBF16, FIT>(weight, t.vec * V, t.left, w);
    else load_wide<kF32, FIT>(weight, t.vec * V, t.left, w);
}

// Registers for three CTAs of 512 threads an SM: 8192 x 4101 bf16 with residual and checkpoint 87 us with one, 76 with three; narrower ones gain nothing.
template <int DT, int FMT, int FIT, int K, bool SMALL, int T>
__global__ void __launch_bounds__(T, T == 512 ? 3 : 1) k_add_rmsnorm8(const void* x, size_t x_stride, const void* residual, size_t r_stride, const void* weight, int weight_dtype,
                                                                     float eps, float inv_cols, NormShape n, void* out_sum, size_t s_stride, Held8 out, Held8 kept, float* out_rstd) {
    constexpr int V = vec_elems(DT);
    __shared__ float4 sums[(T + 127) / 128];
    wait_for_prior_grid();
    release_dependents();
    if constexpr (!SMALL) {
        if (threadIdx.x < sizeof(sums) / 4) reinterpret_cast<float*>(sums)[threadIdx.x] = 0.0f;
        __syncthreads();
    }
    const size_t row = SMALL ? (size_t)blockIdx.x * (256 / n.group) + threadIdx.x / n.group : blockIdx.x;
    float h[K][V];
    float sq = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const Place t = place_of<V, SMALL>(n, row, k);
        load_wide<DT, FIT>(x, row * x_stride + t.vec * V, t.left, h[k]);
        if (residual) {
            float r[V];
            load_wide<DT, FIT>(residual, row * r_stride + t.vec * V, t.left, r);
#pragma unroll
            for (int j = 0; j < V; ++j) h[k][j] += r[j];
            uint32_t w[V * elem_bytes(DT) / 4];
            pack<DT, V>(h[k], w);
            unpack<DT, V>(w, h[k]);
            store_wide<DT, FIT>(out_sum, row * s_stride + t.vec * V, t, h[k]);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) sq = __fmaf_rn(h[k][j], h[k][j], sq);
        if (kept.codes) put_held<FMT, FIT>(kept, h[k], t, n.cols, n.blocks, n.lanes_log2);
    }
    if constexpr (SMALL) sq = group_sum(sq, n.group);
    else sq = cta_sum<T>(sq, reinterpret_cast<float*>(sums));
    const float rstd = rsqrtf(__fmaf_rn(sq, inv_cols, eps));
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const Place t = place_of<V, SMALL>(n, row, k);
        if (out_rstd && t.vec == 0 && row < n.rows) out_rstd[row] = rstd;
        float w[V];
        load_weight<FIT, V>(weight, weight_dtype, t, w);
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const float2 y = mul2(mul2(make_float2(h[k][j], h[k][j + 1]), make_float2(rstd, rstd)), make_float2(w[j], w[j + 1]));
            w[j] = y.x, w[j + 1] = y.y;
        }
        put_held<FMT, FIT>(out, w, t, n.cols, n.blocks, n.lanes_log2);
    }
}

// A CTA takes every gridDim.x-th row (or group of rows); a thread holds the same K vectors of each and adds up its columns' part of the
// weight's gradient.  The workspace's address has no say in which kernel runs (here and below), only in how wide the parts are stored, so that
// dx and dweight are the same bits with any workspace.
// Registers for two CTAs of 512 threads an SM: 8192 x 4101 bf16 146 us with one, 100 with two (8192 x 4104: 101, 58); limiting those of 256 threads to
// three an SM costs 0 to 20 %.
// PARTS: how the parts are stored, FIT or, of whole rows in a workspace that does not start on 32 bytes, kHalf.  (Both in one kernel, behind a branch, cost registers:
// 2048 x 32768 bf16 269 us like this and 373, fp32 391 and 422.)
template <int DT, int FMT, int FIT, int PARTS, int K, bool SMALL, int T>
__global__ void __launch_bounds__(T, T == 512 ? 2 : 1) k_add_rmsnorm8_backward(const void* dy, size_t dy_stride, const void* dsum, size_t ds_stride, const void* weight,
                                                                              int weight_dtype, Held8 kept, const float* rstd, float inv_cols, NormShape n, void* dx, size_t dx_stride,
                                                                              float* parts) {
    constexpr int V = vec_elems(DT);
    __shared__ float4 sums[2][(T + 127) / 128];
    __shared__ float by_group[SMALL ? 256 * V : 1];
    wait_for_prior_grid();
    release_dependents();
    float dw[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) dw[k][j] = 0.0f;
    if constexpr (!SMALL) {
        if (threadIdx.x < sizeof(sums) / 4) reinterpret_cast<float*>(sums)[threadIdx.x] = 0.0f;
        __syncthreads();
    }
    const size_t rows_cta = SMALL ? 256 / n.group : 1;
    int turn = 0;
    for (size_t first = blockIdx.x * rows_cta; first < n.rows; first += gridDim.x * rows_cta, turn ^= 1) {
        const size_t row = SMALL ? first + threadIdx.x / n.group : first;
        const float rs = row < n.rows ? rstd[row] : 0.0f;
        // while this row is worked on, L2 fetches the next one
        if (const size_t after = row + gridDim.x * rows_cta; after < n.rows) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const Place t = place_of<V, SMALL>(n, row, k);
                if (t.left > 0) {
                    prefetch_l2(static_cast<const char*>(dy) + (after * dy_stride + t.vec * V) * elem_bytes(DT));
                    prefetch_l2(kept.codes + after * n.cols + t.vec * V);
                    if (dsum) prefetch_l2(static_cast<const char*>(dsum) + (after * ds_stride + t.vec * V) * elem_bytes(DT));
                }
            }
        }
        float wd[K][V], xh[K][V];
        float dot = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const Place t = place_of<V, SMALL>(n, row, k);
            load_wide<DT, FIT>(dy, row * dy_stride + t.vec * V, t.left, wd[k]);
            get_held<FMT, FIT>(kept, xh[k], t, n.cols, n.blocks, n.lanes_log2);
            float w[V];
            load_weight<FIT, V>(weight, weight_dtype, t, w);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                xh[k][j] *= rs;
                dw[k][j] = __fmaf_rn(wd[k][j], xh[k][j], dw[k][j]);
                wd[k][j] *= w[j];
                dot = __fmaf_rn(wd[k][j], xh[k][j], dot);
            }
        }
        if constexpr (SMALL) dot = group_sum(dot, n.group);
        else dot = cta_sum<T>(dot, reinterpret_cast<float*>(sums[turn]));
        const float c = dot * inv_cols;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const Place t = place_of<V, SMALL>(n, row, k);
            float ds[V];
            if (dsum) load_wide<DT, FIT>(dsum, row * ds_stride + t.vec * V, t.left, ds);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float e = __fmaf_rn(-xh[k][j], c, wd[k][j]);
                wd[k][j] = dsum ? __fmaf_rn(e, rs, ds[j]) : e * rs;
            }
            store_wide<DT, FIT>(dx, row * dx_stride + t.vec * V, t, wd[k]);
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
            store_wide<kF32, PARTS>(parts, blockIdx.x * n.cols + t.vec * V, t, dw[k]);
        }
    }
}

// ---- rows of whole vectors, one vector a thread ------------------------------------------------------------------------------------
// A CTA takes every gridDim.x-th row and copies the next one into shared memory while it works on the present one, so that what is under way
// from memory does not depend on the threads' registers, nor stop while the CTA meets in its barrier.  T: the most threads of a CTA.  Only where the weight's
// vectors are as aligned as the rows: 8192 x 4096 bf16 gradient 43 us, and 62 with a weight on 16 bytes, 83 on 2 (norm 43, 48, 63), from the kernels above.

// The 32 vectors of a warp: each lane copies two of their 64 pieces of 16 bytes, 512 bytes apart, so that an instruction asks for whole
// sectors (each lane its own two pieces: twice the requests to L2).  Piece p lies at p ^ (p >> 3 & 1), without which the lanes' reads of every
// second piece would meet in the banks.
struct WarpCopy {
    bool low, high;   // whether the row has this lane's pieces
    int at;
    __device__ __forceinline__ explicit WarpCopy(long long bytes) {   // of the row, from the warp's first vector on
        const int lane = threadIdx.x & 31;
        low = lane * 16 < bytes;
        high = lane * 16 + 512 < bytes;
        at = lane ^ (lane >> 3 & 1);
    }
    __device__ __forceinline__ void operator()(uint4* to, const char* piece) const {
        if (low) copy_async16(to + at, piece);
        if (high) copy_async16(to + at + 32, piece + 512);
    }
};
__device__ __forceinline__ void read32(const uint4* from, uint32_t (&w)[8]) {
    const int p = 2 * (threadIdx.x & 31), flip = p >> 3 & 1;
    const uint4 a = from[p ^ flip], b = from[(p + 1) ^ flip];
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
}

// Resident CTAs.  With a residual two of 256 threads and the registers that they leave are faster than three with fewer (8192 x 4096, us: with the
// checkpoint too 43.5 / 49.1, else 37.7 / 39.9), two of 384 than one, one of 512 or 1024 is enough.  Without, half as much is under way from memory for each,
// and more of them are better: four of 256 (three: 20.1 -> 19.2, with the checkpoint 24.7 -> 23.8), three of 384 (8192 x 5120 26.5 -> 24.2), two of
// 512 (8192 x 8192 47.0 -> 37.6).
template <int DT, int FMT, bool RES, bool KEEP, int T>
__global__ void __launch_bounds__(T, T == 256 ? (RES ? 2 : 4) : T <= 384 ? (RES ? 2 : 3) : T == 512 && !RES ? 2 : 1)
    k_add_rmsnorm8_rows(const char* x, size_t x_step, const char* residual, size_t r_step, const void* weight, int weight_dtype, float eps, float inv_cols, NormShape n,
                        char* out_sum, size_t s_step, Held8 out, Held8 kept, float* out_rstd) {
    constexpr int V = vec_elems(DT);
    const int n_thr = blockDim.x, slot_size = (RES ? 4 : 2) * n_thr;
    extern __shared__ uint4 ring[];
    __shared__ float4 sums[2][(T + 127) / 128];
    wait_for_prior_grid();
    release_dependents();
    const Place t = place_of<V, false>(n, 0, 0);
    const bool here = t.left > 0, leads = here && (threadIdx.x & ((1u << n.lanes_log2) - 1)) == 0;
    const int warp0 = threadIdx.x & ~31;   // the warp's first vector
    const WarpCopy copy(((long long)n.cols - (long long)warp0 * V) * (32 / V));
    const size_t step = gridDim.x;
    size_t row = blockIdx.x;
    const char* px = x + row * x_step + warp0 * 32 + (threadIdx.x & 31) * 16;
    const char* pr = residual + row * r_step + warp0 * 32 + (threadIdx.x & 31) * 16;
    char* ps = out_sum + row * s_step + threadIdx.x * 32;
    size_t code = row * n.cols + threadIdx.x * V, scale = row * n.blocks + (threadIdx.x >> n.lanes_log2);
    uint4* slot = ring + warp0 * 2;
    uint4* other = slot + slot_size;
    if (threadIdx.x < sizeof(sums) / 4) reinterpret_cast<float*>(sums)[threadIdx.x] = 0.0f;
    copy(slot, px);
    if constexpr (RES) copy(slot + 2 * n_thr, pr);
    copy_commit();
    float w[V];
    load_weight<kWhole, V>(weight, weight_dtype, t, w);
    __syncthreads();   // the zeros in `sums`
    for (int turn = 0; row < n.rows; row += step, turn ^= 1) {
        __syncwarp();   // the other lanes have read what the next copies replace
        px += step * x_step;
        pr += step * r_step;
        if (row + step < n.rows) {
            copy(other, px);
            if constexpr (RES) copy(other + 2 * n_thr, pr);
        }
        copy_commit();
        copy_wait<1>();
        __syncwarp();
        float h[V];
        uint32_t a[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
        if (here) read32(slot, a);
        unpack<DT, V>(a, h);
        if constexpr (RES) {
            float r[V];
            if (here) read32(slot + 2 * n_thr, a);
            unpack<DT, V>(a, r);
#pragma unroll
            for (int j = 0; j < V; ++j) h[j] += r[j];
            pack<DT, V>(h, a);
            unpack<DT, V>(a, h);
            if (here) store256(ps, a);
            ps += step * s_step;
        }
        float2 sq = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < V; j += 2) sq = fma2(make_float2(h[j], h[j + 1]), make_float2(h[j], h[j + 1]), sq);
        uint32_t c[V / 4];
        if constexpr (KEEP) {
            const uint32_t byte = quantize_block<FMT, V>(h, n.lanes_log2, c);
            if (here) store_codes<V>(kept.codes + code, c);
            if (leads) kept.scales[scale] = (uint8_t)byte;
        }
        const float rstd = rsqrtf(__fmaf_rn(cta_sum<T>(sq.x + sq.y, reinterpret_cast<float*>(sums[turn])), inv_cols, eps));
        if (out_rstd && threadIdx.x == 0) out_rstd[row] = rstd;
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const float2 y = mul2(mul2(make_float2(h[j], h[j + 1]), make_float2(rstd, rstd)), make_float2(w[j], w[j + 1]));
            h[j] = y.x, h[j + 1] = y.y;
        }
        const uint32_t byte = quantize_block<FMT, V>(h, n.lanes_log2, c);
        if (here) store_codes<V>(out.codes + code, c);
        if (leads) out.scales[scale] = (uint8_t)byte;
        code += step * n.cols;
        scale += step * n.blocks;
        uint4* const done = slot;
        slot = other;
        other = done;
    }
}

// The scale bytes of a warp's 32 vectors and the row's rstd are copied as well, in the aligned words that hold them (kMeta a warp): a register
// that is loaded one row ahead has to arrive within that row, because the loop's end moves it (8192 x 4096: 62 us, and 47 like this).
constexpr int kMeta = 12;   // 32 bytes off the grid lie in 9 words; rstd; 2 unused

// bf16: 126 to 128 registers a thread at 256 threads and 96 at 320, which its bound asks for: two CTAs an SM (8192 x 5120 62.5 us with one, 51.4 with
// two); 142 to 150 at 384 and 128 at 512: one.  fp32: 96 to 114, 64 at 1024 threads.  Limited to what a third CTA of 256 threads, or a second
// one of 384, leaves, the compiler spills (8192 x 4096 41.9 -> 62.4, 8192 x 6144 68.8 -> 88.8).
template <int DT, int FMT, bool DSUM, int T>
__global__ void __launch_bounds__(T, T <= 320 ? 2 : 1)
    k_add_rmsnorm8_backward_rows(const char* dy, size_t dy_step, const char* dsum, size_t ds_step, const void* weight, int weight_dtype, Held8 kept, const float* rstd,
                                 float inv_cols, NormShape n, char* dx, size_t dx_step, float* parts) {
    constexpr int V = vec_elems(DT), C = DSUM ? 5 : 3;
    const int n_thr = blockDim.x, slot_size = C * n_thr + kMeta * n_thr / 128;
    extern __shared__ uint4 ring[];
    __shared__ float4 sums[2][(T + 127) / 128];
    wait_for_prior_grid();
    release_dependents();
    const Place t = place_of<V, false>(n, 0, 0);
    const bool here = t.left > 0;
    const int lane = threadIdx.x & 31, warp0 = threadIdx.x & ~31;
    const WarpCopy copy(((long long)n.cols - (long long)warp0 * V) * (32 / V));
    const size_t step = gridDim.x;
    size_t row = blockIdx.x;
    const char* py = dy + row * dy_step + warp0 * 32 + lane * 16;
    const char* ps = dsum + row * ds_step + warp0 * 32 + lane * 16;
    const uint8_t* pc = kept.codes + row * n.cols + threadIdx.x * V;
    const uint8_t* pb = kept.scales + row * n.blocks + (warp0 >> n.lanes_log2);   // the warp's first scale byte
    const int bytes = (int)min((long long)(32 >> n.lanes_log2), (long long)n.blocks - (warp0 >> n.lanes_log2));
    const float* pr = rstd + row;
    char* px = dx + row * dx_step + threadIdx.x * 32;
    uint4* slot = ring;
    uint4* other = ring + slot_size;
    auto fetch = [&](uint4* to) {
        copy(to + warp0 * 2, py);
        if constexpr (DSUM) copy(to + 2 * n_thr + warp0 * 2, ps);
        if (here) {
            if constexpr (V == 16) copy_async16(to + (C - 1) * n_thr + threadIdx.x, pc);
            else copy_async8(to + (C - 1) * n_thr + threadIdx.x, pc);
        }
        uint32_t* const meta = reinterpret_cast<uint32_t*>(to + C * n_thr) + kMeta * (threadIdx.x / 32);
        const int off = (int)(reinterpret_cast<uintptr_t>(pb) & 3u);
        if (lane < 9 ? bytes > 0 && 4 * lane < off + bytes : lane == 9) copy_async4(meta + lane, lane < 9 ? (const void*)(pb - off + 4 * lane) : (const void*)pr);
    };
    if (threadIdx.x < sizeof(sums) / 4) reinterpret_cast<float*>(sums)[threadIdx.x] = 0.0f;
    fetch(slot);
    copy_commit();
    float w[V], dw[V];
    load_weight<kWhole, V>(weight, weight_dtype, t, w);
#pragma unroll
    for (int j = 0; j < V; ++j) dw[j] = 0.0f;
    __syncthreads();   // the zeros in `sums`
    for (int turn = 0; row < n.rows; row += step, turn ^= 1) {
        const unsigned off = (unsigned)(reinterpret_cast<uintptr_t>(pb) & 3u) + (lane >> n.lanes_log2);
        __syncwarp();   // the other lanes have read what the next copies replace
        py += step * dy_step, ps += step * ds_step, pc += step * n.cols, pb += step * n.blocks, pr += step;
        if (row + step < n.rows) fetch(other);
        copy_commit();
        copy_wait<1>();
        __syncwarp();
        const uint32_t* const meta = reinterpret_cast<const uint32_t*>(slot + C * n_thr) + kMeta * (threadIdx.x / 32);
        const float rs = __uint_as_float(meta[9]);
        float wd[V], xh[V];
        {
            uint32_t a[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u}, c[V / 4] = {}, byte = 0u;
            if (here) {
                read32(slot + warp0 * 2, a);
                const uint4 q = slot[(C - 1) * n_thr + threadIdx.x];
                c[0] = q.x, c[1] = q.y;
                if constexpr (V == 16) c[2] = q.z, c[3] = q.w;
                byte = reinterpret_cast<const uint8_t*>(meta)[off];
            }
            unpack<DT, V>(a, wd);
            dequantize_block<FMT, V>(c, byte, xh);
        }
        float2 dot = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const float2 d = make_float2(wd[j], wd[j + 1]);
            const float2 h = mul2(make_float2(xh[j], xh[j + 1]), make_float2(rs, rs));
            const float2 s = fma2(d, h, make_float2(dw[j], dw[j + 1]));
            const float2 e = mul2(d, make_float2(w[j], w[j + 1]));
            dot = fma2(e, h, dot);
            dw[j] = s.x, dw[j + 1] = s.y, xh[j] = h.x, xh[j + 1] = h.y, wd[j] = e.x, wd[j + 1] = e.y;
        }
        const float c = -cta_sum<T>(dot.x + dot.y, reinterpret_cast<float*>(sums[turn])) * inv_cols;
        float ds[V];
        uint32_t b[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
        if constexpr (DSUM)
            if (here) read32(slot + 2 * n_thr + warp0 * 2, b);
        unpack<DT, V>(b, ds);
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            float2 e = fma2(make_float2(xh[j], xh[j + 1]), make_float2(c, c), make_float2(wd[j], wd[j + 1]));
            if constexpr (DSUM) e = fma2(e, make_float2(rs, rs), make_float2(ds[j], ds[j + 1]));
            else e = mul2(e, make_float2(rs, rs));
            ds[j] = e.x, ds[j + 1] = e.y;
        }
        pack<DT, V>(ds, b);
        if (here) store256(px, b);
        px += step * dx_step;
        uint4* const done = slot;
        slot = other;
        other = done;
    }
    if (parts) store_parts(parts, blockIdx.x * n.cols + t.vec * V, t, dw);
}

// The same for rows of 8193 to 16384 bf16 elements: 512 threads of two vectors.  Nothing but the weight's gradient is kept in registers; dy and the codes
// are read from the copy and the weight from L1 before the barrier and again behind it.  4096 x 16384: 118 us, and 138 with a CTA of 1024 threads, whose 64
// registers spill; two CTAs of 512 threads in a cluster, their sums exchanged through shared memory, wait 1.5 us a row for its barriers (129 us).
template <int FMT, bool DSUM>
__global__ void __launch_bounds__(512, 1)
    k_add_rmsnorm8_backward_wide(const char* dy, size_t dy_step, const char* dsum, size_t ds_step, const void* weight, int weight_dtype, Held8 kept, const float* rstd,
                                 float inv_cols, NormShape n, char* dx, size_t dx_step, float* parts) {
    constexpr int V = 16, K = 2, T = 512, C = DSUM ? 5 : 3;
    const int n_thr = blockDim.x, half = C * n_thr + kMeta * n_thr / 128, slot_size = K * half;   // half: one vector a thread
    extern __shared__ uint4 ring[];
    __shared__ float4 sums[2][T / 128];
    wait_for_prior_grid();
    release_dependents();
    const int lane = threadIdx.x & 31, warp0 = threadIdx.x & ~31;
    const size_t step = gridDim.x;
    size_t row = blockIdx.x;
    auto fetch = [&](uint4* to, size_t r) {
#pragma unroll
        for (int k = 0; k < K; ++k, to += half) {
            const size_t vec0 = (size_t)k * n_thr + warp0;   // the warp's first vector
            const WarpCopy copy(((long long)n.cols - (long long)vec0 * V) * 2);
            copy(to + warp0 * 2, dy + r * dy_step + vec0 * 32 + lane * 16);
            if constexpr (DSUM) copy(to + 2 * n_thr + warp0 * 2, dsum + r * ds_step + vec0 * 32 + lane * 16);
            if ((vec0 + lane) * V < n.cols) copy_async16(to + (C - 1) * n_thr + threadIdx.x, kept.codes + r * n.cols + (vec0 + lane) * V);
            const size_t block0 = vec0 >> n.lanes_log2;
            const int bytes = (int)min((long long)(32 >> n.lanes_log2), (long long)n.blocks - (long long)block0);
            const uint8_t* const pb = kept.scales + r * n.blocks + block0;
            const int off = (int)(reinterpret_cast<uintptr_t>(pb) & 3u);
            uint32_t* const meta = reinterpret_cast<uint32_t*>(to + C * n_thr) + kMeta * (threadIdx.x / 32);
            if (lane < 9 ? bytes > 0 && 4 * lane < off + bytes : lane == 9) copy_async4(meta + lane, lane < 9 ? (const void*)(pb - off + 4 * lane) : (const void*)(rstd + r));
        }
    };
    // dy and n = h rstd of this thread's k-th vector of the row in `slot`
    auto read = [&](const uint4* slot, int k, const Place& t, float (&d)[V], float (&xh)[V]) {
        const uint4* const at = slot + k * half;
        const uint32_t* const meta = reinterpret_cast<const uint32_t*>(at + C * n_thr) + kMeta * (threadIdx.x / 32);
        uint32_t a[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u}, c[V / 4] = {}, byte = 0u;
        const float rs = __uint_as_float(meta[9]);
        if (t.left > 0) {
            read32(at + warp0 * 2, a);
            const uint4 q = at[(C - 1) * n_thr + threadIdx.x];
            c[0] = q.x, c[1] = q.y, c[2] = q.z, c[3] = q.w;
            const size_t first = row * n.blocks + (((size_t)k * n_thr + warp0) >> n.lanes_log2);
            byte = reinterpret_cast<const uint8_t*>(meta)[((unsigned)reinterpret_cast<uintptr_t>(kept.scales + first) & 3u) + (lane >> n.lanes_log2)];
        }
        unpack<kBF16, V>(a, d);
        dequantize_block<FMT, V>(c, byte, xh);
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const float2 h = mul2(make_float2(xh[j], xh[j + 1]), make_float2(rs, rs));
            xh[j] = h.x, xh[j + 1] = h.y;
        }
        return rs;
    };
    if (threadIdx.x < sizeof(sums) / 4) reinterpret_cast<float*>(sums)[threadIdx.x] = 0.0f;
    uint4* slot = ring;
    uint4* other = ring + slot_size;
    fetch(slot, row);
    copy_commit();
    float dw[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) dw[k][j] = 0.0f;
    __syncthreads();   // the zeros in `sums`
    for (int turn = 0; row < n.rows; row += step, turn ^= 1) {
        __syncwarp();   // the other lanes have read what the next copies replace
        if (row + step < n.rows) fetch(other, row + step);
        copy_commit();
        copy_wait<1>();
        __syncwarp();
        float2 dot = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const Place t = place_of<V, false>(n, row, k);
            float d[V], xh[V], w[V];
            load_weight<kWhole, V>(weight, weight_dtype, t, w);
            read(slot, k, t, d, xh);
#pragma unroll
            for (int j = 0; j < V; j += 2) {
                const float2 y = make_float2(d[j], d[j + 1]), h = make_float2(xh[j], xh[j + 1]);
                const float2 s = fma2(y, h, make_float2(dw[k][j], dw[k][j + 1]));
                dot = fma2(mul2(y, make_float2(w[j], w[j + 1])), h, dot);
                dw[k][j] = s.x, dw[k][j + 1] = s.y;
            }
        }
        const float c = -cta_sum<T>(dot.x + dot.y, reinterpret_cast<float*>(sums[turn])) * inv_cols;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const Place t = place_of<V, false>(n, row, k);
            float d[V], xh[V], w[V], ds[V];
            load_weight<kWhole, V>(weight, weight_dtype, t, w);
            const float rs = read(slot, k, t, d, xh);
            uint32_t b[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
            if constexpr (DSUM)
                if (t.left > 0) read32(slot + k * half + 2 * n_thr + warp0 * 2, b);
            unpack<kBF16, V>(b, ds);
#pragma unroll
            for (int j = 0; j < V; j += 2) {
                float2 e = fma2(make_float2(xh[j], xh[j + 1]), make_float2(c, c), mul2(make_float2(d[j], d[j + 1]), make_float2(w[j], w[j + 1])));
                if constexpr (DSUM) e = fma2(e, make_float2(rs, rs), make_float2(ds[j], ds[j + 1]));
                else e = mul2(e, make_float2(rs, rs));
                ds[j] = e.x, ds[j + 1] = e.y;
            }
            pack<kBF16, V>(ds, b);
            if (t.left > 0) store256(dx + row * dx_step + t.vec * 32, b);
        }
        uint4* const done = slot;
        slot = other;
        other = done;
    }
    if (!parts) return;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const Place t = place_of<V, false>(n, 0, k);
        store_parts(parts, blockIdx.x * n.cols + t.vec * V, t, dw[k]);
    }
}

// dweight[c] = sum over the parts, in a fixed order: each of 32 warps every 32nd part, then a tree over the warps.  With 8 warps a warp's
// loads come in turns, and the launch takes 2 us more.
__global__ void __launch_bounds__(1024) k_rmsnorm8_dweight(const float* parts, int n_parts, size_t cols, float* dweight) {
    __shared__ float sums[32][33];
    wait_for_prior_grid();
    release_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const size_t col = (size_t)blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (col < cols) {
#pragma unroll 8
        for (int p = warp; p < n_parts; p += 32) s += parts[(size_t)p * cols + col];
    }
    sums[warp][lane] = s;
    __syncthreads();
    s = sums[lane][warp];   // warp: the column, lane: the part
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
    const size_t mine = (size_t)blockIdx.x * 32 + warp;
    if (lane == 0 && mine < cols) dweight[mine] = s;
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
static cudaError_t pick(int dtype, int fmt, int fit, const NormLaunch& l, F f) {
    using std::integral_constant;
    using Yes = integral_constant<bool, true>;
    using No = integral_constant<bool, false>;
    auto by_k = [&](auto dt, auto fm, auto fit) {
        if (l.n.group) return f(dt, fm, fit, integral_constant<int, 1>{}, Yes{}, integral_constant<int, 256>{});
        if constexpr (fit() != kWhole) {   // those are rows_fit()
            if (l.K == 1 && l.threads <= 256) return f(dt, fm, fit, integral_constant<int, 1>{}, No{}, integral_constant<int, 256>{});
            if (l.K == 1 && l.threads <= 512) return f(dt, fm, fit, integral_constant<int, 1>{}, No{}, integral_constant<int, 512>{});
            if (l.K == 1) return f(dt, fm, fit, integral_constant<int, 1>{}, No{}, integral_constant<int, 1024>{});
        }
        static_assert(kNorm8MaxCols <= 2 * 1024 * vec_elems(kBF16) && kNorm8MaxCols <= 4 * 1024 * vec_elems(kF32), "vectors of a thread");
        if constexpr (dt() == kF32) {
            if (l.K == 4) return f(dt, fm, fit, integral_constant<int, 4>{}, No{}, integral_constant<int, 1024>{});
        }
        return f(dt, fm, fit, integral_constant<int, 2>{}, No{}, integral_constant<int, 1024>{});
    };
    auto by_fit = [&](auto dt, auto fm) {
        return fit == kWhole  ? by_k(dt, fm, integral_constant<int, kWhole>{})
               : fit == kHalf ? by_k(dt, fm, integral_constant<int, kHalf>{})
                              : by_k(dt, fm, integral_constant<int, kAny>{});
    };
    auto by_fmt = [&](auto dt) { return fmt == kE4M3 ? by_fit(dt, integral_constant<int, kE4M3>{}) : by_fit(dt, integral_constant<int, kE5M2>{}); };
    return dtype == kBF16 ? by_fmt(integral_constant<int, kBF16>{}) : by_fmt(integral_constant<int, kF32>{});
}

static bool rows_fit(const NormLaunch& l, int fit) { return fit == kWhole && l.n.group == 0 && l.K == 1; }

// A vector of cols elements that goes with rows of `dtype`: pieces of as many elements as theirs.
static int fit_of_weight(const void* p, int weight_dtype, int dtype, size_t cols) {
    const size_t v = (size_t)vec_elems(dtype);
    const uintptr_t bytes = v * (weight_dtype == kF32 ? 4 : 2), at = reinterpret_cast<uintptr_t>(p);   // of a vector: 16, 32 or 64
    const uintptr_t whole = bytes < 32 ? bytes : 32, half = bytes / 2 < 16 ? bytes / 2 : 16;
    if (at % whole == 0 && cols % v == 0) return kWhole;
    return at % half == 0 && cols % (v / 2) == 0 ? kHalf : kAny;
}

// Grid of a kernel whose CTAs take turns on `work` rows (or groups of rows): the resident CTAs of the device, `most` at most.  smem: of this launch;
// smem_most: of the kernel's largest, which its limit has to allow whatever launch comes first.  cache: one for each number of warps.
static cudaError_t rows_grid(const void* kernel, size_t smem, size_t smem_most, unsigned threads, std::atomic<int> (*cache)[kMaxDevices], size_t work, size_t most,
                             unsigned& grid) {
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    if (dev >= kMaxDevices) return cudaErrorInvalidDevice;
    int ctas = cache[threads / 32][dev].load(std::memory_order_relaxed);
    if (ctas == 0) {   // threads that race here store the same value
        err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_most);
        if (err != cudaSuccess) return err;
        err = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&ctas, kernel, (int)threads, smem);
        if (err != cudaSuccess) return err;
        if (ctas < 1) ctas = 1;
        cache[threads / 32][dev].store(ctas, std::memory_order_relaxed);
    }
    size_t g = (size_t)ctas * (size_t)sm_count(dev);
    if (g > most) g = most;
    grid = (unsigned)(g < work ? g : work);
    return cudaSuccess;
}

template <typename F>
static cudaError_t pick_rows(int dtype, int fmt, const NormLaunch& l, F f) {
    using std::integral_constant;
    auto by_threads = [&](auto dt, auto fm) {
        return l.threads <= 256   ? f(dt, fm, integral_constant<int, 256>{})
               : l.threads <= 320 ? f(dt, fm, integral_constant<int, 320>{})
               : l.threads <= 384 ? f(dt, fm, integral_constant<int, 384>{})
               : l.threads <= 512 ? f(dt, fm, integral_constant<int, 512>{})
                                  : f(dt, fm, integral_constant<int, 1024>{});
    };
    auto by_fmt = [&](auto dt) { return fmt == kE4M3 ? by_threads(dt, integral_constant<int, kE4M3>{}) : by_threads(dt, integral_constant<int, kE5M2>{}); };
    return dtype == kBF16 ? by_fmt(integral_constant<int, kBF16>{}) : by_fmt(integral_constant<int, kF32>{});
}

cudaError_t launch_add_rmsnorm8(const Wide8& x, const Wide8& residual, const void* weight, int weight_dtype, size_t rows, size_t cols, float eps, int B, int dtype, int fmt,
                                const Wide8& out_sum, const Held8& out, const Held8& kept, float* out_rstd, cudaStream_t s) {
    const NormLaunch l = norm_launch(rows, cols, B, dtype);
    int fit = worst_fit(fit_of(x, cols, dtype), fit_of_weight(weight, weight_dtype, dtype, cols));
    if (residual.p) fit = worst_fit(fit, worst_fit(fit_of(residual, cols, dtype), fit_of(out_sum, cols, dtype)));
    if (rows_fit(l, fit)) {
        return pick_rows(dtype, fmt, l, [&](auto dt, auto fm, auto threads) {
            auto go = [&](auto res, auto keep) {
                static std::atomic<int> cache[33][kMaxDevices];
                auto* kernel = k_add_rmsnorm8_rows<dt(), fm(), res(), keep(), threads()>;
                auto smem_of = [&](size_t n) { return 2 * (res() ? 4 : 2) * n * 16; };
                const size_t smem = smem_of(l.threads);
                unsigned grid = 0;
                cudaError_t err = rows_grid((const void*)kernel, smem, smem_of(threads()), l.threads, cache, rows, SIZE_MAX, grid);
                if (err != cudaSuccess) return err;
                count_launch();
                const size_t es = dtype == kF32 ? 4 : 2;
                return launch_pdl(kernel, grid, l.threads, smem, s, (const char*)x.p, x.stride * es, (const char*)residual.p, residual.stride * es, weight, weight_dtype, eps, 1.0f / (float)cols, l.n,
                                  (char*)out_sum.p, out_sum.stride * es, out, kept, out_rstd);
            };
            using Yes = std::integral_constant<bool, true>;
            using No = std::integral_constant<bool, false>;
            if (residual.p) return kept.codes ? go(Yes{}, Yes{}) : go(Yes{}, No{});
            return kept.codes ? go(No{}, Yes{}) : go(No{}, No{});
        });
    }
    return pick(dtype, fmt, fit, l, [&](auto dt, auto fm, auto v, auto k, auto small, auto threads) {
        count_launch();
        return launch_pdl(k_add_rmsnorm8<dt(), fm(), v(), k(), small(), threads()>, (unsigned)((rows + l.rows_cta - 1) / l.rows_cta), l.threads, 0, s, (const void*)x.p, x.stride,
                          (const void*)residual.p, residual.stride, weight, weight_dtype, eps, 1.0f / (float)cols, l.n, out_sum.p, out_sum.stride, out, kept, out_rstd);
    });
}

cudaError_t launch_add_rmsnorm8_backward(const Wide8& dy, const Wide8& dsum, const void* weight, int weight_dtype, const Held8& kept, const float* rstd, size_t rows, size_t cols,
                                         int B, int dtype, int fmt, const Wide8& dx, float* dweight, float* parts, cudaStream_t s) {
    const NormLaunch l = norm_launch(rows, cols, B, dtype);
    int fit = worst_fit(worst_fit(fit_of(dy, cols, dtype), fit_of(dx, cols, dtype)), fit_of_weight(weight, weight_dtype, dtype, cols));
    if (dsum.p) fit = worst_fit(fit, fit_of(dsum, cols, dtype));
    unsigned grid = 0;
    cudaError_t err;
    if (rows_fit(l, fit)) {
        err = pick_rows(dtype, fmt, l, [&](auto dt, auto fm, auto threads) {
            auto go = [&](auto ds) {
                static std::atomic<int> cache[33][kMaxDevices];
                auto launch = [&](auto* kernel, unsigned n, auto smem_of, unsigned most) {
                    cudaError_t e = rows_grid((const void*)kernel, smem_of(n), smem_of(most), n, cache, rows, kNorm8Parts, grid);
                    if (e != cudaSuccess) return e;
                    count_launch();
                    const size_t es = dtype == kF32 ? 4 : 2;
                    return launch_pdl(kernel, grid, n, smem_of(n), s, (const char*)dy.p, dy.stride * es, (const char*)dsum.p, dsum.stride * es, weight, weight_dtype, kept, rstd,
                                      1.0f / (float)cols, l.n, (char*)dx.p, dx.stride * es, dweight ? parts : (float*)nullptr);
                };
                auto smem_of = [&](size_t n) { return 2 * ((ds() ? 5 : 3) * n * 16 + kMeta * n / 8); };
                if constexpr (dt() == kBF16 && threads() == 1024) {
                    return launch(k_add_rmsnorm8_backward_wide<fm(), ds()>, (l.threads / 2 + 31) / 32 * 32, [&](size_t n) { return 2 * smem_of(n); }, 512u);
                } else {
                    return launch(k_add_rmsnorm8_backward_rows<dt(), fm(), ds(), threads()>, l.threads, smem_of, (unsigned)threads());
                }
            };
            return dsum.p ? go(std::integral_constant<bool, true>{}) : go(std::integral_constant<bool, false>{});
        });
    } else {
        err = pick(dtype, fmt, fit, l, [&](auto dt, auto fm, auto v, auto k, auto small, auto threads) {
            static std::atomic<int> cache[33][kMaxDevices];
            auto* kernel = k_add_rmsnorm8_backward<dt(), fm(), v(), v(), k(), small(), threads()>;
            if constexpr (v() == kWhole && !small()) {   // 1024 threads either way: one CTA an SM, the same split of the rows
                if (reinterpret_cast<uintptr_t>(parts) & 31u) kernel = k_add_rmsnorm8_backward<dt(), fm(), v(), kHalf, k(), small(), threads()>;
            }
            cudaError_t e = rows_grid((const void*)kernel, 0, 0, l.threads, cache, (rows + l.rows_cta - 1) / l.rows_cta, kNorm8Parts, grid);
            if (e != cudaSuccess) return e;
            count_launch();
            return launch_pdl(kernel, grid, l.threads, 0, s, (const void*)dy.p, dy.stride, (const void*)dsum.p, dsum.stride, weight, weight_dtype, kept, rstd,
                              1.0f / (float)cols, l.n, dx.p, dx.stride, dweight ? parts : (float*)nullptr);
        });
    }
    if (err != cudaSuccess || !dweight) return err;
    count_launch();
    return launch_pdl(k_rmsnorm8_dweight, (unsigned)((cols + 31) / 32), 1024, 0, s, (const float*)parts, (int)grid, cols, dweight);
}

}  // namespace mxq
