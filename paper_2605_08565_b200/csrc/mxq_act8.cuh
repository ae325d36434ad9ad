// Device-side building blocks of the operators on block-scaled 8-bit activations: rows of E4M3 or E5M2 elements with one
// power-of-two scale byte (UE8M0) per block of B = 16, 32, 64 or 128 consecutive elements of a row.
//
// A thread works on vectors of 8 consecutive elements (16 bytes of bf16, 32 of fp32, 8 code bytes), so a block lies in B / 8
// neighbouring lanes of one warp and its maximum takes log2(B / 8) shuffles.  Rows are padded to whole blocks in this numbering: the
// lanes behind the end of a row hold zeros and store nothing.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "mxq_device.cuh"

namespace mxq {

constexpr int kE4M3 = 0, kE5M2 = 1;
constexpr int kVec = 8;   // elements of a vector

// ---- vectors of 8 elements as fp32 ---------------------------------------------------------------
// VEC: the caller has checked that rows start on 16 bytes and hold whole vectors.  Otherwise element by element, `left` (<= 0: none)
// of them; the rest are zeros.
template <int DT, bool VEC>
__device__ __forceinline__ void load8(const void* base, size_t at, int left, float (&v)[kVec]) {
    if constexpr (VEC) {
        if (left <= 0) {
#pragma unroll
            for (int j = 0; j < kVec; ++j) v[j] = 0.0f;
            return;
        }
        if constexpr (DT == kBF16) {
            const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at);
            const uint32_t p[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[2 * j] = __uint_as_float(p[j] << 16);
                v[2 * j + 1] = __uint_as_float(p[j] & 0xFFFF0000u);
            }
        } else {
            const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
            const float4 a = q[0], b = q[1];
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            v[j] = 0.0f;
            if (j < left) {
                if constexpr (DT == kBF16) v[j] = __uint_as_float((uint32_t) static_cast<const uint16_t*>(base)[at + j] << 16);
                else v[j] = static_cast<const float*>(base)[at + j];
            }
        }
    }
}

// Rounds to bf16 (to nearest even) where the type asks for it: bits of two elements in a word, the first in the low half.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}

template <int DT, bool VEC>
__device__ __forceinline__ void store8(void* base, size_t at, int left, const float (&v)[kVec]) {
    if constexpr (VEC) {
        if (left <= 0) return;
        if constexpr (DT == kBF16) {
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + at) =
                make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
        } else {
            float4* q = reinterpret_cast<float4*>(static_cast<float*>(base) + at);
            q[0] = make_float4(v[0], v[1], v[2], v[3]);
            q[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            if (j < left) {
                if constexpr (DT == kBF16) static_cast<uint16_t*>(base)[at + j] = (uint16_t)pack_bf16(v[j], 0.0f);
                else static_cast<float*>(base)[at + j] = v[j];
            }
        }
    }
}

// What a value becomes when it is stored as DT and read back.
template <int DT>
__device__ __forceinline__ void round8(float (&v)[kVec]) {
    if constexpr (DT == kBF16) {
#pragma unroll
        for (int j = 0; j < kVec; j += 2) {
            const uint32_t p = pack_bf16(v[j], v[j + 1]);
            v[j] = __uint_as_float(p << 16);
            v[j + 1] = __uint_as_float(p & 0xFFFF0000u);
        }
    }
}

template <bool VEC>
__device__ __forceinline__ uint2 load_codes8(const uint8_t* base, size_t at, int left) {
    if constexpr (VEC) return left > 0 ? *reinterpret_cast<const uint2*>(base + at) : make_uint2(0u, 0u);
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < kVec; ++j)
        if (j < left) w[j >> 2] |= (uint32_t)base[at + j] << (8 * (j & 3));
    return make_uint2(w[0], w[1]);
}

template <bool VEC>
__device__ __forceinline__ void store_codes8(uint8_t* base, size_t at, int left, uint2 c) {
    if constexpr (VEC) {
        if (left > 0) *reinterpret_cast<uint2*>(base + at) = c;
    } else {
        const uint32_t w[2] = {c.x, c.y};
#pragma unroll
        for (int j = 0; j < kVec; ++j)
            if (j < left) base[at + j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
    }
}

// ---- block scales --------------------------------------------------------------------------------
// Scale byte of a block whose largest magnitude has these bits: c = e + 127 with the smallest e >= -127 for which
// amax <= top * 2^e, top = 1.75 * 2^t the largest element (t = 8 for E4M3, 15 for E5M2).  amax = m * 2^E with 1 <= m < 2 gives
// e = E - t for m <= 1.75 and one more above; adding 2^21 - 1 to the bits carries into the exponent field exactly for m > 1.75.
// Magnitudes order like their bits, infinity and NaN above all finite ones: byte 0xFF.
template <int FMT>
__device__ __forceinline__ uint32_t pow2_scale_byte(uint32_t amax_bits) {
    constexpr int T = FMT == kE4M3 ? 8 : 15;
    if (amax_bits >= 0x7F800000u) return 0xFFu;
    return (uint32_t)max((int)((amax_bits + 0x1FFFFFu) >> 23) - T, 0);
}
// 2^(127 - c), by which elements are multiplied: a power of two, so the products are the quotients.  (Those below 2^-126, which
// round, become zeros all the same.)  NaN for the byte 0xFF.
__device__ __forceinline__ float pow2_scale_inverse(uint32_t c) { return __uint_as_float(c == 0xFFu ? 0x7FC00000u : (254u - c) << 23); }
// 2^(c - 127)
__device__ __forceinline__ float pow2_scale_value(uint32_t c) {
    return __uint_as_float(c == 0xFFu ? 0x7FC00000u : c == 0u ? 0x00400000u : c << 23);
}

// Two values to two codes, to nearest even, a in the low byte; NaN becomes 0x7F.
template <int FMT>
__device__ __forceinline__ uint32_t pack_fp8x2(float a, float b) {
    uint16_t r;
    if constexpr (FMT == kE4M3) asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
    else asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
    return r;
}

// Every 8-bit code is a binary16 value.
template <int FMT>
__device__ __forceinline__ float2 unpack_fp8x2(uint32_t two) {
    uint32_t h;
    if constexpr (FMT == kE4M3) asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    else asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Quantizes the vectors of the `lanes` neighbouring threads that hold a block.  All 32 lanes of the warp call it together.
template <int FMT>
__device__ __forceinline__ uint2 quantize_block8(const float (&v)[kVec], int lanes, uint32_t& byte) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < kVec; ++j) m = max(m, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    for (int o = 1; o < lanes; o <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    byte = pow2_scale_byte<FMT>(m);
    const float inv = pow2_scale_inverse(byte);
    return make_uint2(pack_fp8x2<FMT>(v[0] * inv, v[1] * inv) | pack_fp8x2<FMT>(v[2] * inv, v[3] * inv) << 16,
                      pack_fp8x2<FMT>(v[4] * inv, v[5] * inv) | pack_fp8x2<FMT>(v[6] * inv, v[7] * inv) << 16);
}

template <int FMT>
__device__ __forceinline__ void dequantize8(uint2 c, float scale, float (&v)[kVec]) {
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int j = 0; j < kVec; j += 2) {
        const float2 f = unpack_fp8x2<FMT>(w[j >> 2] >> (8 * (j & 3)));
        v[j] = f.x * scale;
        v[j + 1] = f.y * scale;
    }
}

// Quantizes and stores this thread's vector, `vec` in its row; the first lane of a block stores the scale.  The whole warp calls it.
template <int FMT, bool VEC>
__device__ __forceinline__ void put_held8(Held8 out, const float (&v)[kVec], size_t row, size_t vec, size_t cols, size_t blocks, int lanes, int lanes_log2, int left) {
    uint32_t byte;
    const uint2 c = quantize_block8<FMT>(v, lanes, byte);
    store_codes8<VEC>(out.codes, row * cols + vec * kVec, left, c);
    if (left > 0 && (vec & (size_t)(lanes - 1)) == 0) out.scales[row * blocks + (vec >> lanes_log2)] = (uint8_t)byte;
}

template <int FMT, bool VEC>
__device__ __forceinline__ void get_held8(Held8 in, float (&v)[kVec], size_t row, size_t vec, size_t cols, size_t blocks, int lanes_log2, int left) {
    const uint2 c = load_codes8<VEC>(in.codes, row * cols + vec * kVec, left);
    const float s = left > 0 ? pow2_scale_value(in.scales[row * blocks + (vec >> lanes_log2)]) : 0.0f;
    dequantize8<FMT>(c, s, v);
}

}  // namespace mxq
