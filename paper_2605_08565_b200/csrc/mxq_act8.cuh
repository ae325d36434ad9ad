// Device-side building blocks of the operators on block-scaled 8-bit activations: rows of E4M3 or E5M2 elements with one
// power-of-two scale byte (UE8M0) per block of B = 16, 32, 64 or 128 consecutive elements of a row.
//
// A thread works on vectors of 32 bytes of a wide tensor: 16 bf16 or 8 fp32 elements, 16 or 8 code bytes.  A block lies in
// B / 16 or B / 8 neighbouring lanes of one warp, and its maximum takes at most four shuffles.  Rows are padded to whole blocks in
// this numbering: the lanes behind the end of a row hold zeros and store nothing.
//
// How rows lie (FIT): kWhole, they start on 32 bytes and hold whole vectors, which are read and written at once; kHalf, the same of 16 bytes
// and half vectors; kAny, all others (an odd number of elements, a view that starts anywhere).  Those are read in the aligned 16-byte
// pieces that their bytes lie in, shifted into place in registers; on the way out neighbouring lanes exchange what belongs into the
// other's aligned pieces, and only the two ends of a warp's run of a row are stored in pieces of 1 to 8 bytes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "mxq_device.cuh"

namespace mxq {

constexpr int kE4M3 = 0, kE5M2 = 1;
constexpr unsigned kFull = 0xFFFFFFFFu;
// Elements of a vector.
__host__ __device__ constexpr int vec_elems(int dt) { return dt == kF32 ? 8 : 16; }

// ---- bytes ---------------------------------------------------------------------------------------
// w = the words of c from byte `by` (< 4 * (M - N)) on; EB: by is a multiple of it.  `by` is the same for all vectors of a row, so that the
// branch is one of the whole warp but for its row ends; selecting every word by two bits of it instead made the shifted rows wait for the
// ALU (four fifths busy).
template <int EB, int Q, int N, int M>
__device__ __forceinline__ void words_from(const uint32_t (&c)[M], unsigned by, uint32_t (&w)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (EB == 4) w[i] = c[i + Q];
        else w[i] = __funnelshift_r(c[i + Q], c[i + Q + 1 < M ? i + Q + 1 : i + Q], 8u * (by & 3u));
    }
}
template <int EB, int N, int M>
__device__ __forceinline__ void shift_down(const uint32_t (&c)[M], unsigned by, uint32_t (&w)[N]) {
    switch (by >> 2) {
    case 0: words_from<EB, 0>(c, by, w); break;
    case 1: words_from<EB, 1>(c, by, w); break;
    case 2:
        if constexpr (M - N > 2) words_from<EB, 2>(c, by, w);
        break;
    default:
        if constexpr (M - N > 2) words_from<EB, 3>(c, by, w);
        break;
    }
}

__device__ __forceinline__ void load256(const void* p, uint32_t* w) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void store256(void* p, const uint32_t* w) {
    asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]),
                 "l"(p)
                 : "memory");
}

// NB bytes from p on, of which the first `valid` exist (the others become zeros), in elements of EB bytes.  Under kAny the aligned pieces are read whole: a
// piece that holds a byte of the row is mapped as a whole.
template <int NB, int EB, int FIT>
__device__ __forceinline__ void load_bytes(const void* p, int valid, uint32_t (&w)[NB / 4]) {
    constexpr int N = NB / 4;
    if constexpr (FIT == kWhole) {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = 0u;
        if (valid <= 0) return;
        if constexpr (NB == 8) {
            const uint2 a = *static_cast<const uint2*>(p);
            w[0] = a.x, w[1] = a.y;
        } else if constexpr (NB == 16) {
            const uint4 a = *static_cast<const uint4*>(p);
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 8) load256(static_cast<const char*>(p) + 4 * i, w + i);
        }
    } else if constexpr (FIT == kHalf) {
        constexpr int G = NB / 2 < 16 ? NB / 2 : 16;
        const char* q = static_cast<const char*>(p);
#pragma unroll
        for (int i = 0; i < NB / G; ++i) {
            const bool on = i * G < valid;
            if constexpr (G == 4) {
                w[i] = on ? *reinterpret_cast<const uint32_t*>(q + 4 * i) : 0u;
            } else if constexpr (G == 8) {
                const uint2 a = on ? *reinterpret_cast<const uint2*>(q + 8 * i) : make_uint2(0u, 0u);
                w[2 * i] = a.x, w[2 * i + 1] = a.y;
            } else {
                const uint4 a = on ? *reinterpret_cast<const uint4*>(q + 16 * i) : make_uint4(0u, 0u, 0u, 0u);
                w[4 * i] = a.x, w[4 * i + 1] = a.y, w[4 * i + 2] = a.z, w[4 * i + 3] = a.w;
            }
        }
    } else {
        constexpr int G = NB < 16 ? NB : 16, M = N + G / 4;
        const unsigned by = (unsigned)(reinterpret_cast<uintptr_t>(p) & (G - 1));
        const char* q = static_cast<const char*>(p) - by;
        uint32_t c[M];
#pragma unroll
        for (int i = 0; i < M; ++i) c[i] = 0u;
#pragma unroll
        for (int i = 0; i < M * 4 / G; ++i) {
            if (valid > 0 && i * G < (int)by + valid) {
                if constexpr (G == 16) {
                    const uint4 a = *reinterpret_cast<const uint4*>(q + i * G);
                    c[4 * i] = a.x, c[4 * i + 1] = a.y, c[4 * i + 2] = a.z, c[4 * i + 3] = a.w;
                } else {
                    const uint2 a = *reinterpret_cast<const uint2*>(q + i * G);
                    c[2 * i] = a.x, c[2 * i + 1] = a.y;
                }
            }
        }
        shift_down<EB>(c, by, w);
        if (valid < NB) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int n = valid - 4 * i;
                w[i] = n >= 4 ? w[i] : n <= 0 ? 0u : w[i] & (0xFFFFFFFFu >> (32 - 8 * n));
            }
        }
    }
}

template <int EB>
__device__ __forceinline__ void store_element(char* to, uint32_t v) {
    if constexpr (EB == 4) *reinterpret_cast<uint32_t*>(to) = v;
    else if constexpr (EB == 2) *reinterpret_cast<uint16_t*>(to) = (uint16_t)v;
    else *reinterpret_cast<uint8_t*>(to) = (uint8_t)v;
}

// NB bytes to p on, of which the first `valid` are stored, in elements of EB bytes.  A warp's lanes hold consecutive vectors, of one row
// or of several: `first` tells that a vector starts its row, and `after` counts the bytes that its row holds behind it.  All 32 lanes call it.
template <int NB, int EB, int FIT>
__device__ __forceinline__ void store_bytes(void* p, int valid, bool first, int after, const uint32_t (&w)[NB / 4]) {
    constexpr int N = NB / 4;
    if constexpr (FIT == kWhole) {
        if (valid <= 0) return;
        if constexpr (NB == 8) {
            *static_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        } else if constexpr (NB == 16) {
            *static_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 8) store256(static_cast<char*>(p) + 4 * i, w + i);
        }
    } else if constexpr (FIT == kHalf) {
        constexpr int G = NB / 2 < 16 ? NB / 2 : 16;
        char* q = static_cast<char*>(p);
#pragma unroll
        for (int i = 0; i < NB / G; ++i) {
            if (i * G >= valid) continue;
            if constexpr (G == 4) *reinterpret_cast<uint32_t*>(q + 4 * i) = w[i];
            else if constexpr (G == 8) *reinterpret_cast<uint2*>(q + 8 * i) = make_uint2(w[2 * i], w[2 * i + 1]);
            else *reinterpret_cast<uint4*>(q + 16 * i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        }
    } else {
        constexpr int G = NB < 16 ? NB : 16, GW = G / 4, C = NB / G;
        const unsigned lane = threadIdx.x & 31;
        const int h = (int)((0u - (unsigned)reinterpret_cast<uintptr_t>(p)) & (G - 1));   // bytes in front of the first aligned piece
        uint32_t c[N + GW];
#pragma unroll
        for (int i = 0; i < N; ++i) c[i] = w[i];
#pragma unroll
        for (int i = 0; i < GW; ++i) c[N + i] = __shfl_down_sync(kFull, w[i], 1);
        uint32_t out[N];
        shift_down<EB>(c, (unsigned)h, out);
        if (valid <= 0) return;
        const bool head_taken = h == 0 || (lane > 0 && !first && valid >= h);   // by the lane before
        const bool last_whole = valid == NB && (h == 0 || (lane < 31 && after >= h));
        char* q = static_cast<char*>(p) + h;
        int done = h;   // bytes in front of which everything but an untaken head is stored
#pragma unroll
        for (int i = 0; i < C; ++i) {
            if (i + 1 < C ? h + (i + 1) * G <= valid : last_whole) {
                if constexpr (G == 16) *reinterpret_cast<uint4*>(q + i * G) = make_uint4(out[4 * i], out[4 * i + 1], out[4 * i + 2], out[4 * i + 3]);
                else *reinterpret_cast<uint2*>(q + i * G) = make_uint2(out[2 * i], out[2 * i + 1]);
                done += G;
            }
        }
        if (!head_taken) {   // the first h bytes, in pieces of 1, 2, 4 and 8 up to the first aligned address
            char* to = static_cast<char*>(p);
            if (valid < h) {   // a short vector that does not come so far
#pragma unroll
                for (int b = 0; b < G; b += EB)
                    if (b < valid) store_element<EB>(to + b, w[b / 4] >> (8 * (b & 3)));
            } else {
                const unsigned sh = 8u * (h & 3);
                if (EB <= 1 && (h & 1)) store_element<1>(to, w[0]);
                if (EB <= 2 && (h & 2)) store_element<2>(to + (h & 1), w[0] >> (8 * (h & 1)));
                if (h & 4) store_element<4>(to + (h & 3), __funnelshift_r(w[0], w[1], sh));
                if constexpr (G == 16) {
                    if (h & 8) {
                        const bool q = h & 4;
                        const uint32_t a0 = q ? w[1] : w[0], a1 = q ? w[2] : w[1], a2 = q ? w[3] : w[2];
                        *reinterpret_cast<uint2*>(to + (h & 7)) = make_uint2(__funnelshift_r(a0, a1, sh), __funnelshift_r(a1, a2, sh));
                    }
                }
            }
        }
        if (done < valid) {   // the last bytes, from an aligned address on, in pieces of 8, 4, 2 and 1
            char* to = static_cast<char*>(p) + done;
            const int n = valid - done;
            uint32_t t[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int k = 0; k < GW; ++k) t[k] = done == h + i * G ? out[i * GW + k] : t[k];
            if constexpr (G == 16)
                if (n & 8) *reinterpret_cast<uint2*>(to) = make_uint2(t[0], t[1]);
            const uint32_t t4 = n & 8 ? t[2] : t[0], t5 = n & 8 ? t[3] : t[1];
            if (n & 4) store_element<4>(to + (n & 8), t4);
            const uint32_t t2 = n & 4 ? t5 : t4;
            if (EB <= 2 && (n & 2)) store_element<2>(to + (n & 12), t2);
            if (EB <= 1 && (n & 1)) store_element<1>(to + (n & 14), t2 >> (8 * (n & 2)));
        }
    }
}

// ---- values --------------------------------------------------------------------------------------
// Rounds two values to bf16 (to nearest even): a in the low half of the word.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}

template <int DT, int V>
__device__ __forceinline__ void unpack(const uint32_t* w, float (&v)[V]) {
    if constexpr (DT == kBF16) {
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            v[j] = __uint_as_float(w[j / 2] << 16);
            v[j + 1] = __uint_as_float(w[j / 2] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = __uint_as_float(w[j]);
    }
}
template <int DT, int V>
__device__ __forceinline__ void pack(const float (&v)[V], uint32_t* w) {
    if constexpr (DT == kBF16) {
#pragma unroll
        for (int j = 0; j < V; j += 2) w[j / 2] = pack_bf16(v[j], v[j + 1]);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = __float_as_uint(v[j]);
    }
}

// Two binary32 products in one instruction, each rounded to nearest even.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    uint64_t x, y, z;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a.x), "f"(a.y));
    asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(b.x), "f"(b.y));
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(z) : "l"(x), "l"(y));
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(z));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t x, y, t, z;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a.x), "f"(a.y));
    asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(b.x), "f"(b.y));
    asm("mov.b64 %0, {%1, %2};" : "=l"(t) : "f"(c.x), "f"(c.y));
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(z) : "l"(x), "l"(y), "l"(t));
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(z));
    return r;
}

__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// ---- asynchronous copies into shared memory: a thread reads back only what it copied itself ----
__device__ __forceinline__ void copy_async16(void* to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_async8(void* to, const void* from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_async4(void* to, const void* from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Waits until at most `N` of this thread's groups are under way.
template <int N>
__device__ __forceinline__ void copy_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
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

// Four values to four codes, to nearest even, the first in the low byte; NaN becomes 0x7F.
template <int FMT>
__device__ __forceinline__ uint32_t pack_fp8x4(float2 a, float2 b) {
    uint32_t r;
    if constexpr (FMT == kE4M3)
        asm("{\n .reg .b16 l, h;\n cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n mov.b32 %0, {l, h};\n}"
            : "=r"(r) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    else
        asm("{\n .reg .b16 l, h;\n cvt.rn.satfinite.e5m2x2.f32 l, %2, %1;\n cvt.rn.satfinite.e5m2x2.f32 h, %4, %3;\n mov.b32 %0, {l, h};\n}"
            : "=r"(r) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

// Four codes to four values; every 8-bit code is a binary16 value.
template <int FMT>
__device__ __forceinline__ void unpack_fp8x4(uint32_t four, float2& a, float2& b) {
    uint32_t l, h;
    if constexpr (FMT == kE4M3)
        asm("{\n .reg .b16 x, y;\n mov.b32 {x, y}, %2;\n cvt.rn.f16x2.e4m3x2 %0, x;\n cvt.rn.f16x2.e4m3x2 %1, y;\n}" : "=r"(l), "=r"(h) : "r"(four));
    else
        asm("{\n .reg .b16 x, y;\n mov.b32 {x, y}, %2;\n cvt.rn.f16x2.e5m2x2 %0, x;\n cvt.rn.f16x2.e5m2x2 %1, y;\n}" : "=r"(l), "=r"(h) : "r"(four));
    a = __half22float2(*reinterpret_cast<const __half2*>(&l));
    b = __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Bits of the largest magnitude; a NaN wins over everything.
template <int V>
__device__ __forceinline__ uint32_t amax_bits(const float (&v)[V]) {
    float m = 0.0f;
#pragma unroll
    for (int j = 0; j < V; j += 2) asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(m), "f"(v[j]), "f"(v[j + 1]));
    return __float_as_uint(m) & 0x7FFFFFFFu;
}

// Quantizes a vector together with those of the 2^lanes_log2 neighbouring threads that hold its block.  All 32 lanes of the warp call it.
template <int FMT, int V>
__device__ __forceinline__ uint32_t quantize_block(const float (&v)[V], int lanes_log2, uint32_t (&codes)[V / 4]) {
    uint32_t m = amax_bits<V>(v);
#pragma unroll
    for (int l = 0; l < (V == 16 ? 3 : 4); ++l)
        if (l < lanes_log2) m = max(m, __shfl_xor_sync(kFull, m, 1 << l));
    const uint32_t byte = pow2_scale_byte<FMT>(m);
    const float inv = pow2_scale_inverse(byte);
#pragma unroll
    for (int j = 0; j < V; j += 4)
        codes[j / 4] = pack_fp8x4<FMT>(mul2(make_float2(v[j], v[j + 1]), make_float2(inv, inv)), mul2(make_float2(v[j + 2], v[j + 3]), make_float2(inv, inv)));
    return byte;
}

template <int FMT, int V>
__device__ __forceinline__ void dequantize_block(const uint32_t* codes, uint32_t byte, float (&v)[V]) {
    const float s = pow2_scale_value(byte);
#pragma unroll
    for (int j = 0; j < V; j += 4) {
        float2 a, b;
        unpack_fp8x4<FMT>(codes[j / 4], a, b);
        a = mul2(a, make_float2(s, s)), b = mul2(b, make_float2(s, s));
        v[j] = a.x, v[j + 1] = a.y, v[j + 2] = b.x, v[j + 3] = b.y;
    }
}

// ---- vectors of rows -----------------------------------------------------------------------------
// One vector: its place in the row and what of the row is left there.
struct Place {
    size_t row, vec;
    int left;   // elements from its first one to the end of the row, a large number for more than that; <= 0: it lies behind the end
};
__device__ __forceinline__ int left_of(size_t cols, size_t first) {
    const long long n = (long long)cols - (long long)first;
    return n < 1024 ? (int)n : 1024;
}

// A wide tensor's vector as fp32.
template <int DT, int FIT, int V>
__device__ __forceinline__ void load_wide(const void* base, size_t at, int left, float (&v)[V]) {
    constexpr int EB = elem_bytes(DT);
    uint32_t w[V * EB / 4];
    load_bytes<V * EB, EB, FIT>(static_cast<const char*>(base) + at * EB, min(left, V) * EB, w);
    unpack<DT, V>(w, v);
}
template <int DT, int FIT, int V>
__device__ __forceinline__ void store_wide(void* base, size_t at, const Place& t, const float (&v)[V]) {
    constexpr int EB = elem_bytes(DT);
    uint32_t w[V * EB / 4];
    pack<DT, V>(v, w);
    store_bytes<V * EB, EB, FIT>(static_cast<char*>(base) + at * EB, min(t.left, V) * EB, t.vec == 0, (t.left - V) * EB, w);
}

// Quantizes and stores this thread's vector; the first lane of a block stores the scale.  The whole warp calls it.
template <int FMT, int FIT, int V>
__device__ __forceinline__ void put_held(const Held8& out, const float (&v)[V], const Place& t, size_t cols, size_t blocks, int lanes_log2) {
    uint32_t c[V / 4];
    const uint32_t byte = quantize_block<FMT, V>(v, lanes_log2, c);
    store_bytes<V, 1, FIT>(out.codes + t.row * cols + t.vec * V, min(t.left, V), t.vec == 0, t.left - V, c);
    if (t.left > 0 && (t.vec & (size_t)((1 << lanes_log2) - 1)) == 0) out.scales[t.row * blocks + (t.vec >> lanes_log2)] = (uint8_t)byte;
}

template <int FMT, int FIT, int V>
__device__ __forceinline__ void get_held(const Held8& in, float (&v)[V], const Place& t, size_t cols, size_t blocks, int lanes_log2) {
    uint32_t c[V / 4];
    load_bytes<V, 1, FIT>(in.codes + t.row * cols + t.vec * V, min(t.left, V), c);
    const uint32_t byte = t.left > 0 ? in.scales[t.row * blocks + (t.vec >> lanes_log2)] : 0u;
    dequantize_block<FMT, V>(c, byte, v);
}

template <int V>
__device__ __forceinline__ void store_codes(uint8_t* to, const uint32_t (&c)[V / 4]) {
    if constexpr (V == 16) *reinterpret_cast<uint4*>(to) = make_uint4(c[0], c[1], c[2], c[3]);
    else *reinterpret_cast<uint2*>(to) = make_uint2(c[0], c[1]);
}

// log2 of the lanes that hold a block.
inline int lanes_log2_of(int block_size, int dtype) {
    int l = 0;
    while ((vec_elems(dtype) << l) < block_size) ++l;
    return l;
}

}  // namespace mxq
