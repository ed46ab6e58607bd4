// Shared between the kernels of the serving operators (lc_w4.hip, lc_i8.hip, lc_kv.hip, lc_prompt.hip, lc_pages.hip, lc_draft.hip): element types, packing, matrix instructions.  gfx950 only.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include "../../include/lc_serve.h"

namespace lc {
namespace serve {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

constexpr float kSmallest = 1.17549435e-38f;      // 2^-126: scales below it are stored as zero, so that 1/s stays finite

inline bool served_type(int dtype) { return dtype == LC_F32 || dtype == LC_BF16 || dtype == LC_F16; }
inline bool off(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
inline int launched() { return hipGetLastError() == hipSuccess ? LC_OK : LC_ERR_HIP; }
inline uintptr_t size_of(int dtype) { return dtype == LC_F32 ? 4 : 2; }

// n / d for 32-bit n by a product with what the host worked out once (round-up method: exact for every n).
struct FastDiv {
    uint32_t d, m, s;
    FastDiv(uint32_t d_ = 1) : d(d_), m(0), s(0) {
        while (s < 32 && (1ull << s) < d) ++s;
        m = (uint32_t)(((1ull << 32) * ((1ull << s) - d)) / d + 1);
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const {
        const uint32_t t = __umulhi(m, n);
        return s == 0 ? n : (t + ((n - t) >> 1)) >> (s - 1);
    }
};

// 16 bytes from anywhere that suits the element (global loads need no more than that here).
template <typename V> __device__ __forceinline__ V load_any(const void* p) { V v; __builtin_memcpy(&v, p, sizeof(V)); return v; }
// ... and the same past the caches, for what is read or written once and too long to stay in them.
template <typename V> __device__ __forceinline__ V load_once(const void* p) {
    typedef V __attribute__((aligned(2))) Any;
    return __builtin_nontemporal_load(static_cast<const Any*>(p));
}
template <typename V> __device__ __forceinline__ void store_once(void* p, V v) {
    typedef V __attribute__((aligned(2))) Any;
    __builtin_nontemporal_store(v, static_cast<Any*>(p));
}

__device__ __forceinline__ uint32_t bits_of(float f) { return __float_as_uint(f); }
__device__ __forceinline__ float float_of(uint32_t b) { return __uint_as_float(b); }

// To nearest even; a NaN stays one.
__device__ __forceinline__ uint32_t bf16_of(float f) {
    const uint32_t b = bits_of(f);
    const uint32_t r = (b + 0x7fffu + ((b >> 16) & 1u)) >> 16;
    return (b & 0x7fffffffu) > 0x7f800000u ? 0x7fc0u : r;
}
__device__ __forceinline__ float of_bf16(uint32_t b) { return float_of(b << 16); }
__device__ __forceinline__ uint32_t f16_of(float f) { const _Float16 h = (_Float16)f; uint16_t u; __builtin_memcpy(&u, &h, 2); return u; }
__device__ __forceinline__ float of_f16(uint32_t b) { const uint16_t u = (uint16_t)b; _Float16 h; __builtin_memcpy(&h, &u, 2); return (float)h; }

// One element of an array of type T (LC_F32, LC_BF16, LC_F16).
template <int T> __device__ __forceinline__ float load_one(const void* p, uint64_t i) {
    if (T == LC_F32) return static_cast<const float*>(p)[i];
    const uint32_t u = static_cast<const uint16_t*>(p)[i];
    return T == LC_BF16 ? of_bf16(u) : of_f16(u);
}
template <int T> __device__ __forceinline__ void store_one(void* p, uint64_t i, float v) {
    if (T == LC_F32) static_cast<float*>(p)[i] = v;
    else static_cast<uint16_t*>(p)[i] = (uint16_t)(T == LC_BF16 ? bf16_of(v) : f16_of(v));
}
// Eight elements in a row, the first `valid` of them (the others read as zero, or are not written).
template <int T> __device__ __forceinline__ void load_eight(const void* p, uint64_t i, int valid, float v[8]) {
    if (valid >= 8) {
        if (T == LC_F32) {
            const f32x4 a = load_once<f32x4>(static_cast<const float*>(p) + i), b = load_once<f32x4>(static_cast<const float*>(p) + i + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
        } else {
            const u32x4 a = load_once<u32x4>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t u = a[e / 2];
                v[e] = T == LC_BF16 ? float_of(e % 2 ? u & 0xffff0000u : u << 16) : of_f16(e % 2 ? u >> 16 : u & 0xffffu);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < valid ? load_one<T>(p, i + e) : 0.0f;
    }
}
// The elements a lane writes at once, 16 bytes, the first `valid` of them: the lanes' stores then fill whole lines, past the caches.  (8 fp32
// elements a lane, in two stores of every other 16 bytes: 69 us instead of 33 through the caches for 11008x4096 read back.)
template <int T> constexpr int kAtOnce = T == LC_F32 ? 4 : 8;
template <int T> __device__ __forceinline__ void store_some(void* p, uint64_t i, int valid, const float* v) {
    if (valid >= kAtOnce<T>) {
        if (T == LC_F32) store_once(static_cast<float*>(p) + i, f32x4{v[0], v[1], v[2], v[3]});
        else {
            u32x4 a;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                a[e] = T == LC_BF16 ? bf16_of(v[2 * e]) | bf16_of(v[2 * e + 1]) << 16 : f16_of(v[2 * e]) | f16_of(v[2 * e + 1]) << 16;
            store_once(static_cast<uint16_t*>(p) + i, a);
        }
    } else {
#pragma unroll
        for (int e = 0; e < kAtOnce<T>; ++e)
            if (e < valid) store_one<T>(p, i + e, v[e]);
    }
}

// Four elements in a row, aligned to their size together.
template <int T> __device__ __forceinline__ void store_four(void* p, uint64_t i, f32x4 v) {
    if (T == LC_F32) { *reinterpret_cast<f32x4*>(static_cast<float*>(p) + i) = v; return; }
    const u32x2 w = T == LC_BF16 ? u32x2{bf16_of(v[0]) | bf16_of(v[1]) << 16, bf16_of(v[2]) | bf16_of(v[3]) << 16}
                                 : u32x2{f16_of(v[0]) | f16_of(v[1]) << 16, f16_of(v[2]) | f16_of(v[3]) << 16};
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p) + i) = w;
}

// Between what lanes of a wavefront put into LDS and what others of it read there, or the other way round: the compiler moves neither past it.  (A wavefront's
// LDS operations come about in their order, so it takes no instruction.)
__device__ __forceinline__ void lanes_meet() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// The largest of `lanes` neighbouring lanes' values in every one of them (lanes: 4, 8, 16 or 32, aligned).
template <int LANES> __device__ __forceinline__ uint32_t max_of_lanes(uint32_t v) {
#define LC_DPP_MAX(ctrl) { const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, false); v = v > o ? v : o; }
    if (LANES >= 2) LC_DPP_MAX(0xB1)      // the other of each two
    if (LANES >= 4) LC_DPP_MAX(0x4E)      // the other two of each four
    if (LANES >= 8) LC_DPP_MAX(0x141)     // the other four of each eight
    if (LANES >= 16) LC_DPP_MAX(0x140)    // the other eight of each sixteen
#undef LC_DPP_MAX
    if (LANES >= 32) { const uint32_t o = (uint32_t)__shfl_xor((int)v, 16); v = v > o ? v : o; }
    return v;
}

// The sum over 4, 8 or 16 neighbouring lanes in every one of them.
template <int LANES> __device__ __forceinline__ float sum_of_lanes(float v) {
#define LC_DPP_SUM(ctrl) v += float_of((uint32_t)__builtin_amdgcn_update_dpp(0, (int)bits_of(v), ctrl, 0xf, 0xf, false))
    LC_DPP_SUM(0xB1);
    LC_DPP_SUM(0x4E);
    if (LANES >= 8) LC_DPP_SUM(0x141);
    if (LANES >= 16) LC_DPP_SUM(0x140);
#undef LC_DPP_SUM
    return v;
}

// rint(t) + bias for |t| <= 127 in the low bits: added to 1.5 * 2^23 the sum has no room for a fraction, and its rounding is the
// one to nearest even.
__device__ __forceinline__ uint32_t rounded(float t, float bias) { return bits_of(t + (12582912.0f + bias)); }

// Nibble j of a word of 4-bit codes as a sixteenth of what it stands for: the instruction reads four bits as a two's complement number
// of sixteenths, which the code with its top bit turned round is.
__device__ __forceinline__ uint32_t turned(uint32_t w) { return w ^ 0x88888888u; }
__device__ __forceinline__ float nibble_of(uint32_t w, int j) { return __builtin_amdgcn_cvt_off_f32_i4((int)(w >> (4 * j))); }
// ... and the lower nibble of byte j, which the instruction picks by itself; the upper ones' word, which the compiler does not see through, so
// that it is shifted once and not for every byte.
__device__ __forceinline__ float low_nibble_of(uint32_t w, int j) { return __builtin_amdgcn_cvt_off_f32_i4((int)(w >> (8 * j) & 255u)); }
__device__ __forceinline__ uint32_t upper_nibbles(uint32_t w) {
    w >>= 4;
    asm("" : "+v"(w));
    return w;
}

// D = A B + C, 16 x 16 x 32: lane l gives row l % 16 of A and column l % 16 of B, eight places of the inner dimension of its
// own (the same ones for A and B) per quarter l / 16, and receives column l % 16, rows 4 (l / 16) + 0..3 of D.
__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
    bf16x8 x, y; __builtin_memcpy(&x, &a, 16); __builtin_memcpy(&y, &b, 16);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f16(u32x4 a, u32x4 b, f32x4 c) {
    f16x8 x, y; __builtin_memcpy(&x, &a, 16); __builtin_memcpy(&y, &b, 16);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0);
}

// c plus the two products of a pair, in 32 bits.
template <bool HALF> __device__ __forceinline__ float dot_16(uint32_t a, uint32_t b, float c) {
    if (HALF) {
        typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
        f16x2 x, y; __builtin_memcpy(&x, &a, 4); __builtin_memcpy(&y, &b, 4);
        return __builtin_amdgcn_fdot2(x, y, c, false);
    }
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    bf16x2 x, y; __builtin_memcpy(&x, &a, 4); __builtin_memcpy(&y, &b, 4);
    return __builtin_amdgcn_fdot2_f32_bf16(x, y, c, false);
}

// a and b rounded to bf16 (to nearest even), a below b.
__device__ __forceinline__ uint32_t rounded_halves(float a, float b) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const bf16x2 r = __builtin_convertvector(f32x2{a, b}, bf16x2);
    uint32_t u; __builtin_memcpy(&u, &r, 4);
    return u;
}
// The high halves of a and b, a's below b's.
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

}  // namespace serve
}  // namespace lc
