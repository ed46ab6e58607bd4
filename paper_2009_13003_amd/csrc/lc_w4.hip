// Weights in 4 bits with group scales: quantising, reading back, and the product with activations (include/lc_serve.h).
#include "lc_serve.h"

namespace lc {
namespace serve {
namespace {

// ---------------------------------------------------------------- quantising and reading back
// A lane takes eight elements (4 bytes of codes), a group is 4, 8 or 16 neighbouring lanes, and a row's lanes are rounded up to whole
// groups, so that no group is split over wavefronts.  s = bf16(max |w| / 7), q = rint(w (1 / s)) held to +-7; a group too small for 1 / s to be a
// number has scale 0, one that holds what is not finite a NaN for a scale.  Bound by memory: 11008x4096 in fp32 38 us, 5.4 TB/s of what is
// read and written, and read back 29 us, 7 TB/s; both stream past the caches, 16 bytes a lane at a time (through them, and 32 at a time, the two
// took 78 us together).
template <int T, int LANES>
__global__ __launch_bounds__(256) void k_w4_quantize(const void* w, uint64_t ldw, uint8_t* codes, uint64_t codes_pitch, uint16_t* scales,
                                                     uint64_t scales_pitch, uint32_t rows, uint32_t k, uint32_t row_bytes, uint32_t row_lanes, FastDiv div) {
    const uint32_t lane = blockIdx.x * 256u + threadIdx.x;
    const uint32_t row = div(lane), at = lane - row * row_lanes;
    const bool in = row < rows;
    float v[8];
    const uint64_t col = 8ull * at;
    const int valid = in && col < k ? (int)(k - col < 8 ? k - col : 8) : 0;
    load_eight<T>(w, (in ? row : 0) * ldw + col, valid, v);
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) { const uint32_t a = bits_of(v[e]) & 0x7fffffffu; most = a > most ? a : most; }   // (as whole numbers: NaN above infinity above the rest)
    most = max_of_lanes<LANES>(most);
    uint32_t sb = bf16_of(float_of(most) * (1.0f / 7.0f));
    float s = of_bf16(sb), inv = 0.0f;
    if (most >= 0x7f800000u) { sb = 0x7fc0u; }
    else if (s < kSmallest) { sb = 0; }
    else inv = 1.0f / s;
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = fminf(fmaxf(inv == 0.0f ? 0.0f : v[e] * inv, -7.0f), 7.0f);
        word |= (rounded(t, 8.0f) & 15u) << (4 * e);
    }
    if (!in) return;
    if (4ull * at < row_bytes) *reinterpret_cast<uint32_t*>(codes + row * codes_pitch + 4ull * at) = word;
    if (at % LANES == 0) scales[row * scales_pitch + at / LANES] = (uint16_t)sb;
}

template <int T, int G>
__global__ __launch_bounds__(256) void k_w4_dequantize(const uint8_t* codes, uint64_t codes_pitch, const uint16_t* scales, uint64_t scales_pitch,
                                                       void* w, uint64_t ldw, uint32_t rows, uint32_t k, uint32_t row_lanes, FastDiv div) {
    constexpr int N = kAtOnce<T>;
    const uint32_t lane = blockIdx.x * 256u + threadIdx.x;
    const uint32_t row = div(lane), at = lane - row * row_lanes;
    const uint64_t col = (uint64_t)N * at;
    if (row >= rows || col >= k) return;
    const uint8_t* from = codes + row * codes_pitch + col / 2;
    const uint32_t word = N == 8 ? *reinterpret_cast<const uint32_t*>(from) : *reinterpret_cast<const uint16_t*>(from);
    const float s = of_bf16(scales[row * scales_pitch + col / G]);
    float v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (float)((int)(word >> (4 * e) & 15u) - 8) * s;
    store_some<T>(w, row * ldw + col, (int)(k - col < N ? k - col : N), v);
}

// Launches over at most this many rows of `row_lanes` lanes at once, so that lanes are counted in 31 bits.
uint64_t rows_at_once(uint64_t row_lanes) { const uint64_t r = (1ull << 31) / row_lanes; return r ? r : 1; }

template <int T, int LANES>
void quantize(const void* w, uint64_t ldw, const lc_w4& q, hipStream_t s) {
    const uint32_t lanes = (uint32_t)((q.k + q.group - 1) / q.group * LANES);
    const uint64_t step = rows_at_once(lanes);
    for (uint64_t r = 0; r < q.n; r += step) {
        const uint32_t rows = (uint32_t)(q.n - r < step ? q.n - r : step);
        k_w4_quantize<T, LANES><<<(uint32_t)(((uint64_t)rows * lanes + 255) / 256), 256, 0, s>>>(
            static_cast<const uint8_t*>(w) + r * ldw * (T == LC_F32 ? 4 : 2), ldw, static_cast<uint8_t*>(q.codes) + r * q.codes_pitch, q.codes_pitch,
            static_cast<uint16_t*>(q.scales) + r * q.scales_pitch, q.scales_pitch, rows, (uint32_t)q.k, (uint32_t)lc_w4_row_bytes(q.k), lanes, FastDiv(lanes));
    }
}
template <int T, int G>
void dequantize(const lc_w4& q, void* w, uint64_t ldw, hipStream_t s) {
    const uint32_t lanes = (uint32_t)((q.k + kAtOnce<T> - 1) / kAtOnce<T>);
    const uint64_t step = rows_at_once(lanes);
    for (uint64_t r = 0; r < q.n; r += step) {
        const uint32_t rows = (uint32_t)(q.n - r < step ? q.n - r : step);
        k_w4_dequantize<T, G><<<(uint32_t)(((uint64_t)rows * lanes + 255) / 256), 256, 0, s>>>(
            static_cast<const uint8_t*>(q.codes) + r * q.codes_pitch, q.codes_pitch, static_cast<const uint16_t*>(q.scales) + r * q.scales_pitch,
            q.scales_pitch, static_cast<uint8_t*>(w) + r * ldw * (T == LC_F32 ? 4 : 2), ldw, rows, (uint32_t)q.k, lanes, FastDiv(lanes));
    }
}

// ---------------------------------------------------------------- the product
// For 16-bit types codes enter the matrix instructions as whole numbers: a nibble c put where the mantissa of 2^7 (bf16) or 2^6 (fp16) counts
// whole numbers makes 128 + c = q + 136, or 64 + c = q + 72, in little more than two operations for two codes, and 136 (72) times the sum of x is taken
// away first, by the same instruction with a constant for B or as x is brought into LDS.  All of that is exact but for the sums' own rounding in 32 bits,
// which this makes larger by as much as a group's 136 (72) sum |x| is larger than its sum of q x: for x without a mean it leaves some 3e-6 (1e-6) of the
// result, in groups of 128 for |x| and for x with an offset 2e-5 (1e-5), beside the result's own rounding of 1.6e-3 (2e-4).  (fp16 has room for 1024 + c as
// well, but 1032 sum |x| left 1.4e-4.)  fp32 has no such rounding behind it: there codes are converted to sixteenths of q, which bf16 holds exactly
// (three operations for two codes), and x is three bf16 parts that add up to it.  (Lifted codes, 16 + c, left 9e-7
// of the result at a width of 2043 instead of 1e-7.)
template <int T> struct Num;
template <> struct Num<LC_BF16> {
    static constexpr bool kLifted = true;
    static constexpr float kTaken = -136.0f, kUnit = 1.0f;  // what is taken away, and what the operand counts in
    static constexpr int kParts = 1;
    static constexpr uint32_t kBase = 0x43004300u, kLess = 0xC308C308u, kCode = 0x000F000Fu;        // 128, -136, where a code's bits go
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) { return mfma_bf16(a, b, c); }
};
template <> struct Num<LC_F32> {
    static constexpr bool kLifted = false;
    static constexpr float kTaken = 0.0f, kUnit = 16.0f;
    static constexpr int kParts = 3;
    static constexpr uint32_t kBase = 0, kLess = 0, kCode = 0;
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) { return mfma_bf16(a, b, c); }
};
template <> struct Num<LC_F16> {
    static constexpr bool kLifted = true;
    static constexpr float kTaken = -72.0f, kUnit = 1.0f;
    static constexpr int kParts = 1;
    static constexpr uint32_t kBase = 0x54005400u, kLess = 0xD480D480u, kCode = 0x00F000F0u;        // 64, -72
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) { return mfma_f16(a, b, c); }
};
template <int T> __device__ __forceinline__ f32x4 less_of(u32x4 x, f32x4 c) { return Num<T>::mfma(x, u32x4{Num<T>::kLess, Num<T>::kLess, Num<T>::kLess, Num<T>::kLess}, c); }

// Eight codes as operand, in their order.  (The mask is kept in a register that the compiler does not see through: as constants, mask and
// base would take an instruction each.)
template <int T> __device__ __forceinline__ u32x4 codes_as_operand(uint32_t w) {
    u32x4 r;
    uint32_t mask = Num<T>::kCode;
    asm("" : "+v"(mask));
    if (!Num<T>::kLifted) {
        const uint32_t t = turned(w), u = upper_nibbles(t);
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = high_halves(bits_of(low_nibble_of(t, j)), bits_of(low_nibble_of(u, j)));
        return r;
    }
    // The lower nibble of byte j and the upper one, in words in which they stand in that byte as they go into a half: bf16 in its lower four bits, fp16 in
    // its upper ones.
    const uint32_t low = T == LC_F16 ? w << 4 : w, high = T == LC_F16 ? w : w >> 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t pair = __builtin_amdgcn_perm(high, low, 0x0C000C00u | (uint32_t)j | (uint32_t)(4 + j) << 16);      // byte j of low, byte j of high
        r[j] = (pair & mask) | Num<T>::kBase;
    }
    return r;
}

// Eight elements of x from place i, the first `valid` of them (the others zero), as they lie in memory.
template <int T> struct Raw { u32x4 w[T == LC_F32 ? 2 : 1]; };
template <int T> __device__ __forceinline__ Raw<T> x_as_it_is(const void* x, uint64_t i, int valid) {
    Raw<T> r;
    if (valid >= 8) {
#pragma unroll
        for (int j = 0; j < (T == LC_F32 ? 2 : 1); ++j) r.w[j] = load_any<u32x4>(static_cast<const uint8_t*>(x) + i * (T == LC_F32 ? 4 : 2) + 16 * j);
    } else if (T == LC_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.w[e / 4][e % 4] = e < valid ? static_cast<const uint32_t*>(x)[i + e] : 0u;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = 2 * j < valid ? static_cast<const uint16_t*>(x)[i + 2 * j] : 0u;
            const uint32_t hi = 2 * j + 1 < valid ? static_cast<const uint16_t*>(x)[i + 2 * j + 1] : 0u;
            r.w[0][j] = lo | hi << 16;
        }
    }
    return r;
}
// ... and as operand: fp32 as three bf16 parts that add up to it.
template <int T> struct Operand { u32x4 part[Num<T>::kParts]; };
template <int T> __device__ __forceinline__ Operand<T> x_as_operand(const Raw<T>& x) {
    Operand<T> r;
    if (T == LC_F32) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = float_of(x.w[e / 4][e % 4]);
#pragma unroll
        for (int p = 0; p < Num<T>::kParts; ++p) {
#pragma unroll
            for (int j = 0; j < 4; ++j) r.part[p][j] = high_halves(bits_of(v[2 * j]), bits_of(v[2 * j + 1]));
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] -= float_of(bits_of(v[e]) & 0xffff0000u);     // what the part leaves: at most 16, then 8 bits
        }
    } else r.part[0] = x.w[0];
    return r;
}

// The sum of an operand's eight elements (of 16 bits), in 32 bits.
template <int T> __device__ __forceinline__ float sum_of(const Raw<T>& x) {
    float s = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) s = dot_16<T == LC_F16>(x.w[0][j], T == LC_F16 ? 0x3C003C00u : 0x3F803F80u, s);
    return s;
}

struct Product {
    const void* x; uint64_t ldx;
    const uint8_t* codes; uint64_t codes_pitch;
    const uint16_t* scales; uint64_t scales_pitch;
    const void* bias;
    void* y; uint64_t ldy;
    uint32_t m, n, k, row_bytes, groups;
};

// One element of y straight from the formula, where the sums above are not finite: infinity - infinity is not what an infinity in
// x gives, and what is taken away, the sum before its scale or sixteen times a scale may be out of range where the result is not.  One sum after
// another, 32 elements of the width to a step, up to the first NaN, behind which nothing changes any more; a NaN among the scales is looked for first.
// (Element by element to the end an infinity in one row of 4096 took 400 us, 256 rows of NaN by 4096x4096 14.5 ms.)
template <int T, int G>
__device__ __forceinline__ float one_by_formula(const Product& p, uint32_t i, uint32_t j) {
    const uint8_t* codes = p.codes + j * p.codes_pitch;
    const uint16_t* scales = p.scales + j * p.scales_pitch;
    float total = 0;
#pragma unroll 4
    for (uint32_t g = 0; g < p.groups; ++g)
        if ((scales[g] & 0x7fffu) > 0x7f80u) total = __builtin_nanf("");
    for (uint32_t l = 0; l < p.k && total == total; l += 32) {
        const u32x4 words = *reinterpret_cast<const u32x4*>(codes + l / 2);
        const float s = of_bf16(scales[l / G]);
        Raw<T> raw[4];
#pragma unroll
        for (uint32_t o = 0; o < 4; ++o) {
            const uint32_t at = l + 8 * o;
            raw[o] = x_as_it_is<T>(p.x, i * p.ldx + at, at < p.k ? (int)(p.k - at < 8 ? p.k - at : 8) : 0);
        }
#pragma unroll
        for (uint32_t e = 0; e < 32; ++e) {
            const uint32_t at = e % 8, bits = T == LC_F32 ? raw[e / 8].w[at / 4][at % 4] : raw[e / 8].w[0][at / 2] >> (16 * (at % 2)) & 0xffffu;
            const float x = T == LC_F32 ? float_of(bits) : T == LC_BF16 ? of_bf16(bits) : of_f16(bits);
            if (l + e < p.k) total = fmaf(x, (float)((int)(words[e / 8] >> (4 * at) & 15u) - 8) * s, total);      // (q s is exact)
        }
    }
    return total;
}

template <int T, int G>
__device__ __forceinline__ void finish(const Product& p, uint32_t i, uint32_t j, float v) {
    if (!(fabsf(v) < __builtin_inff())) v = one_by_formula<T, G>(p, i, j);
    if (p.bias) v += load_one<T>(p.bias, j);
    store_one<T>(p.y, i * p.ldy + j, v);
}

// Sixteen bytes of codes a lane, 64 to each of 16 rows, as the words that four matrix instructions take.  A lane holds row l % 16,
// quarter l / 16 of the 64 bytes.  With groups of 128 its four words go to four instructions as they are (instruction i and quarter h: the
// eight elements from 32 h + 8 i); with shorter groups they change places between the quarters first, so that every instruction stays
// inside a group (from 32 i + 8 h): word (a, b) of quarter (h1, h0) is the 8 codes from (h1 h0 a b); a and h1, then b and h0 change places.
template <int G> __device__ __forceinline__ u32x4 words_in_order(u32x4 w) {
    if (G == 128) return w;
    const auto p02 = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    const auto p13 = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    const auto q01 = __builtin_amdgcn_permlane16_swap(p02[0], p13[0], false, false);
    const auto q23 = __builtin_amdgcn_permlane16_swap(p02[1], p13[1], false, false);
    return u32x4{q01[0], q01[1], q23[0], q23[1]};
}
template <int G> __device__ __forceinline__ uint32_t place(uint32_t h, uint32_t i) { return G == 128 ? 32 * h + 8 * i : 32 * i + 8 * h; }

// Few rows: up to 16 rows of x by 16 rows of w a workgroup; each wavefront has a part of the width of its own, `per` steps of 128 elements
// (64 bytes of a row of codes), and their sums meet in LDS.  Columns of the matrix instruction are rows of w, so a lane's four results
// share a scale.  S steps are asked for at once: 16 bytes of codes a lane and step, the scales of all S in one load, and x row by row, whole
// lines, put into a piece of LDS of the wavefront's own and read from there as operands.  (Operands straight from memory and a scale at a
// time, one row by 11008x4096: 10.0 us, of which the loads of x took 2.4 and those of scales 1.8; a bare read of the codes takes 4.9, of which
// 2.3 are the launch.)
template <int T, int MR, int WAVES, int S> struct Rows {
    static constexpr int kSize = T == LC_F32 ? 4 : 2, kBytes = S * 128 * kSize, kPitch = kBytes + 16, kLoads = MR * kBytes / 1024;
    static_assert(MR * kBytes % 1024 == 0, "whole loads");
    static uint32_t lds(uint32_t rows) { const uint32_t x = WAVES * rows * kPitch, sums = WAVES * 1024; return x > sums ? x : sums; }
};
template <int T, int G, int MR, int WAVES, int S>
__global__ __launch_bounds__(WAVES * 64) void k_w4_rows(Product p, uint32_t per) {
    using L = Rows<T, MR, WAVES, S>;
    constexpr int PARTS = Num<T>::kParts, PER = G / 32, GROUPS = 128 / G;
    extern __shared__ __align__(16) uint8_t held[];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), c = lane % 16, h = lane / 16;
    const uint32_t n0 = blockIdx.x * 16, m0 = blockIdx.y * MR;
    const uint32_t rows = p.m - m0 < MR ? p.m - m0 : MR;
    const uint32_t steps = p.k / 128;                       // whole ones
    const uint32_t begin = wave * per, end = begin + per < steps ? begin + per : steps;
    const uint32_t row = n0 + c < p.n ? n0 + c : p.n - 1;
    const uint8_t* codes = p.codes + row * p.codes_pitch + 16 * h;
    const uint16_t* scales = p.scales + row * p.scales_pitch;
    uint8_t* own = held + wave * rows * L::kPitch;
    const uint8_t* x_at = own + (c < rows ? c : 0) * L::kPitch;      // (a row beyond the last: any, its results go nowhere)
    struct Batch { u32x4 w[S]; uint16_t s[S * GROUPS]; u32x4 x[L::kLoads]; };
    auto fetch = [&](Batch& f, uint32_t first) {
#pragma unroll
        for (int i = 0; i < S; ++i)
            if (first + i < end) f.w[i] = *reinterpret_cast<const u32x4*>(codes + (first + i) * 64);
        if (first + S <= end) __builtin_memcpy(f.s, scales + first * GROUPS, sizeof(f.s));
        else {
#pragma unroll
            for (int g = 0; g < S * GROUPS; ++g)
                if (first * GROUPS + g < end * GROUPS) f.s[g] = scales[first * GROUPS + g];
        }
#pragma unroll
        for (int l = 0; l < L::kLoads; ++l) {
            const uint32_t at = (l * 64 + lane) * 16, r = at / L::kBytes, b = at % L::kBytes;
            if (r < rows && b < (end - first) * 128 * L::kSize)
                f.x[l] = load_any<u32x4>(static_cast<const uint8_t*>(p.x) + ((m0 + r) * p.ldx + first * 128) * L::kSize + b);
        }
    };
    auto keep = [&](const Batch& f) {
#pragma unroll
        for (int l = 0; l < L::kLoads; ++l) {
            const uint32_t at = (l * 64 + lane) * 16, r = at / L::kBytes, b = at % L::kBytes;
            if (r < rows) *reinterpret_cast<u32x4*>(own + r * L::kPitch + b) = f.x[l];
        }
    };
    f32x4 total = {0, 0, 0, 0};
    auto use = [&](u32x4 codes16, const uint16_t (&s)[GROUPS], const Raw<T> (&raw)[4]) {
        const u32x4 w = words_in_order<G>(codes16);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            f32x4 acc = {0, 0, 0, 0};
            Operand<T> x[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                x[i] = x_as_operand<T>(raw[g * PER + i]);
#pragma unroll
                for (int q = PARTS - 1; q >= 0 && Num<T>::kLifted; --q) acc = less_of<T>(x[i].part[q], acc);
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const u32x4 b = codes_as_operand<T>(w[g * PER + i]);
#pragma unroll
                for (int q = PARTS - 1; q >= 0; --q) acc = Num<T>::mfma(x[i].part[q], b, acc);
            }
            const float scale = of_bf16(s[g]) * Num<T>::kUnit;
#pragma unroll
            for (int r = 0; r < 4; ++r) total[r] = fmaf(acc[r], scale, total[r]);
        }
    };
    auto use_batch = [&](const Batch& f, uint32_t first) {
#pragma unroll
        for (int i = 0; i < S; ++i) {
            if (first + i >= end) break;
            Raw<T> raw[4];
            uint16_t s[GROUPS];
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) s[g] = f.s[i * GROUPS + g];
#pragma unroll
            for (int o = 0; o < 4; ++o)
#pragma unroll
                for (int q = 0; q < L::kSize / 2; ++q)
                    raw[o].w[q] = *reinterpret_cast<const u32x4*>(x_at + (i * 128 + place<G>(h, o)) * L::kSize + 16 * q);
            use(f.w[i], s, raw);
        }
    };
    // (Each set of registers keeps its own loads: moved on to another, they would have to be waited for.)
    Batch two[2];
    if (begin < end) fetch(two[0], begin);
    for (uint32_t first = begin; first < end; first += 2 * S) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const uint32_t now = first + b * S;
            if (now >= end) break;
            keep(two[b]);
            lanes_meet();                                    // (a lane reads what others of its wavefront put there ...)
            if (now + S < end) fetch(two[1 - b], now + S);
            use_batch(two[b], now);
            lanes_meet();                                    // (... which is read before the next batch takes its place)
        }
    }
    if (p.k % 128 && wave == WAVES - 1) {                    // what is left behind the last whole step, straight from memory
        u32x4 w = {0, 0, 0, 0};
        if (steps * 64 + h * 16 < p.row_bytes) w = *reinterpret_cast<const u32x4*>(codes + steps * 64);
        uint16_t s[GROUPS];
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) s[g] = steps * GROUPS + g < p.groups ? scales[steps * GROUPS + g] : 0;
        Raw<T> raw[4];
#pragma unroll
        for (int o = 0; o < 4; ++o) {
            const uint32_t at = steps * 128 + place<G>(h, o);
            raw[o] = x_as_it_is<T>(p.x, (m0 + (c < rows ? c : 0)) * p.ldx + at, at < p.k ? (int)(p.k - at < 8 ? p.k - at : 8) : 0);
        }
        use(w, s, raw);
    }
    __syncthreads();
    float* sums = reinterpret_cast<float*>(held);
#pragma unroll
    for (int r = 0; r < 4; ++r) sums[(wave * 4 + r) * 64 + lane] = total[r];
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < 16 * rows; e += WAVES * 64) {                 // neighbours write neighbours
        const uint32_t i = e / 16, j = e % 16;
        if (n0 + j >= p.n) continue;
        float v = 0;
#pragma unroll
        for (int q = 0; q < WAVES; ++q) v += sums[(q * 4 + i % 4) * 64 + i / 4 * 16 + j];
        finish<T, G>(p, m0 + i, n0 + j, v);
    }
}

// More rows: a tile of 16 MT WM rows of x by 16 NT WN rows of w a workgroup of WM x WN x WK wavefronts, WK of them on different parts of the
// width.  x passes through LDS, 128 WK elements of the width at a time, twice buffered: the next piece is under way in registers while this
// one is worked on, and goes into the other buffer between two of the products of this one: what puts it there then waits in the products' shade.
// Codes come straight into registers and are unpacked by the wavefront that needs them.
// 2048 rows by 4096x11008 (bf16, groups of 128): 224 to 234 us from run to run, 790 to 825 TFLOP/s, 191 on constant data; a plain product of bf16 by the library takes 164 to 167.  x put
// away behind all products 261; matrix instructions are under way a third of the time, vector instructions half of it: unpacking eight codes takes
// eight of them and a scale one for each four sums, and the two share a wavefront's turn.  More loads ahead (three buffers, two pieces in registers)
// cost the third wavefront a SIMD and were slower.
template <int T, int MT, int NT, int WM, int WN, int WK> struct Tile {
    static constexpr int kThreads = 64 * WM * WN * WK, kRows = 16 * MT * WM, kCols = 16 * NT * WN, kParts = Num<T>::kParts;
    // Of 128 elements of the width, kLanes threads bring in a row's, and each kEach rows'.
    static constexpr int kLanes = WN > MT ? 4 * WN / MT : 4, kEach = kLanes * MT / (4 * WN), kItems = 16 / kLanes;
    static_assert(kEach * 4 * WN == kLanes * MT && (kLanes == 4 || kLanes == 8), "whole items");
    // In LDS they stand by fours of eights, and a four by rows, an eight's place in it crossed with the row's number: both the sixteen lanes that put
    // four rows' eights there and the lanes that read sixteen rows' find all banks, whatever four they read.  (By rows of 272 bytes a third of the
    // cycles that LDS was busy went on conflicts.)
    static constexpr uint32_t kFour = kRows * 64, kPart = WK * 4 * kFour;
    static __device__ uint32_t place_of(uint32_t r, uint32_t four, uint32_t eight) { return four * kFour + r * 64 + 16 * (eight ^ (r / 4 % 4)); }
    static constexpr uint32_t kLess = kParts * kPart, kBuffer = kLess + (Num<T>::kLifted ? WK * 4 * kRows * 4 : 0);      // behind x what is taken away for each of (at most four) groups and rows, added up by those who bring x in
    static constexpr uint32_t kSums = WK * kRows * (kCols + 4) * 4;
    static constexpr uint32_t kLds = 2 * kBuffer > kSums ? 2 * kBuffer : kSums;
};
// Which tile a workgroup takes.  Workgroups go round the eight dies, each with an L2 of its own: each die has one stretch of the tiles, ordered down
// panels of kPanel tiles' height, so that those it works on at a time share both rows of x and rows of w.
struct TileAt { uint32_t across, down; };
__device__ __forceinline__ TileAt tile_of(uint32_t wide, uint32_t high) {
    constexpr uint32_t kDies = 8, kPanel = 4;
    const uint32_t tiles = wide * high, die = blockIdx.x % kDies, each = tiles / kDies, more = tiles % kDies;
    const uint32_t t = die * each + (die < more ? die : more) + blockIdx.x / kDies;
    const uint32_t panel = t / (kPanel * wide), in = t - panel * kPanel * wide, tall = high - panel * kPanel < kPanel ? high - panel * kPanel : kPanel;
    return {in / tall, panel * kPanel + in % tall};
}
template <int T, int G, int MT, int NT, int WM, int WN, int WK, int PERSIMD>
__global__ __launch_bounds__(64 * WM * WN * WK, PERSIMD) void k_w4_tiles(Product p) {
    using L = Tile<T, MT, NT, WM, WN, WK>;
    constexpr int PARTS = L::kParts, PER = G / 32, GROUPS = 128 / G;
    extern __shared__ __align__(16) uint8_t held[];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = lane % 16, h = lane / 16;
    const uint32_t wk = wave % WK, wn = wave / WK % WN, wm = wave / WK / WN;
    const auto [across, down] = tile_of((p.n + L::kCols - 1) / L::kCols, (p.m + L::kRows - 1) / L::kRows);
    const uint32_t n0 = across * L::kCols, m0 = down * L::kRows;
    const uint32_t rounds = p.k / (128 * WK);               // whole ones
    const uint8_t* codes[NT];
    const uint16_t* scales[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint32_t j = n0 + 16 * (wn * NT + n) + c, row = j < p.n ? j : p.n - 1;
        codes[n] = p.codes + row * p.codes_pitch + 16 * h;
        scales[n] = p.scales + row * p.scales_pitch;
    }
    struct Step { u32x4 w[NT]; uint16_t s[NT][GROUPS]; };
    auto fetch = [&](Step& f, uint32_t step) {              // a whole step
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            f.w[n] = *reinterpret_cast<const u32x4*>(codes[n] + step * 64);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) f.s[n][g] = scales[n][step * GROUPS + g];
        }
    };
    auto fetch_rest = [&](Step& f, uint32_t step) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            f.w[n] = u32x4{0, 0, 0, 0};
            if (step * 64 + h * 16 < p.row_bytes) f.w[n] = *reinterpret_cast<const u32x4*>(codes[n] + step * 64);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) f.s[n][g] = step * GROUPS + g < p.groups ? scales[n][step * GROUPS + g] : 0;
        }
    };
    struct Piece { Raw<T> x[L::kEach][L::kItems]; };
    const uint32_t own = threadIdx.x % L::kLanes;
    const uint8_t* x_from[L::kEach];
    uint32_t first[L::kEach], row_of[L::kEach];
#pragma unroll
    for (int u = 0; u < L::kEach; ++u) {
        const uint32_t unit = threadIdx.x / L::kLanes + u * (L::kThreads / L::kLanes), r = unit % L::kRows;
        row_of[u] = r, first[u] = unit / L::kRows * 128 + 8 * own;
        x_from[u] = static_cast<const uint8_t*>(p.x) + ((m0 + r < p.m ? m0 + r : p.m - 1) * p.ldx + first[u]) * (T == LC_F32 ? 4 : 2);      // (a row beyond the last: any, its results go nowhere)
    }
    auto bring = [&](Piece& next, uint32_t round, bool whole) {
        const uint32_t from = round * WK * 128;
#pragma unroll
        for (int u = 0; u < L::kEach; ++u)
#pragma unroll
            for (int i = 0; i < L::kItems; ++i) {
                const uint32_t at = from + first[u] + 8 * L::kLanes * i;
                next.x[u][i] = x_as_it_is<T>(x_from[u], from + 8 * L::kLanes * i, whole ? 8 : at < p.k ? (int)(p.k - at < 8 ? p.k - at : 8) : 0);
            }
    };
    auto keep = [&](const Piece& next, uint32_t buffer) {
        uint8_t* to = held + buffer * L::kBuffer;
#pragma unroll
        for (int u = 0; u < L::kEach; ++u) {
            const uint32_t at = L::place_of(row_of[u], first[u] / 32, own % 4);
#pragma unroll
            for (int i = 0; i < L::kItems; ++i) {
                const Operand<T> x = x_as_operand<T>(next.x[u][i]);
#pragma unroll
                for (int q = 0; q < PARTS; ++q) *reinterpret_cast<u32x4*>(to + q * L::kPart + at + L::kLanes / 4 * i * L::kFour) = x.part[q];
            }
            if (!Num<T>::kLifted) continue;
            constexpr int EIGHTS = G / 8, TOGETHER = EIGHTS > L::kLanes ? EIGHTS / L::kLanes : 1;
#pragma unroll
            for (int i = 0; i < L::kItems; i += TOGETHER) {
                float sum = 0;
#pragma unroll
                for (int t = 0; t < TOGETHER; ++t) sum += sum_of<T>(next.x[u][i + t]);
                const float taken = Num<T>::kTaken * sum_of_lanes<(EIGHTS < L::kLanes ? EIGHTS : L::kLanes)>(sum);
                *reinterpret_cast<float*>(to + L::kLess + ((first[u] + 8 * L::kLanes * i) / G * L::kRows + row_of[u]) * 4) = taken;      // (a group's lanes all write it: no branch)
            }
        }
    };
    f32x4 total[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) total[m][n] = f32x4{0, 0, 0, 0};
    uint32_t at_eight[G == 128 ? 4 : 1];                    // where the eights of the lane stand in LDS
#pragma unroll
    for (int o = 0; o < (G == 128 ? 4 : 1); ++o) at_eight[o] = L::place_of(16 * MT * wm + c, 4 * wk + (G == 128 ? h : 0), G == 128 ? o : h);
    auto use = [&](const Step& f, const uint8_t* x_at, const uint8_t* less_at, auto meanwhile) {
        u32x4 w[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) w[n] = words_in_order<G>(f.w[n]);
        u32x4 x[2][MT][PARTS];
        auto read = [&](u32x4 (&to)[MT][PARTS], int o) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int q = 0; q < PARTS; ++q) to[m][q] = *reinterpret_cast<const u32x4*>(x_at + (G == 128 ? at_eight[o] : at_eight[0] + o * L::kFour) + m * 1024 + q * L::kPart);
        };
        read(x[0], 0);
        f32x4 acc[NT][MT];
#pragma unroll
        for (int o = 0; o < 4; ++o) {                       // eights of the width, the next one's x on its way while one is worked on
            const int g = o / PER;
            if (o < 3) read(x[(o + 1) % 2], o + 1);
            if (o % PER == 0) {
                f32x4 less[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    less[m] = Num<T>::kLifted ? *reinterpret_cast<const f32x4*>(less_at + (g * L::kRows + 16 * m) * 4) : f32x4{0, 0, 0, 0};
#pragma unroll
                    for (int n = 0; n < NT; ++n) acc[n][m] = less[m];
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const u32x4 b = codes_as_operand<T>(w[n][o]);
#pragma unroll
                for (int q = PARTS - 1; q >= 0; --q)
#pragma unroll
                    for (int m = 0; m < MT; ++m) acc[n][m] = Num<T>::mfma(x[o % 2][m][q], b, acc[n][m]);
            }
            __builtin_amdgcn_sched_barrier(0);              // (else all reads of x come first, and their registers)
            if (o == 1) meanwhile();
            if (o % PER == PER - 1) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float s = of_bf16(f.s[n][g]) * Num<T>::kUnit;
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int r = 0; r < 4; ++r) total[m][n][r] = fmaf(acc[n][m][r], s, total[m][n][r]);
                }
            }
        }
    };
    // Round r works on buffer r % 2 and on the codes that were asked for two rounds before; x of round r + 1 is put into the other buffer
    // meanwhile.  Two rounds are written out, so that every set of registers keeps its own loads and none has to be moved on, and the
    // last rounds ask for the last piece again instead of asking whether there is one: a branch there costs more than the loads.
    Piece next;
    Step codes_of[2];
    const uint8_t* less_at = held + L::kLess + (wk * GROUPS * L::kRows + 16 * MT * wm + 4 * h) * 4;
    if (rounds) {
        const uint32_t last = rounds - 1;
        bring(next, 0, true);
        fetch(codes_of[0], wk);
        keep(next, 0);
        fetch(codes_of[1], (last < 1 ? last : 1) * WK + wk);
        bring(next, last < 1 ? last : 1, true);
        __syncthreads();
        uint32_t round = 0;
        for (; round < last; round += 2) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                use(codes_of[b], held + b * L::kBuffer, less_at + b * L::kBuffer, [&]() {
                    keep(next, 1 - b);
                    bring(next, round + b + 2 < last ? round + b + 2 : last, true);
                });
                fetch(codes_of[b], (round + b + 2 < last ? round + b + 2 : last) * WK + wk);
                __syncthreads();
            }
        }
        if (round == last) use(codes_of[0], held, less_at, []() {});
        __syncthreads();
    }
    if (p.k % (128 * WK)) {                                  // what is left behind the last whole round
        bring(next, rounds, false);
        fetch_rest(codes_of[0], rounds * WK + wk);
        keep(next, 0);
        __syncthreads();
        use(codes_of[0], held, less_at, []() {});
        __syncthreads();
    }
    float* sums = reinterpret_cast<float*>(held);
    constexpr uint32_t kSumPitch = L::kCols + 4;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) sums[(wk * L::kRows + 16 * (wm * MT + m) + 4 * h + r) * kSumPitch + 16 * (wn * NT + n) + c] = total[m][n][r];
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < L::kRows * L::kCols; e += L::kThreads) {
        const uint32_t r = e / L::kCols, j = e % L::kCols;
        if (m0 + r >= p.m || n0 + j >= p.n) continue;
        float v = 0;
#pragma unroll
        for (int q = 0; q < WK; ++q) v += sums[(q * L::kRows + r) * kSumPitch + j];
        finish<T, G>(p, m0 + r, n0 + j, v);
    }
}

template <int T>
__global__ __launch_bounds__(256) void k_w4_bias_only(Product p) {      // k = 0
    for (uint64_t e = blockIdx.x * 256ull + threadIdx.x; e < (uint64_t)p.m * p.n; e += gridDim.x * 256ull) {
        const uint64_t i = e / p.n, j = e % p.n;
        store_one<T>(p.y, i * p.ldy + j, p.bias ? load_one<T>(p.bias, j) : 0.0f);
    }
}

// A launch's threads have to be fewer than 2^32.
constexpr uint64_t kMostRows = 1ull << 19;                  // of x
constexpr uint64_t kAtOnce16 = 1ull << 22, kAtOnceTiles = (1ull << 17) - 128;      // rows of w in a launch, for up to 16 rows of x and for more
constexpr uint32_t kMostBiasBlocks = 1u << 22;
template <typename L> constexpr bool kLaunches = (kMostRows + L::kRows - 1) / L::kRows * ((kAtOnceTiles + L::kCols - 1) / L::kCols) * L::kThreads < 1ull << 32;

template <int T, int G, int MR, int WAVES, int S>
void product_of_rows(const Product& p, hipStream_t s) {
    const uint32_t steps = p.k / 128, rows = p.m < MR ? p.m : MR;
    k_w4_rows<T, G, MR, WAVES, S><<<dim3((p.n + 15) / 16, (p.m + MR - 1) / MR), WAVES * 64, Rows<T, MR, WAVES, S>::lds(rows), s>>>(p, (steps + WAVES - 1) / WAVES);
}

template <int T, int G, int MT, int NT, int WM, int WN, int WK, int PERSIMD>
void product_of_tiles(const Product& p, hipStream_t s) {
    using L = Tile<T, MT, NT, WM, WN, WK>;
    static_assert(L::kLds <= 160 * 1024, "LDS of a compute unit");
    const uint32_t grid = (p.n + L::kCols - 1) / L::kCols * ((p.m + L::kRows - 1) / L::kRows);
    k_w4_tiles<T, G, MT, NT, WM, WN, WK, PERSIMD><<<grid, L::kThreads, L::kLds, s>>>(p);
}

// More wavefronts a workgroup where there are few workgroups, as long as each has some steps to go, and two steps at a time where that leaves
// enough wavefronts to a SIMD.  Measured with 4, 8 and 16 wavefronts a workgroup, us: one row by 4096x4096 (bf16, groups of 128) 4.6, 4.3, 4.4, by
// 11008x4096 7.8, 8.9, 11.5, by 8192x8192 10.6, 9.6, 13.1, by 32000x4096 (groups of 32) 20.0, 21.6, 28.7, by 4096x11008 (32) 11.8, 9.0, 8.0; 13 rows
// there 19.5, 12.5, 11.0; one row by 4096x4096 in fp32 8.8, 6.9, 6.9, 16 rows by 11008x4096 20.6, 24.4, 47.5.  Two steps instead of one: 11008x4096
// 7.8 for 8.7 with 4 wavefronts, 8192x8192 9.6 for 11.0 with 8; but in groups of 32 32000x4096 21.1 for 20.0.
// Sixteen for eight where workgroups are no more than compute units (kernels in a row, bf16, groups of 128): 13 rows by 4096x1500 4.0 for 3.8, x2048 3.9
// for 4.1, x4096 6.0 for 6.5, x8192 9.4 for 10.0, x16384 15.1 for 16.7, by 512x2048 3.6 for 3.8; so from a step for each on.  One row by 4096x2048 3.4 for
// 3.3, x4096 4.9 for 5.2, x8192 7.5 for 7.3, x11008 7.5 for 8.4, x16384 11.4 for 10.9, by 1000x8192 6.3 for 5.7, x11008 6.5 for 7.0, in groups of 32 by
// 4096x4096 5.2 for 5.4, x8192 7.9 for 7.9, x11008 8.3 for 9.3, x16384 12.0 for 12.6, by 1000x4096 4.5 for 4.4, x8192 6.7 for 7.0: from four steps for each on.  By
// 6144 and more columns of y sixteen are slower at any width (13 rows by 6144x11008 17.4 for 16.8).
template <int T, int G, int MR>
void product_of_few(const Product& p, hipStream_t s) {
    constexpr int FOUR = T != LC_F32 && G == 128 ? 2 : 1, EIGHT = T != LC_F32 && G == 128 && MR == 4 ? 2 : 1;
    const uint32_t blocks = (p.n + 15) / 16;
    if constexpr (T != LC_F32)
        if (blocks <= 256 && p.k >= (MR == 16 ? 1 : 4) * 16 * 128) return product_of_rows<T, G, MR, 16, 1>(p, s);
    if (blocks <= 512) product_of_rows<T, G, MR, 8, EIGHT>(p, s);
    else product_of_rows<T, G, MR, 4, FOUR>(p, s);
}

template <int T, int G>
void product(const Product& p, hipStream_t s) {
    if (p.m > 16) {
        // The smaller the tile, the more wavefronts share a tile's width: smaller tiles as long as they fit the chip in one go, those of 64 x 64 two a
        // compute unit.  Measured in tiles of 32 x 16, 32 x 32, 32 x 64, 64 x 64 and 64 x 128, us (bf16, groups of 128): 24 rows by 4096x4096 8.4, 10.3,
        // 13.2, 16.1, 29.8; 64 rows 15.7, 10.9, 13.9, 16.7, 32.8; 100 rows 29.4, 20.3, 14.0, 16.8, 32.9; 256 rows 57.2, 38.9, 26.8, 17.1, 32.8; 512
        // rows 113, 75.9, 52.0, 28.8, 33.4; 1024 rows 223, 150, 102, 53.3, 48.2; 128 by 11008x4096 77.8, 57.1, 39.4, 28.5, 33.1.
        // fp32, whose three parts take three times the LDS, in tiles of 16 x 32, 32 x 64 and 32 x 128: 24 rows by 4096x4096 13.9, 21.0, 37.6; 100 rows
        // 51.0, 21.9, 38.3; 256 rows 101, 42.0, 39.3; 1024 rows 400, 163, 97.7.
        const auto fits = [&](uint32_t rows, uint32_t cols, uint32_t blocks = 256) { return (uint64_t)((p.m + rows - 1) / rows) * ((p.n + cols - 1) / cols) <= blocks; };
        if constexpr (T == LC_F32) {
            if (fits(16, 32)) product_of_tiles<T, G, 1, 2, 1, 1, 4, 1>(p, s);
            else if (fits(32, 64)) product_of_tiles<T, G, 2, 1, 1, 4, 2, 1>(p, s);
            else product_of_tiles<T, G, 2, 2, 1, 4, 1, 1>(p, s);
            static_assert(kLaunches<Tile<T, 2, 2, 1, 4, 1>>, "threads of the largest launch");      // (the others' tiles are a few hundred)
        } else {
            if (p.m <= 32) product_of_tiles<T, G, 2, 1, 1, 1, 8, 1>(p, s);
            else if (fits(32, 32)) product_of_tiles<T, G, 2, 2, 1, 1, 8, 1>(p, s);
            else if (fits(32, 64)) product_of_tiles<T, G, 2, 2, 1, 2, 4, 1>(p, s);
            else if (fits(64, 64, 512)) product_of_tiles<T, G, 4, 1, 1, 4, 2, 1>(p, s);
            else product_of_tiles<T, G, 4, 2, 1, 4, 1, 3>(p, s);
            static_assert(kLaunches<Tile<T, 4, 2, 1, 4, 1>>, "threads of the largest launch");
        }
        return;
    }
    if (p.m <= 4) product_of_few<T, G, 4>(p, s);
    else product_of_few<T, G, 16>(p, s);
}

// Whether a matrix in 4 bits is one the kernels can take.
bool bad(const lc_w4* q) {
    if (!q || (q->group != 32 && q->group != 64 && q->group != 128) || q->n > 0x7fffffffull || q->k > 0x7fffffffull) return true;
    if (q->n == 0 || q->k == 0) return false;
    return !q->codes || !q->scales || off(q->codes, 16) || off(q->scales, 2) || q->codes_pitch % 16 || q->codes_pitch < lc_w4_row_bytes(q->k) ||
           q->scales_pitch < (q->k + q->group - 1) / q->group || q->codes_pitch > (1ull << 40) || q->scales_pitch > (1ull << 40);
}


}  // namespace
}  // namespace serve
}  // namespace lc

using namespace lc::serve;

#define LC_BY_GROUP(call, T, q) \
    do { if ((q).group == 32) call(T, 32); else if ((q).group == 64) call(T, 64); else call(T, 128); } while (0)
#define LC_BY_TYPE(call, dtype, q) \
    do { if ((dtype) == LC_F32) LC_BY_GROUP(call, LC_F32, q); else if ((dtype) == LC_BF16) LC_BY_GROUP(call, LC_BF16, q); \
         else LC_BY_GROUP(call, LC_F16, q); } while (0)

extern "C" {

size_t lc_w4_row_bytes(uint64_t k) { return k > 0x7fffffffull ? 0 : (size_t)(((k + 1) / 2 + 15) / 16 * 16); }

int lc_w4_quantize(const void* w, uint64_t ldw, int dtype, const lc_w4* w4, void* stream) {
    if (!served_type(dtype) || bad(w4)) return LC_ERR_BADARG;
    if (w4->n == 0 || w4->k == 0) return LC_OK;
    if (!w || off(w, size_of(dtype)) || ldw < w4->k || ldw > (1ull << 40)) return LC_ERR_BADARG;
    const lc_w4 q = *w4;
    hipStream_t s = static_cast<hipStream_t>(stream);
#define CALL(T, G) quantize<T, G / 8>(w, ldw, q, s)
    LC_BY_TYPE(CALL, dtype, q);
#undef CALL
    return launched();
}

int lc_w4_dequantize(const lc_w4* w4, void* w, uint64_t ldw, int dtype, void* stream) {
    if (!served_type(dtype) || bad(w4)) return LC_ERR_BADARG;
    if (w4->n == 0 || w4->k == 0) return LC_OK;
    if (!w || off(w, size_of(dtype)) || ldw < w4->k || ldw > (1ull << 40)) return LC_ERR_BADARG;
    const lc_w4 q = *w4;
    hipStream_t s = static_cast<hipStream_t>(stream);
#define CALL(T, G) dequantize<T, G>(q, w, ldw, s)
    LC_BY_TYPE(CALL, dtype, q);
#undef CALL
    return launched();
}

int lc_w4_matmul(const void* x, uint64_t ldx, uint64_t m, const lc_w4* w4, const void* bias, void* y, uint64_t ldy, int dtype, void* stream) {
    if (!served_type(dtype) || bad(w4) || m > kMostRows) return LC_ERR_BADARG;
    if (m == 0 || w4->n == 0) return LC_OK;
    const uintptr_t size = size_of(dtype);
    if (!y || off(y, size) || ldy < w4->n || ldy > (1ull << 40) || (bias && off(bias, size))) return LC_ERR_BADARG;
    if (w4->k && (!x || off(x, size) || ldx < w4->k || ldx > (1ull << 40))) return LC_ERR_BADARG;
    const lc_w4 q = *w4;
    const Product p = {x, ldx, static_cast<const uint8_t*>(q.codes), q.codes_pitch, static_cast<const uint16_t*>(q.scales), q.scales_pitch, bias, y, ldy,
                       (uint32_t)m, (uint32_t)q.n, (uint32_t)q.k, (uint32_t)lc_w4_row_bytes(q.k), (uint32_t)((q.k + q.group - 1) / q.group)};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (q.k == 0) {
        const uint64_t all = ((uint64_t)p.m * p.n + 255) / 256;
        const uint32_t blocks = all < kMostBiasBlocks ? (uint32_t)all : kMostBiasBlocks;
        if (dtype == LC_F32) k_w4_bias_only<LC_F32><<<blocks, 256, 0, s>>>(p);
        else if (dtype == LC_BF16) k_w4_bias_only<LC_BF16><<<blocks, 256, 0, s>>>(p);
        else k_w4_bias_only<LC_F16><<<blocks, 256, 0, s>>>(p);
        return launched();
    }
    const uint64_t step = m > 16 ? kAtOnceTiles : kAtOnce16;
    for (uint64_t j = 0; j < q.n; j += step) {
        Product some = p;
        some.codes += j * q.codes_pitch, some.scales += j * q.scales_pitch, some.n = (uint32_t)(q.n - j < step ? q.n - j : step);
        some.y = static_cast<uint8_t*>(y) + j * size;
        if (bias) some.bias = static_cast<const uint8_t*>(bias) + j * size;
#define CALL(T, G) product<T, G>(some, s)
        LC_BY_TYPE(CALL, dtype, q);
#undef CALL
    }
    return launched();
}

}  // extern "C"
