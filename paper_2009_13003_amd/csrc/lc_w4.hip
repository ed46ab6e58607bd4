// Weights in 4 bits with group scales: quantising, reading back, and the product with activations (include/lc_serve.h).
#include "lc_serve.h"

namespace lc {
namespace serve {
namespace {

// ---------------------------------------------------------------- quantising and reading back
// A lane takes eight elements (4 bytes of codes), a group is 4, 8 or 16 neighbouring lanes, and a row's lanes are rounded up to whole
// groups, so that no group is split over wavefronts.
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

template <int T, int LANES>
__global__ __launch_bounds__(256) void k_w4_dequantize(const uint8_t* codes, uint64_t codes_pitch, const uint16_t* scales, uint64_t scales_pitch,
                                                       void* w, uint64_t ldw, uint32_t rows, uint32_t k, uint32_t row_lanes, FastDiv div) {
    const uint32_t lane = blockIdx.x * 256u + threadIdx.x;
    const uint32_t row = div(lane), at = lane - row * row_lanes;
    const uint64_t col = 8ull * at;
    if (row >= rows || col >= k) return;
    const uint32_t word = *reinterpret_cast<const uint32_t*>(codes + row * codes_pitch + 4ull * at);
    const float s = of_bf16(scales[row * scales_pitch + at / LANES]);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)((int)(word >> (4 * e) & 15u) - 8) * s;
    store_eight<T>(w, row * ldw + col, (int)(k - col < 8 ? k - col : 8), v);
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
template <int T, int LANES>
void dequantize(const lc_w4& q, void* w, uint64_t ldw, hipStream_t s) {
    const uint32_t lanes = (uint32_t)((q.k + 7) / 8);
    const uint64_t step = rows_at_once(lanes);
    for (uint64_t r = 0; r < q.n; r += step) {
        const uint32_t rows = (uint32_t)(q.n - r < step ? q.n - r : step);
        k_w4_dequantize<T, LANES><<<(uint32_t)(((uint64_t)rows * lanes + 255) / 256), 256, 0, s>>>(
            static_cast<const uint8_t*>(q.codes) + r * q.codes_pitch, q.codes_pitch, static_cast<const uint16_t*>(q.scales) + r * q.scales_pitch,
            q.scales_pitch, static_cast<uint8_t*>(w) + r * ldw * (T == LC_F32 ? 4 : 2), ldw, rows, (uint32_t)q.k, lanes, FastDiv(lanes));
    }
}

// ---------------------------------------------------------------- the product
// Codes enter the matrix instructions as whole numbers: a nibble c put into the mantissa of 16 makes 16 + c = q + 24 in two
// operations for two codes, and -24 times the sum of x, which the same instruction works out with a constant for B, takes the 24
// away again.  All of that is exact but for the sums' own rounding in 32 bits.
template <int T> struct Num;
template <> struct Num<LC_BF16> {
    static constexpr int kParts = 1;
    static constexpr uint32_t kMask = 0x00780078u, kBase = 0x41804180u, kMinus24 = 0xC1C0C1C0u;
    static constexpr int kAt = 3;           // where a nibble lies in the mantissa
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) { return mfma_bf16(a, b, c); }
};
template <> struct Num<LC_F32> : Num<LC_BF16> { static constexpr int kParts = 3; };
template <> struct Num<LC_F16> {
    static constexpr int kParts = 1;
    static constexpr uint32_t kMask = 0x03C003C0u, kBase = 0x4C004C00u, kMinus24 = 0xCE00CE00u;
    static constexpr int kAt = 6;
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) { return mfma_f16(a, b, c); }
};

// Eight codes as operand: elements 0 4 1 5 2 6 3 7 in this order.
template <int T> __device__ __forceinline__ u32x4 codes_as_operand(uint32_t w) {
    u32x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int up = Num<T>::kAt - 4 * j;
        r[j] = ((up >= 0 ? w << (up & 31) : w >> (-up & 31)) & Num<T>::kMask) | Num<T>::kBase;
    }
    return r;
}

// Eight elements of x from place i, the first `valid` of them, as the operand that goes with codes_as_operand (fp32: its three parts).
template <int T> struct Operand { u32x4 part[Num<T>::kParts]; };
template <int T> __device__ __forceinline__ Operand<T> x_as_operand(const void* x, uint64_t i, int valid) {
    Operand<T> r;
    if (T == LC_F32) {
        float v[8];
        load_eight<T>(x, i, valid, v);
#pragma unroll
        for (int p = 0; p < Num<T>::kParts; ++p) {
#pragma unroll
            for (int j = 0; j < 4; ++j) r.part[p][j] = high_halves(bits_of(v[j]), bits_of(v[j + 4]));
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] -= float_of(bits_of(v[e]) & 0xffff0000u);     // what the part leaves: at most 16, then 8 bits
        }
    } else {
        u32x4 a;
        if (valid >= 8) a = load_any<u32x4>(static_cast<const uint16_t*>(x) + i);
        else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t lo = 2 * j < valid ? static_cast<const uint16_t*>(x)[i + 2 * j] : 0u;
                const uint32_t hi = 2 * j + 1 < valid ? static_cast<const uint16_t*>(x)[i + 2 * j + 1] : 0u;
                a[j] = lo | hi << 16;
            }
        }
        r.part[0] = u32x4{low_halves(a[0], a[2]), high_halves(a[0], a[2]), low_halves(a[1], a[3]), high_halves(a[1], a[3])};
    }
    return r;
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
// x gives, and 24 times a group's sum, or the sum before its scale, may be out of range where the result is not.
template <int T, int G>
__device__ __forceinline__ float one_by_formula(const Product& p, uint32_t i, uint32_t j) {
    float total = 0;
    for (uint32_t l = 0; l < p.k; ++l) {
        const uint32_t c = p.codes[j * p.codes_pitch + l / 2] >> (4 * (l % 2)) & 15u;
        total = fmaf(load_one<T>(p.x, i * p.ldx + l), (float)((int)c - 8) * of_bf16(p.scales[j * p.scales_pitch + l / G]), total);   // (q s is exact)
    }
    return total;
}

template <int T, int G>
__device__ __forceinline__ void finish(const Product& p, uint32_t i, uint32_t j, float v) {
    if (!(fabsf(v) < __builtin_inff())) v = one_by_formula<T, G>(p, i, j);
    if (p.bias) v += load_one<T>(p.bias, j);
    store_one<T>(p.y, i * p.ldy + j, v);
}

// Up to 16 rows of x by 16 rows of w a workgroup; its wavefronts take the width in turn, 128 elements (64 bytes of a row of codes)
// at a time, and their sums meet in LDS.  Columns of the matrix instruction are rows of w, so a lane's four results share a scale.
// Lane l loads 16 bytes of row l % 16, quarter l / 16 of the 64: with groups of 128 its four words go to four instructions as they
// are; with shorter groups they change places between the quarters first, so that every instruction stays inside a group.
template <int T, int G, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_w4_rows(Product p) {
    __shared__ float sums[WAVES][4][64];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = lane % 16, h = lane / 16;
    const uint32_t n0 = blockIdx.x * 16, m0 = blockIdx.y * 16;
    const uint32_t row = n0 + c < p.n ? n0 + c : p.n - 1;
    const uint8_t* codes = p.codes + row * p.codes_pitch;
    const uint16_t* scales = p.scales + row * p.scales_pitch;
    const bool has_x = m0 + c < p.m;
    const uint64_t x_row = (m0 + (has_x ? c : 0)) * p.ldx;
    const uint32_t steps = (p.k + 127) / 128;
    constexpr int PER = G / 32, GROUPS = 128 / G;
    f32x4 total = {0, 0, 0, 0};
    for (uint32_t step = wave; step < steps; step += WAVES) {
        u32x4 w = {0, 0, 0, 0};
        if (step * 64 + h * 16 < p.row_bytes) w = *reinterpret_cast<const u32x4*>(codes + step * 64 + h * 16);
        float s[GROUPS];
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) s[g] = step * GROUPS + g < p.groups ? of_bf16(scales[step * GROUPS + g]) : 0.0f;
        if (G < 128) {      // word (a, b) of quarter (h1, h0) holds the 8 codes from (h1 h0 a b): a and h1 change places, then b and h0
            const auto p02 = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
            const auto p13 = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
            const auto q01 = __builtin_amdgcn_permlane16_swap(p02[0], p13[0], false, false);
            const auto q23 = __builtin_amdgcn_permlane16_swap(p02[1], p13[1], false, false);
            w = u32x4{q01[0], q01[1], q23[0], q23[1]};
        }
        f32x4 acc;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t at = step * 128 + (G == 128 ? 32 * h + 8 * i : 32 * i + 8 * h);
            const int valid = has_x && at < p.k ? (int)(p.k - at < 8 ? p.k - at : 8) : 0;
            const Operand<T> x = x_as_operand<T>(p.x, x_row + at, valid);
            const u32x4 b = codes_as_operand<T>(w[i]);
            if (i % PER == 0) acc = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int q = Num<T>::kParts - 1; q >= 0; --q) {
                acc = Num<T>::mfma(x.part[q], u32x4{Num<T>::kMinus24, Num<T>::kMinus24, Num<T>::kMinus24, Num<T>::kMinus24}, acc);
                acc = Num<T>::mfma(x.part[q], b, acc);
            }
            if (i % PER == PER - 1) {
#pragma unroll
                for (int r = 0; r < 4; ++r) total[r] = fmaf(acc[r], s[i / PER], total[r]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) sums[wave][r][lane] = total[r];
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < 256; e += WAVES * 64) {
        const uint32_t i = m0 + 4 * (e / 64) + e % 64 / 16, j = n0 + e % 16;      // neighbours write neighbours
        const uint32_t from = (e / 64) * 16 + e % 16, r = e % 64 / 16;
        if (i >= p.m || j >= p.n) continue;
        float v = 0;
#pragma unroll
        for (int q = 0; q < WAVES; ++q) v += sums[q][r][from];
        finish<T, G>(p, i, j, v);
    }
}

template <int T>
__global__ __launch_bounds__(256) void k_w4_bias_only(Product p) {      // k = 0
    const uint64_t e = blockIdx.x * 256ull + threadIdx.x;
    if (e >= (uint64_t)p.m * p.n) return;
    const uint64_t i = e / p.n, j = e % p.n;
    store_one<T>(p.y, i * p.ldy + j, p.bias ? load_one<T>(p.bias, j) : 0.0f);
}

template <int T, int G>
void product(const Product& p, hipStream_t s) {
    const uint32_t steps = (p.k + 127) / 128;
    const dim3 grid((p.n + 15) / 16, (p.m + 15) / 16);
    if (steps <= 1) k_w4_rows<T, G, 1><<<grid, 64, 0, s>>>(p);
    else if (steps <= 4) k_w4_rows<T, G, 4><<<grid, 256, 0, s>>>(p);
    else k_w4_rows<T, G, 8><<<grid, 512, 0, s>>>(p);
}

// Whether a matrix in 4 bits is one the kernels can take.
bool bad(const lc_w4* q) {
    if (!q || (q->group != 32 && q->group != 64 && q->group != 128) || q->n > 0x7fffffffull || q->k > 0x7fffffffull) return true;
    if (q->n == 0 || q->k == 0) return false;
    return !q->codes || !q->scales || off(q->codes, 16) || off(q->scales, 2) || q->codes_pitch % 16 || q->codes_pitch < lc_w4_row_bytes(q->k) ||
           q->scales_pitch < (q->k + q->group - 1) / q->group || q->codes_pitch > (1ull << 40) || q->scales_pitch > (1ull << 40);
}

int launched() { return hipGetLastError() == hipSuccess ? LC_OK : LC_ERR_HIP; }

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
#define CALL(T, G) dequantize<T, G / 8>(q, w, ldw, s)
    LC_BY_TYPE(CALL, dtype, q);
#undef CALL
    return launched();
}

int lc_w4_matmul(const void* x, uint64_t ldx, uint64_t m, const lc_w4* w4, const void* bias, void* y, uint64_t ldy, int dtype, void* stream) {
    if (!served_type(dtype) || bad(w4) || m > (1u << 19)) return LC_ERR_BADARG;
    if (m == 0 || w4->n == 0) return LC_OK;
    const uintptr_t size = size_of(dtype);
    if (!y || off(y, size) || ldy < w4->n || ldy > (1ull << 40) || (bias && off(bias, size))) return LC_ERR_BADARG;
    if (w4->k && (!x || off(x, size) || ldx < w4->k || ldx > (1ull << 40))) return LC_ERR_BADARG;
    const lc_w4 q = *w4;
    const Product p = {x, ldx, static_cast<const uint8_t*>(q.codes), q.codes_pitch, static_cast<const uint16_t*>(q.scales), q.scales_pitch, bias, y, ldy,
                       (uint32_t)m, (uint32_t)q.n, (uint32_t)q.k, (uint32_t)lc_w4_row_bytes(q.k), (uint32_t)((q.k + q.group - 1) / q.group)};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (q.k == 0) {
        const uint64_t blocks = ((uint64_t)p.m * p.n + 255) / 256;
        if (blocks > 0x7fffffffull) return LC_ERR_BADARG;
        if (dtype == LC_F32) k_w4_bias_only<LC_F32><<<(uint32_t)blocks, 256, 0, s>>>(p);
        else if (dtype == LC_BF16) k_w4_bias_only<LC_BF16><<<(uint32_t)blocks, 256, 0, s>>>(p);
        else k_w4_bias_only<LC_F16><<<(uint32_t)blocks, 256, 0, s>>>(p);
        return launched();
    }
#define CALL(T, G) product<T, G>(p, s)
    LC_BY_TYPE(CALL, dtype, q);
#undef CALL
    return launched();
}

}  // extern "C"
