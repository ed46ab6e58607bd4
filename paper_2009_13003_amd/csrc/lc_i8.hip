// Matrices in 8 bits with a scale a row: quantising, reading back, and the products of two of them (include/lc_serve.h).
#include "lc_serve.h"

#include <algorithm>
#include <type_traits>

namespace lc {
namespace serve {
namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) int i32x16;

// ---------------------------------------------------------------- quantising and reading back
// A row's scale and its reciprocal by its largest magnitude, as the bits of a number: NaN above infinity above the rest.
__device__ __forceinline__ float scale_of(uint32_t most, float& inv) {
    const float s = float_of(most) * (1.0f / 127.0f);
    inv = 0.0f;
    if (most >= 0x7f800000u) return __builtin_nanf("");
    if (s < kSmallest) return 0.0f;
    inv = 1.0f / s;
    return s;
}
__device__ __forceinline__ uint32_t largest_of(const float x[8], uint32_t most) {
#pragma unroll
    for (int e = 0; e < 8; ++e) { const uint32_t a = bits_of(x[e]) & 0x7fffffffu; most = a > most ? a : most; }
    return most;
}
__device__ __forceinline__ uint32_t largest_of_wave(uint32_t most) {
    most = max_of_lanes<32>(most);
    const uint32_t o = (uint32_t)__shfl_xor((int)most, 32);
    return o > most ? o : most;
}
__device__ __forceinline__ u32x2 codes_of(const float x[8], float inv) {
    u32x2 q = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e / 4] |= (rounded(fminf(fmaxf(inv == 0.0f ? 0.0f : x[e] * inv, -127.0f), 127.0f), 0.0f) & 255u) << (8 * (e % 4));
    return q;
}

// Eights of a row's elements from `first` on, `step` apart, zeros behind its end at k: all whole ones are under way before the first is looked at (in a branch each, every one would be
// waited for), the one that the row ends in by itself.
template <int T, int R>
__device__ __forceinline__ void load_eights(const void* x, uint64_t row, uint32_t first, uint32_t step, uint32_t k, float v[R][8]) {
    const uint32_t whole = k & ~7u;
    f32x4 raw[R][T == LC_F32 ? 2 : 1];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < (T == LC_F32 ? 2 : 1); ++i) raw[r][i] = f32x4{0, 0, 0, 0};
    if (whole)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint64_t at = row + (first + r * step < whole ? first + r * step : 0);
            if (T == LC_F32) {
                raw[r][0] = load_once<f32x4>(static_cast<const float*>(x) + at);
                raw[r][T == LC_F32 ? 1 : 0] = load_once<f32x4>(static_cast<const float*>(x) + at + 4);
            } else raw[r][0] = load_once<f32x4>(static_cast<const uint16_t*>(x) + at);
        }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t at = first + r * step;
        const bool in = at < whole;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t u = bits_of(raw[r][0][e / 2 % 4]);
            const float f = T == LC_F32 ? raw[r][T == LC_F32 ? e / 4 : 0][e % 4] : T == LC_BF16 ? float_of(e % 2 ? u & 0xffff0000u : u << 16) : of_f16(e % 2 ? u >> 16 : u & 0xffffu);
            v[r][e] = in ? f : 0.0f;
        }
        if (!in && at < k) load_eight<T>(x, row + at, (int)(k - at), v[r]);
    }
}

// A row to a workgroup, or of short rows to a wavefront: 8 elements a lane at a time, kept in registers between the search for the largest and the rounding
// (rows too long for that are read again).  s = max |w| / 127, q = rint(w (1 / s)).  Bound by memory: 2048 rows of 11008 in bf16 12.5 us, 5.4 TB/s of what is read and
// written, a copy's rate.
template <int T, int WAVES, int R>
__global__ __launch_bounds__(256) void k_i8_quantize(const void* w, uint64_t ldw, uint8_t* codes, uint64_t pitch, float* scales, uint32_t rows, uint32_t k) {
    __shared__ uint32_t tops[4];
    constexpr uint32_t LANES = WAVES * 64;
    const uint32_t row = WAVES == 4 ? blockIdx.x : blockIdx.x * 4 + threadIdx.x / 64, lane = WAVES == 4 ? threadIdx.x : threadIdx.x % 64;
    if (row >= rows) return;
    float v[R][8];
    uint32_t most = 0;
    auto load = [&](uint32_t at, float x[8]) { load_eight<T>(w, row * ldw + at, at < k ? (int)(k - at < 8 ? k - at : 8) : 0, x); };
    load_eights<T, R>(w, row * ldw, lane * 8, LANES * 8, k, v);
#pragma unroll
    for (int r = 0; r < R; ++r) most = largest_of(v[r], most);
    for (uint32_t at = (R * LANES + lane) * 8; at < k; at += LANES * 8) {
        float x[8];
        load(at, x);
        most = largest_of(x, most);
    }
    most = largest_of_wave(most);
    if (WAVES == 4) {
        if (lane % 64 == 0) tops[lane / 64] = most;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) most = tops[i] > most ? tops[i] : most;
    }
    float inv;
    const float s = scale_of(most, inv);
    const uint32_t end = (k + 15) & ~15u;
    auto store = [&](uint32_t at, const float x[8]) {
        if (at < end) *reinterpret_cast<u32x2*>(codes + row * pitch + at) = codes_of(x, inv);
    };
#pragma unroll
    for (int r = 0; r < R; ++r) store((r * LANES + lane) * 8, v[r]);
    for (uint32_t at = (R * LANES + lane) * 8; at < end; at += LANES * 8) {
        float x[8];
        load(at, x);
        store(at, x);
    }
    if (lane == 0) scales[row] = s;
}

// A lane writes 16 bytes.  Bound by memory: 11008x4096 to fp32 32 us, 7.0 TB/s of what is read and written, to bf16 and fp16 20.5, 6.6 TB/s.
template <int T>
__global__ __launch_bounds__(256) void k_i8_dequantize(const uint8_t* codes, uint64_t pitch, const float* scales, void* w, uint64_t ldw, uint32_t lanes, uint32_t k,
                                                       FastDiv by_row) {
    constexpr int N = kAtOnce<T>;
    const uint32_t lane = blockIdx.x * 256u + threadIdx.x;
    if (lane >= lanes) return;
    const uint32_t row = by_row(lane), at = N * (lane - row * by_row.d);
    typedef typename std::conditional<N == 8, uint64_t, uint32_t>::type Word;
    const Word q = *reinterpret_cast<const Word*>(codes + row * pitch + at);
    const float s = scales[row];
    float v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
        v[e] = (float)(int8_t)(q >> (8 * e)) * s;
        if (T == LC_F16) asm("" : "+v"(v[e]));              // (else product and conversion become one instruction, with one rounding for the two)
    }
    store_some<T>(w, row * ldw + at, (int)(k - at < N ? k - at : N), v);
}

// ---------------------------------------------------------------- the product
struct Product {
    const uint8_t *x, *w;
    const float *sx, *sw;
    const void* bias;
    void* y;
    uint64_t x_pitch, w_pitch, ldy;
    uint32_t m, n, k16;         // k16: bytes of a row, a multiple of 16
    int dtype;
};

__device__ __forceinline__ float bias_of(const Product& p, uint32_t j) {
    return !p.bias ? 0.0f : p.dtype == LC_F32 ? load_one<LC_F32>(p.bias, j) : p.dtype == LC_BF16 ? load_one<LC_BF16>(p.bias, j) : load_one<LC_F16>(p.bias, j);
}
__device__ __forceinline__ float result_of(const Product& p, int sum, float sx, float sw, uint32_t j) {
    float v = (float)sum * sx * sw;
    if (p.bias) v += bias_of(p, j);
    return v;
}
__device__ __forceinline__ void put(const Product& p, uint64_t at, float v) {
    if (p.dtype == LC_F32) store_one<LC_F32>(p.y, at, v);
    else if (p.dtype == LC_BF16) store_one<LC_BF16>(p.y, at, v);
    else store_one<LC_F16>(p.y, at, v);
}

// D = A B^T + C in whole numbers, 16 x 16 x 64: lane l gives row l % 16 of A and of B, 16 bytes of the inner dimension per quarter (the same ones for both), and
// receives column l % 16, rows 4 (l / 16) + 0..3.  And 32 x 32 x 32: row l % 32, 16 bytes per half; column l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4.
__device__ __forceinline__ i32x4 mfma_16(u32x4 a, u32x4 b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}
__device__ __forceinline__ i32x16 mfma_32(u32x4 a, u32x4 b, i32x16 c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// Few rows: MT tiles of 16 rows of x by 16 rows of w a workgroup, whose wavefronts take steps of 128 bytes of the width in turn; a lane loads 32 bytes of a row, so
// that four lanes have a whole line, and their sums meet in LDS.  13 rows by 4096x11008 14 us, of which the bytes of w take 6.4 and a launch 2.3 (4 wavefronts 14.0, 16 18.2), 7 by
// 1000x2043 5.4; what is above that are waits: 256 workgroups, one a compute unit, that read all of x each.
template <int MT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_i8_rows(Product p) {
    __shared__ int sums[WAVES][MT * 16][17];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = lane % 16, h = lane / 16;
    const uint32_t n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MT;
    const uint32_t j = n0 + c < p.n ? n0 + c : p.n - 1;
    const uint8_t* w = p.w + j * p.w_pitch;
    const uint8_t* x[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) { const uint32_t i = m0 + 16 * t + c < p.m ? m0 + 16 * t + c : p.m - 1; x[t] = p.x + i * p.x_pitch; }
    i32x4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = i32x4{0, 0, 0, 0};
    constexpr int S = 4;
    for (uint32_t k0 = wave * 128; k0 < p.k16; k0 += S * WAVES * 128) {
        u32x4 a[S][2], b[S][MT][2];
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t at = k0 + s * WAVES * 128 + 32 * h + 16 * i;
                const bool in = at < p.k16;
                a[s][i] = load_once<u32x4>(w + (in ? at : 0));
#pragma unroll
                for (int t = 0; t < MT; ++t) { b[s][t][i] = *reinterpret_cast<const u32x4*>(x[t] + (in ? at : 0)); if (!in) b[s][t][i] = u32x4{0, 0, 0, 0}; }
            }
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int t = 0; t < MT; ++t) acc[t] = mfma_16(b[s][t][i], a[s][i], acc[t]);
    }
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[wave][16 * t + 4 * h + r][c] = acc[t][r];
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < MT * 256; e += WAVES * 64) {
        const uint32_t r = e / 16, i = m0 + r, col = n0 + e % 16;
        if (i >= p.m || col >= p.n) continue;
        int sum = 0;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) sum += sums[v][r][e % 16];
        put(p, i * p.ldy + col, result_of(p, sum, p.sx[i], p.sw[col], col));
    }
}

// One row of x as it comes: every workgroup works out its codes for itself, into LDS, while its first loads of w are under way.  By 11008x4096 10 us (in two launches 12.4), by
// 4096x4096 5.5, by 4096x11008 with three eights a lane 12.6 (read one after the other 14.4); at the rate of a bare read w takes 6.4 and 2.4, a launch 2.3.  (Sixteen wavefronts for widths above 4096: no faster.)
constexpr uint32_t kFused = 32768;                          // codes of x at most
template <int T, int R>
__global__ __launch_bounds__(512, R == 1 ? 6 : 4) void k_i8_one_row(Product p, const void* x, uint32_t k) {
    constexpr uint32_t WAVES = 8, S = 4;
    extern __shared__ __attribute__((aligned(16))) uint8_t codes[];      // of x
    __shared__ uint32_t tops[WAVES];
    __shared__ int sums[WAVES][16];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = lane % 16, h = lane / 16;
    const uint32_t n0 = blockIdx.x * 16, j = n0 + c < p.n ? n0 + c : p.n - 1;
    const uint8_t* w = p.w + j * p.w_pitch;
    u32x4 a[S][2];
    auto load = [&](uint32_t k0) {
#pragma unroll
        for (uint32_t s = 0; s < S; ++s)
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i) {
                const uint32_t at = k0 + s * WAVES * 128 + 32 * h + 16 * i;
                a[s][i] = load_once<u32x4>(w + (at < p.k16 ? at : 0));
            }
    };
    load(wave * 128);
    float v[R][8];
    uint32_t most = 0;
    load_eights<T, R>(x, 0, threadIdx.x * 8, WAVES * 512, k, v);
#pragma unroll
    for (int r = 0; r < R; ++r) most = largest_of(v[r], most);
    for (uint32_t at = (R * WAVES * 64 + threadIdx.x) * 8; at < k; at += WAVES * 512) {
        float more[8];
        load_eight<T>(x, at, (int)(k - at < 8 ? k - at : 8), more);
        most = largest_of(more, most);
    }
    most = largest_of_wave(most);
    if (lane == 0) tops[wave] = most;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < WAVES; ++i) most = tops[i] > most ? tops[i] : most;
    float inv;
    const float sx = scale_of(most, inv);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t at = (r * WAVES * 64 + threadIdx.x) * 8;
        if (at < p.k16) *reinterpret_cast<u32x2*>(codes + at) = codes_of(v[r], inv);
    }
    for (uint32_t at = (R * WAVES * 64 + threadIdx.x) * 8; at < p.k16; at += WAVES * 512) {
        float more[8];
        load_eight<T>(x, at, at < k ? (int)(k - at < 8 ? k - at : 8) : 0, more);
        *reinterpret_cast<u32x2*>(codes + at) = codes_of(more, inv);
    }
    __syncthreads();
    i32x4 acc = {0, 0, 0, 0};                               // (of sixteen rows of x that are all this one)
    for (uint32_t k0 = wave * 128; k0 < p.k16; k0 += S * WAVES * 128) {
        if (k0 != wave * 128) load(k0);
#pragma unroll
        for (uint32_t s = 0; s < S; ++s)
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i) {
                const uint32_t at = k0 + s * WAVES * 128 + 32 * h + 16 * i;
                u32x4 b = *reinterpret_cast<const u32x4*>(codes + (at < p.k16 ? at : 0));
                if (at >= p.k16) b = u32x4{0, 0, 0, 0};
                acc = mfma_16(b, a[s][i], acc);
            }
    }
    if (h == 0) sums[wave][c] = acc[0];
    __syncthreads();
    const uint32_t col = n0 + threadIdx.x;
    if (threadIdx.x >= 16 || col >= p.n) return;
    int sum = 0;
#pragma unroll
    for (uint32_t i = 0; i < WAVES; ++i) sum += sums[i][threadIdx.x];
    put(p, col, result_of(p, sum, sx, p.sw[col], col));
}

// The same for 2 to 16 rows that are short: eights of their elements a lane, at most R of them, so that x is read once, and its largest by atomics in LDS.  2 rows by 4096x4096 6.5 us (in
// two launches 7.3), 8 by 1024x1024 5.8 (7.3), 16 by 4096x512 5.9 (6.5).  Beyond two eights a lane every workgroup has too much of x to do: 4 rows by 4096x4096 8.9 (7.9), 7 by 1000x2043 8.1 (7.4).
constexpr uint32_t kShort = 8192;                           // elements of all rows at most
template <int T, int R>
__global__ __launch_bounds__(512, 6) void k_i8_short_rows(Product p, const void* x, uint64_t ldx, uint32_t k, FastDiv by_row) {
    constexpr uint32_t WAVES = 8, S = 4;
    extern __shared__ __attribute__((aligned(16))) uint8_t codes[];      // of x, a row every k16 + 16 bytes
    __shared__ uint32_t tops[16];
    __shared__ int sums[WAVES][16][17];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = lane % 16, h = lane / 16, pitch = p.k16 + 16;
    const uint32_t n0 = blockIdx.x * 16, j = n0 + c < p.n ? n0 + c : p.n - 1;
    const uint8_t* w = p.w + j * p.w_pitch;
    u32x4 a[S][2];
    auto load = [&](uint32_t k0) {
#pragma unroll
        for (uint32_t s = 0; s < S; ++s)
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i) {
                const uint32_t at = k0 + s * WAVES * 128 + 32 * h + 16 * i;
                a[s][i] = load_once<u32x4>(w + (at < p.k16 ? at : 0));
            }
    };
    load(wave * 128);
    if (threadIdx.x < 16) tops[threadIdx.x] = 0;
    float v[R][8];
    uint32_t row[R], at[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t i = r * 512 + threadIdx.x;
        row[r] = by_row(i);
        at[r] = (i - row[r] * by_row.d) * 8;
        load_eight<T>(x, row[r] * ldx + at[r], row[r] < p.m && at[r] < k ? (int)(k - at[r] < 8 ? k - at[r] : 8) : 0, v[r]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t most = largest_of(v[r], 0), first = __builtin_amdgcn_readfirstlane(row[r]);
        if (__all(row[r] == first)) {
            const uint32_t all = largest_of_wave(most);
            if (lane == 0 && first < p.m) atomicMax(&tops[first], all);
        } else if (row[r] < p.m) atomicMax(&tops[row[r]], most);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (row[r] < p.m) {
            float inv;
            scale_of(tops[row[r]], inv);
            *reinterpret_cast<u32x2*>(codes + row[r] * pitch + at[r]) = codes_of(v[r], inv);
        }
    __syncthreads();
    i32x4 acc = {0, 0, 0, 0};
    const uint8_t* own = codes + (c < p.m ? c : 0) * pitch; // (rows that are not there give results that nothing takes)
    for (uint32_t k0 = wave * 128; k0 < p.k16; k0 += S * WAVES * 128) {
        if (k0 != wave * 128) load(k0);
#pragma unroll
        for (uint32_t s = 0; s < S; ++s)
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i) {
                const uint32_t place = k0 + s * WAVES * 128 + 32 * h + 16 * i;
                u32x4 b = *reinterpret_cast<const u32x4*>(own + (place < p.k16 ? place : 0));
                if (place >= p.k16) b = u32x4{0, 0, 0, 0};
                acc = mfma_16(b, a[s][i], acc);
            }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) sums[wave][4 * h + r][c] = acc[r];
    __syncthreads();
    const uint32_t i = threadIdx.x / 16, col = n0 + threadIdx.x % 16;
    if (i >= p.m || col >= p.n) return;
    int sum = 0;
#pragma unroll
    for (uint32_t v = 0; v < WAVES; ++v) sum += sums[v][i][threadIdx.x % 16];
    float inv;
    const float sx = scale_of(tops[i], inv);
    put(p, i * p.ldy + col, result_of(p, sum, sx, p.sw[col], col));
}

// 16 bytes of each lane's own place into LDS at `to` + 16 lane, without passing through registers.
__device__ __forceinline__ void load_to_lds(const void* from, void* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(uintptr_t)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// Four results of a row that follow each other, the first `valid` of them.
__device__ __forceinline__ void put_four(const Product& p, uint64_t at, f32x4 v, uint32_t valid) {
    if (valid >= 4) {
        typedef f32x4 __attribute__((aligned(2))) Four;
        typedef u32x2 __attribute__((aligned(2))) Halves;
        typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
        if (p.dtype == LC_F32) *reinterpret_cast<Four*>(static_cast<float*>(p.y) + at) = v;
        else if (p.dtype == LC_BF16) *reinterpret_cast<Halves*>(static_cast<uint16_t*>(p.y) + at) = u32x2{rounded_halves(v[0], v[1]), rounded_halves(v[2], v[3])};
        else *reinterpret_cast<Halves*>(static_cast<uint16_t*>(p.y) + at) = __builtin_bit_cast(u32x2, __builtin_convertvector(v, f16x4));
    } else
        for (uint32_t e = 0; e < valid; ++e) put(p, at + e, v[e]);
}

// N of the loads that go to LDS may still be under way.
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// Many rows: TM rows of x by TN rows of w a workgroup, WM x WN wavefronts, 128 bytes of the width at a time in LDS, in BUFFERS places that are filled in turn.  A load that
// goes to LDS brings eight rows of 128 bytes, each by eight lanes in its own order (turned about within a row, so that LDS has no bank conflicts, such loads cost: 2048x4096x11008
// 105 us for 96), and eight rows apart, so that the sixteen rows that LDS serves at once lie in eight such pieces, 16 bytes more than 1024 apart, and have all of
// its 256 bytes.  Operands are read a step of 32 bytes ahead of their products.  The workgroup meets once a tile, ahead of its last step, whose operands have been read by
// then: behind the meeting the tile's place is filled again.
// Rows of the matrix instruction's result are rows of w, so a lane has four results of a row of y that follow each other.
// 2048 rows by 4096x11008: 87 us, 2.1 PFLOP/s, the matrix unit 68% of its cycles.  Copies of the kernel that leave something out (and so work on whatever registers and LDS hold): products alone
// 61 us, with the reads of LDS 73, with the loads into it 72; loads alone 57, with the reads 58.  So the way of 48 KB a tile into LDS and the one out of it cost the products 12 to 15 us each.
template <int TM, int TN, int WM, int WN, int BUFFERS>
__global__ __launch_bounds__(WM * WN * 64) void k_i8_tiles(Product p) {
    constexpr int WAVES = WM * WN, MT = TM / WM / 32, NT = TN / WN / 32, PIECE = 1024 + 16, BYTES = (TM + TN) / 8 * PIECE, LOADS = (TM + TN) / 8 / WAVES;
    static_assert((TM + TN) % (8 * WAVES) == 0 && TM % 64 == 0 && TN % 64 == 0, "whole loads");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[BUFFERS][BYTES];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), c = lane % 32, h = lane / 32;
    // Workgroups go round the eight dies, each with an L2 of its own: those of one die get tiles that lie together, by bands of eight tiles of x.
    const uint32_t tiles_m = (p.m + TM - 1) / TM, tiles_n = (p.n + TN - 1) / TN, all = tiles_m * tiles_n, whole = all / 8;
    const uint32_t id = blockIdx.x < whole * 8 ? blockIdx.x % 8 * whole + blockIdx.x / 8 : blockIdx.x;
    const uint32_t band = id / (8 * tiles_n), high = tiles_m - band * 8 < 8 ? tiles_m - band * 8 : 8, in_band = id - band * 8 * tiles_n;
    const uint32_t m0 = (band * 8 + in_band % high) * TM, n0 = in_band / high * TN;
    // Where each lane loads from: a scalar place and 32 bits behind it, held to the row's end (what lies behind the width is left out of the products).
    const uint8_t *x0 = p.x + m0 * p.x_pitch, *w0 = p.w + n0 * p.w_pitch;
    uint32_t from[LOADS];
    const uint32_t end = p.k16 - 16;
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
        const uint32_t piece = wave * LOADS + l, row = piece / 8 * 64 + lane / 8 * 8 + piece % 8;      // of x, and behind them of w
        const uint32_t i = row < TM ? (m0 + row < p.m ? row : p.m - 1 - m0) : (n0 + row - TM < p.n ? row - TM : p.n - 1 - n0);
        from[l] = i * (uint32_t)(row < TM ? p.x_pitch : p.w_pitch);
    }
    auto ask = [&](uint32_t tile, int l, uint32_t buffer) {
        const uint32_t piece = wave * LOADS + l, at = tile * 128 + lane % 8 * 16;
        load_to_lds((piece < TM / 8 ? x0 : w0) + (uint64_t)(from[l] + (at < end ? at : end)), &lds[buffer][piece * PIECE]);
    };
    const uint32_t wm = wave % WM * (TM / WM), wn = TM + wave / WM * (TN / WN);
    static_assert(TN <= WAVES * 64, "a lane a column");
    u32x4 a[2][NT], b[2][MT];                               // of w and of x
    auto operand_at = [&](uint32_t buffer, uint32_t u, uint32_t row) {      // unit u of this lane's of the 32 rows from `row` on
        return *reinterpret_cast<const u32x4*>(&lds[buffer][c % 8 * PIECE + c / 8 * 128 + row / 64 * 8 * PIECE + row % 64 / 8 * 128 + u * 16]);
    };
    auto read = [&](uint32_t buffer, int s, int i) {        // the i-th operand of step s
        (i < NT ? a[s % 2][i < NT ? i : 0] : b[s % 2][i < NT ? 0 : i - NT]) = operand_at(buffer, 2 * s + h, i < NT ? wn + 32 * i : wm + 32 * (i - NT));
    };
    i32x16 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
#pragma unroll
    for (int t = 0; t < BUFFERS; ++t)
#pragma unroll
        for (int l = 0; l < (t == BUFFERS - 1 ? LOADS / 4 : LOADS); ++l) ask(t, l, t);
    wait_loads<(BUFFERS - 2) * LOADS + LOADS / 4>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");                          // (the meeting by itself lets the compiler read before it)
#pragma unroll
    for (int i = 0; i < NT + MT; ++i) read(0, 0, i);
    uint32_t buffer = 0, last = BUFFERS - 1;                // the tile's place, and that of the one before
    const uint32_t tiles = p.k16 / 128, rest = p.k16 % 128 / 16;       // whole ones, and 16 bytes behind them
    for (uint32_t t = 0; t < tiles; ++t) {
        const uint32_t next = buffer + 1 == BUFFERS ? 0 : buffer + 1;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (s == 3) {
                // the next tile is there, and everyone has read this one
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((BUFFERS - 2) * LOADS) : "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            }
#pragma unroll
            for (int x = 0; x < MT * NT; ++x) {
                const int i = x / NT, j = x % NT;
                acc[i][j] = mfma_32(a[s % 2][j], b[s % 2][i], acc[i][j]);
#pragma unroll
                for (int y = x * (NT + MT) / (MT * NT); y < (x + 1) * (NT + MT) / (MT * NT); ++y) read(s == 3 ? next : buffer, (s + 1) % 4, y);
                // a quarter of what is asked for beside each step
                const int first = (s + 1) % 4 * LOADS / 4, loads = ((s + 1) % 4 + 1) * LOADS / 4 - first;
#pragma unroll
                for (int y = x * loads / (MT * NT); y < (x + 1) * loads / (MT * NT); ++y) ask(s == 3 ? t + BUFFERS : t - 1 + BUFFERS, first + y, s == 3 ? buffer : last);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        last = buffer;
        buffer = next;
    }
    const uint32_t own = n0 + threadIdx.x < p.n ? n0 + threadIdx.x : p.n - 1;
    const float column = p.sw[own], shift = bias_of(p, own);
    float sx[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) { const uint32_t row = m0 + wm + 32 * i + c; sx[i] = p.sx[row < p.m ? row : p.m - 1]; }
    wait_loads<0>();
    if (rest) {
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        for (uint32_t s = 0; 2 * s < rest; ++s) {
            const bool in = 2 * s + h < rest;
#pragma unroll
            for (int j = 0; j < NT; ++j) a[0][j] = operand_at(buffer, 2 * s + h, wn + 32 * j);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                b[0][i] = operand_at(buffer, 2 * s + h, wm + 32 * i);
                if (!in) b[0][i] = u32x4{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = mfma_32(a[0][j], b[0][i], acc[i][j]);
            }
        }
    }
    // Scales of w's rows and the bias by way of LDS (303 rows by 28891x40 23 us for 40 with loads beside the stores), in an array that there is: a second one has the
    // compiler wait for all loads in every tile (330 us for 113).
    float* columns = reinterpret_cast<float*>(&lds[0][0]);
    __syncthreads();
    if (threadIdx.x < TN) { columns[threadIdx.x] = column; columns[TN + threadIdx.x] = shift; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const uint32_t row = m0 + wm + 32 * i + c;
        if (row >= p.m) continue;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint32_t at = wn - TM + 32 * j + 8 * g + 4 * h, col = n0 + at;
                if (col >= p.n) continue;
                const uint32_t valid = p.n - col < 4 ? p.n - col : 4;
                const f32x4 sw = *reinterpret_cast<const f32x4*>(columns + at);
                f32x4 v;
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) v[e] = (float)acc[i][j][4 * g + e] * sx[i] * sw[e];
                if (p.bias) {
                    const f32x4 more = *reinterpret_cast<const f32x4*>(columns + TN + at);
#pragma unroll
                    for (uint32_t e = 0; e < 4; ++e) v[e] += more[e];
                }
                put_four(p, row * p.ldy + col, v, valid);
            }
    }
}

bool bad(const lc_i8* q) {
    if (!q || q->n > 0x7fffffffull || q->k > LC_I8_MAX_K) return true;
    if (q->n == 0 || q->k == 0) return q->n != 0 && (!q->scales || off(q->scales, 4));
    return !q->codes || !q->scales || off(q->codes, 16) || off(q->scales, 4) || q->pitch % 16 || q->pitch < q->k || q->pitch > (1ull << 40);
}

template <int T, int WAVES, int R>
void quantize_of(const void* w, uint64_t ldw, const lc_i8& q, hipStream_t s) {
    const uint64_t step = 1ull << 23;                       // rows: a launch's lanes are counted in 32 bits
    for (uint64_t r = 0; r < q.n; r += step) {
        const uint32_t rows = (uint32_t)(q.n - r < step ? q.n - r : step);
        k_i8_quantize<T, WAVES, R><<<WAVES == 4 ? rows : (rows + 3) / 4, 256, 0, s>>>(static_cast<const uint8_t*>(w) + r * ldw * (T == LC_F32 ? 4 : 2), ldw,
            static_cast<uint8_t*>(q.codes) + r * q.pitch, q.pitch, q.scales + r, rows, (uint32_t)q.k);
    }
}
template <int T>
void quantize(const void* w, uint64_t ldw, const lc_i8& q, hipStream_t s) {
    // A wavefront a row where there are rows enough to fill the chip with them.
    if (q.n >= 2048 && q.k <= 512) quantize_of<T, 1, 1>(w, ldw, q, s);
    else if (q.n >= 2048 && q.k <= 2048) quantize_of<T, 1, 4>(w, ldw, q, s);
    else if (q.k <= 2048) quantize_of<T, 4, 1>(w, ldw, q, s);
    else if (q.k <= 4096) quantize_of<T, 4, 2>(w, ldw, q, s);
    else if (q.k <= 8192) quantize_of<T, 4, 4>(w, ldw, q, s);
    else if (q.k <= 12288) quantize_of<T, 4, 6>(w, ldw, q, s);
    else quantize_of<T, 4, 8>(w, ldw, q, s);
}
template <int T>
void dequantize(const lc_i8& q, void* w, uint64_t ldw, hipStream_t s) {
    const uint32_t lanes = (uint32_t)((q.k + kAtOnce<T> - 1) / kAtOnce<T>);
    const uint64_t step = (1ull << 30) / lanes;
    for (uint64_t r = 0; r < q.n; r += step) {
        const uint32_t rows = (uint32_t)(q.n - r < step ? q.n - r : step);
        k_i8_dequantize<T><<<(uint32_t)(((uint64_t)rows * lanes + 255) / 256), 256, 0, s>>>(static_cast<const uint8_t*>(q.codes) + r * q.pitch, q.pitch, q.scales + r,
            static_cast<uint8_t*>(w) + r * ldw * (T == LC_F32 ? 4 : 2), ldw, rows * lanes, (uint32_t)q.k, FastDiv(lanes));
    }
}

template <int TM, int TN, int BUFFERS>
void tiles(const Product& p, hipStream_t s) {
    k_i8_tiles<TM, TN, 2, 2, BUFFERS><<<(p.m + TM - 1) / TM * ((p.n + TN - 1) / TN), 256, 0, s>>>(p);
}
void multiply_piece(const Product& p, bool few, hipStream_t s) {
    if (p.m <= 16 || few) { k_i8_rows<1, 8><<<dim3((p.n + 15) / 16, (p.m + 15) / 16), 512, 0, s>>>(p); return; }
    // What takes the least time, by how many workgroups the chip has at once and what such a round takes: some time for its start and its results, and some for 4096 of the width, in
    // tenths of a us as measured (2048 rows by 4096, with the launch's 2.3 us, at widths of 64 / 1024 / 4096: 64 x 64 14.3 / 23.5 / 58, 128 x 64 13.4 / 20.4 / 49, 128 x 128 15.5 / 22.2 / 47,
    // 128 x 256 13.6 / 19.7 / 39; 256 rows 3.9 / 5.3 / 9.9, 4.9 / 6.7 / 13.2, 6.9 / 9.2 / 17.2, 10.4 / 14 / 26.9; 24 rows by 4096x4096 with
    // two tiles of rows 7.4, by 8192x4096 13 and 64 x 64 9.8; widths above 4096 are more than one step of those, 100 rows by 797x9538 22.5 and 64 x 64 16.5).
    auto takes = [&](uint64_t tm, uint64_t tn, uint64_t chip, uint64_t start, uint64_t width) {
        return (((p.m + tm - 1) / tm) * ((p.n + tn - 1) / tn) + chip - 1) / chip * (start * 4096 + width * p.k16);
    };
    const bool a_few = (uint64_t)((p.m + 63) / 64) * ((p.n + 63) / 64) <= 256, b_few = (uint64_t)((p.m + 127) / 128) * ((p.n + 63) / 64) <= 256;
    const uint64_t rows = p.k16 <= 4096 ? takes(32, 16, 256, 15, 39) : ~0ull, a = a_few ? takes(64, 64, 256, 15, 60) : takes(64, 64, 512, 29, 113),
                   b = b_few ? takes(128, 64, 256, 30, 106) : takes(128, 64, 512, 46, 190), c = takes(128, 128, 256, 53, 174), d = takes(128, 256, 256, 110, 260);
    const uint64_t least = std::min({rows, a, b, c, d});
    if (d == least) tiles<128, 256, 3>(p, s);
    else if (c == least) tiles<128, 128, 4>(p, s);
    else if (b == least) tiles<128, 64, 3>(p, s);
    else if (a == least) tiles<64, 64, 4>(p, s);
    else k_i8_rows<2, 8><<<dim3((p.n + 15) / 16, (p.m + 31) / 32), 512, 0, s>>>(p);
}
// By pieces of w's rows of which each makes a launch of fewer than 2^32 threads.
void multiply(const Product& p, hipStream_t s) {
    // (no width, or rows so far apart that 32 bits do not count the bytes of a tile: what is right for any)
    const bool few = p.k16 == 0 || p.x_pitch > (1u << 23) || p.w_pitch > (1u << 23);
    const uint64_t step = p.m <= 64 || few ? (1ull << 22) / ((p.m + 15) / 16) * 16 : (1ull << 22) / ((p.m + 63) / 64) * 64;
    for (uint64_t j = 0; j < p.n; j += step) {
        Product q = p;
        q.n = (uint32_t)(p.n - j < step ? p.n - j : step);
        q.w += j * p.w_pitch;
        q.sw += j;
        if (q.bias) q.bias = static_cast<const uint8_t*>(p.bias) + j * size_of(p.dtype);
        q.y = static_cast<uint8_t*>(p.y) + j * size_of(p.dtype);
        multiply_piece(q, few, s);
    }
}

template <int T>
void one_row(const Product& p, const void* x, uint32_t k, hipStream_t s) {
    const uint32_t blocks = (p.n + 15) / 16;
    if (k <= 4096) k_i8_one_row<T, 1><<<blocks, 512, p.k16, s>>>(p, x, k);
    else k_i8_one_row<T, 3><<<blocks, 512, p.k16, s>>>(p, x, k);
}
template <int T>
void short_rows(const Product& p, const void* x, uint64_t ldx, uint32_t k, hipStream_t s) {
    const uint32_t blocks = (p.n + 15) / 16, lds = p.m * (p.k16 + 16);
    const FastDiv by_row(p.k16 / 8);
    if (p.m * p.k16 <= kShort / 2) k_i8_short_rows<T, 1><<<blocks, 512, lds, s>>>(p, x, ldx, k, by_row);
    else k_i8_short_rows<T, 2><<<blocks, 512, lds, s>>>(p, x, ldx, k, by_row);
}

bool bad_result(const lc_i8* w8, uint64_t m, const void* bias, const void* y, uint64_t ldy, int dtype) {
    return !y || off(y, size_of(dtype)) || off(bias, size_of(dtype)) || ldy > (1ull << 40) || (m > 1 && ldy < w8->n);
}
constexpr uint64_t kMostRows = 1ull << 19;

}  // namespace
}  // namespace serve
}  // namespace lc

using namespace lc::serve;

extern "C" {

int lc_i8_quantize(const void* w, uint64_t ldw, int dtype, const lc_i8* w8, void* stream) {
    if (!served_type(dtype) || bad(w8)) return LC_ERR_BADARG;
    if (w8->n == 0) return LC_OK;
    if ((w8->k && (!w || off(w, size_of(dtype)))) || (w8->n > 1 && ldw < w8->k) || ldw > (1ull << 40)) return LC_ERR_BADARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == LC_F32) quantize<LC_F32>(w, ldw, *w8, s);
    else if (dtype == LC_BF16) quantize<LC_BF16>(w, ldw, *w8, s);
    else quantize<LC_F16>(w, ldw, *w8, s);
    return launched();
}

int lc_i8_dequantize(const lc_i8* w8, void* w, uint64_t ldw, int dtype, void* stream) {
    if (!served_type(dtype) || bad(w8)) return LC_ERR_BADARG;
    if (w8->n == 0 || w8->k == 0) return LC_OK;
    if (!w || off(w, size_of(dtype)) || (w8->n > 1 && ldw < w8->k) || ldw > (1ull << 40)) return LC_ERR_BADARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == LC_F32) dequantize<LC_F32>(*w8, w, ldw, s);
    else if (dtype == LC_BF16) dequantize<LC_BF16>(*w8, w, ldw, s);
    else dequantize<LC_F16>(*w8, w, ldw, s);
    return launched();
}

int lc_i8_matmul(const lc_i8* x8, const lc_i8* w8, const void* bias, void* y, uint64_t ldy, int dtype, void* stream) {
    if (!served_type(dtype) || bad(x8) || bad(w8) || x8->k != w8->k || x8->n > kMostRows) return LC_ERR_BADARG;
    if (x8->n == 0 || w8->n == 0) return LC_OK;
    if (bad_result(w8, x8->n, bias, y, ldy, dtype)) return LC_ERR_BADARG;
    const Product p = {static_cast<const uint8_t*>(x8->codes), static_cast<const uint8_t*>(w8->codes), x8->scales, w8->scales, bias, y, x8->pitch, w8->pitch, ldy,
                       (uint32_t)x8->n, (uint32_t)w8->n, (uint32_t)((w8->k + 15) / 16 * 16), dtype};
    multiply(p, static_cast<hipStream_t>(stream));
    return launched();
}

size_t lc_i8_workspace_bytes(uint64_t m, uint64_t k) {
    if (m > kMostRows || k > LC_I8_MAX_K) return 0;
    return (size_t)((m * ((k + 15) / 16 * 16) + 255) / 256 * 256 + (m * 4 + 255) / 256 * 256 + 256);
}

int lc_i8_linear(const void* x, uint64_t ldx, uint64_t m, const lc_i8* w8, const void* bias, void* y, uint64_t ldy, int dtype, void* ws, size_t ws_bytes,
                 void* stream) {
    if (!served_type(dtype) || bad(w8) || m > kMostRows) return LC_ERR_BADARG;
    if (m == 0 || w8->n == 0) return LC_OK;
    if (bad_result(w8, m, bias, y, ldy, dtype) || (w8->k && (!x || off(x, size_of(dtype)))) || (m > 1 && ldx < w8->k) || ldx > (1ull << 40)) return LC_ERR_BADARG;
    if (!ws || off(ws, 256) || ws_bytes < lc_i8_workspace_bytes(m, w8->k)) return LC_ERR_WORKSPACE;
    const uint64_t row = (w8->k + 15) / 16 * 16;
    if (w8->k && m == 1 && row <= kFused && w8->n <= (1u << 26)) {
        const Product p = {nullptr, static_cast<const uint8_t*>(w8->codes), nullptr, w8->scales, bias, y, 0, w8->pitch, ldy, (uint32_t)m, (uint32_t)w8->n, (uint32_t)row, dtype};
        hipStream_t s = static_cast<hipStream_t>(stream);
        if (dtype == LC_F32) one_row<LC_F32>(p, x, (uint32_t)w8->k, s);
        else if (dtype == LC_BF16) one_row<LC_BF16>(p, x, (uint32_t)w8->k, s);
        else one_row<LC_F16>(p, x, (uint32_t)w8->k, s);
        return launched();
    }
    if (w8->k && m > 1 && m <= 16 && m * row <= kShort && w8->n <= (1u << 26)) {
        const Product p = {nullptr, static_cast<const uint8_t*>(w8->codes), nullptr, w8->scales, bias, y, 0, w8->pitch, ldy, (uint32_t)m, (uint32_t)w8->n, (uint32_t)row, dtype};
        hipStream_t s = static_cast<hipStream_t>(stream);
        if (dtype == LC_F32) short_rows<LC_F32>(p, x, ldx, (uint32_t)w8->k, s);
        else if (dtype == LC_BF16) short_rows<LC_BF16>(p, x, ldx, (uint32_t)w8->k, s);
        else short_rows<LC_F16>(p, x, ldx, (uint32_t)w8->k, s);
        return launched();
    }
    const lc_i8 x8 = {ws, reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + (m * row + 255) / 256 * 256), m, w8->k, row};
    const int st = lc_i8_quantize(x, ldx, dtype, &x8, stream);
    return st != LC_OK ? st : lc_i8_matmul(&x8, w8, bias, y, ldy, dtype, stream);
}

}  // extern "C"
