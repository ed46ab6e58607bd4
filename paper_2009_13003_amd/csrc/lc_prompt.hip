// Attention of many new tokens a sequence over the paged cache in 8 or 4 bits (include/lc_serve.h).
#include "lc_cache.h"

namespace lc {
namespace serve {
namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;

// The rows that share a head of the cache are a sequence's new tokens times the queries to a head.  A workgroup takes 128 of them, a wavefront 32, and walks over the
// tokens 64 at a time.  Codes are converted once for all of its rows, on their way into LDS (K as it lies, V with tokens and elements changed about), and from there:
//   S^T = K Q^T   32 tokens by 32 rows by 16 elements an instruction: lane l gets row l % 32, tokens 8 (i / 4) + 4 (l / 32) + i % 4
//   O^T += V^T P^T   the same lane's probabilities are its part of the second operand as they stand, with the tokens of each 16 in the order 0-3, 8-11, 4-7, 12-15,
//                    in which V^T is kept
// so that the running maximum and the sum are one number a lane.  Codes are whole numbers in 16 bits, exactly; scales of keys multiply the scores, scales of values the
// probabilities, whose product is rounded: in fp32 to three bf16 parts, else to fp16, measured from a power of two near the largest scale that a row of the workgroup has seen so far, so that products
// down to 2^-24 of the largest have all of its 11 bits (in bf16 their rounding would be as large as the result's own: errors 1.4 times as large).
// 2048 of 10000 tokens of 32 / 8 heads of 128 in 8 bits, bf16: 340 us (345 to 355 on some cards), 850 to 885 TFLOP/s, where a large library product's rate would give 211.  Per 32 rows by 64
// tokens 32 matrix instructions stand beside 280 of the vector unit: 63 for conversions, 32 exponentials, 128 for scores, sums, scales and roundings.  The matrix unit
// has 44% of the cycles, vector instructions 56%, LDS 46%, and the clock stands at 1.9 GHz: fewer vector instructions (scales in the values, 48 fewer, sums by the
// matrix unit) and wavefronts that take turns on a SIMD changed nothing or cost 2%.  9 sequences of 57 to 517 new tokens of up to 3001, 32 heads, 4 bits, fp16: 100 us, of which the
// join 11; 25 blocks of rows a head of which a third are partly filled, and codes converted for 128 rows at most.  fp32, three parts each: 2 of 333 of 1500 tokens 23 and 9 us.
constexpr int kTile = 64;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNear = 64;                                // of the unit that has 2^10 of the largest: while no scale in a tile is below that, rows need not look for their own (100 of 100 tokens 8.7 us, 9.0 if all do)
constexpr int kLowest = 90;                                // 16-bit types: how far below its largest score, in powers of two, a row measures at most (2^30 of them have a sum)
constexpr uint32_t kMostParts = 32, kLeastTiles = 4;       // of a sequence's tokens, and tiles that a part has at least

struct Prompt {
    Cache c;
    const void* q; uint64_t ld_q;
    const int32_t* starts;
    const int32_t* table; uint64_t ld_table; uint64_t table_pages;
    const int32_t* lens;
    void* out; uint64_t ld_out;
    uint32_t* deal;             // of more than 64 sequences: how they are dealt (k_kv_prompt_deal); else NULL
    float* stats;               // the maximum and the sum of each [place of a part][row]
    float* part;                // [place of a part][row][dim]
    float scale;                // times log2(e)
    uint32_t tokens, batch, heads, group;
    uint32_t first_unit;        // of this launch
    uint32_t most_parts, share; // parts of a sequence at most; workgroups that are on the chip at once, for one head
    int32_t pages;
    FastDiv by_group;
};

// How many 16-bit parts an element of q, and a probability, are given; whether keys and queries, and probabilities and values, are fp16 (else bf16); and by how much, in powers
// of two, a score may pass what probabilities are measured from (in fp16 they have room for 2^16, of which 2^11 are the scales').
template <int T> struct Kind;
template <> struct Kind<LC_F32> { static constexpr int kParts = 3; static constexpr bool kHalf = false, kHalfValues = false; static constexpr float kFar = 8; };
template <> struct Kind<LC_BF16> { static constexpr int kParts = 1; static constexpr bool kHalf = false, kHalfValues = true; static constexpr float kFar = 4; };
template <> struct Kind<LC_F16> { static constexpr int kParts = 1; static constexpr bool kHalf = true, kHalfValues = true; static constexpr float kFar = 4; };

template <bool HALF> __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    if (HALF) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// a below b, rounded to nearest even.
template <bool HALF> __device__ __forceinline__ uint32_t pair_of(float a, float b) {
    if (!HALF) return rounded_halves(a, b);
    typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));
}
// The other half's number of the same column.
__device__ __forceinline__ float other_half(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(bits_of(v), bits_of(v), false, false);
    return threadIdx.x % 64 < 32 ? float_of(a[1]) : float_of(a[0]);
}

__device__ __forceinline__ uint32_t largest_of_wave(uint32_t v) {
    v = max_of_lanes<16>(v);
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = a[0] > a[1] ? a[0] : a[1];
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return b[0] > b[1] ? b[0] : b[1];
}

__device__ __forceinline__ int32_t held(int32_t v, int32_t lo, int32_t hi) { return v < lo ? lo : v > hi ? hi : v; }

// Which rows of which sequence a workgroup has, and which part of the tokens.  Where a sequence's tokens are more than an even share of all the work, or rows alone leave the
// chip idle, its blocks of rows are split along the tokens; lengths are known on the device only, so every wavefront works it out for itself: with T the tiles that each
// workgroup on the chip would have if all had the same, a sequence of more than 5/4 T is dealt in parts of about T.  (So units are at most the blocks of rows and as
// many as fit the chip, and parts at most twice the latter.)
struct Own {
    uint32_t b, block, part, parts, place;      // place: of the part, among those of all sequences that are split
    int32_t first, count;                       // the sequence's first new token and how many it has
};
struct Work { int32_t first, end; uint32_t blocks, tiles; };
__device__ __forceinline__ Work work_of(const Prompt& a, uint32_t b, uint32_t rows) {
    if (b >= a.batch) return {0, 0, 0, 0};
    const int32_t room = (int32_t)(a.table_pages << a.c.page_shift);
    const int32_t s = held(a.starts[b], 0, (int32_t)a.tokens), e = held(a.starts[b + 1], 0, (int32_t)a.tokens);
    return {s, e, e > s ? (uint32_t)(((uint64_t)(e - s) * a.group + rows - 1) / rows) : 0, (uint32_t)(held(a.lens[b], 0, room) + kTile - 1) / kTile};
}
__device__ __forceinline__ uint32_t even_of(const Prompt& a, uint64_t work) {
    const uint64_t t = (work + a.share - 1) / a.share;
    return a.most_parts == 1 ? 0x7fffffffu : t < kLeastTiles ? kLeastTiles : t < 0x7fffffffu ? (uint32_t)t : 0x7fffffffu;
}
__device__ __forceinline__ uint32_t parts_of(const Prompt& a, uint32_t tiles, uint32_t even) {
    const uint32_t parts = tiles > even + even / 4 ? (tiles + even - 1) / even : 1;
    return parts < a.most_parts ? parts : a.most_parts;
}
// JOIN: of blocks of rows that are split, counted by themselves.  Of up to 64 sequences the longest first, so that no long one begins when the others end.
template <bool JOIN>
__device__ __forceinline__ Own own_of(const Prompt& a, uint32_t unit, uint32_t lane, uint32_t rows) {
    if (a.deal) {
        const uint32_t step = a.batch + 1, *before = a.deal + (JOIN ? step : 0), *places = a.deal + 2 * step;
        if (unit >= before[a.batch]) return {0, 0, 0, 0, 0, 0, 0};
        uint32_t lo = 0, hi = a.batch;                      // the last sequence that begins at `unit` or before
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (before[mid] <= unit) lo = mid; else hi = mid;
        }
        lo = __builtin_amdgcn_readfirstlane(lo);
        const Work w = work_of(a, lo, rows);
        const uint32_t parts = parts_of(a, w.tiles, a.deal[3 * step]), at = unit - before[lo], block = JOIN ? at : at / parts, part = JOIN ? 0 : at - block * parts;
        return {lo, block, part, parts, places[lo] + block * parts + part, w.first, w.end - w.first};
    }
    const Work w = work_of(a, lane, rows);
    uint64_t work = (uint64_t)w.blocks * w.tiles;
    if (a.most_parts > 1)
        for (int x = 32; x; x /= 2) work += __shfl_xor(work, x);
    const uint32_t parts = parts_of(a, w.tiles, even_of(a, work));
    const uint32_t own = JOIN ? (parts > 1 ? w.blocks : 0) : w.blocks * parts, held_places = parts > 1 ? w.blocks * parts : 0;
    uint32_t upto = own, places_upto = held_places;
    for (int j = 0; j < (int)a.batch; ++j) {
        const uint32_t t = __builtin_amdgcn_readlane(w.tiles, j), o = __builtin_amdgcn_readlane(own, j), p = __builtin_amdgcn_readlane(held_places, j);
        const bool ahead = t > w.tiles || (t == w.tiles && j < (int)lane);
        upto += ahead ? o : 0;
        places_upto += ahead ? p : 0;
    }
    const unsigned long long mine = __ballot(lane < a.batch && upto > unit && upto - own <= unit);
    if (!mine) return {0, 0, 0, 0, 0, 0, 0};
    const int from = __builtin_ctzll(mine);
    Own r;
    r.b = from;
    r.parts = __builtin_amdgcn_readlane(parts, from);
    r.first = __builtin_amdgcn_readlane(w.first, from);
    r.count = __builtin_amdgcn_readlane(w.end, from) - r.first;
    const uint32_t at = unit - (__builtin_amdgcn_readlane(upto, from) - __builtin_amdgcn_readlane(own, from));
    r.block = JOIN ? at : at / r.parts;
    r.part = JOIN ? 0 : at - r.block * r.parts;
    r.place = __builtin_amdgcn_readlane(places_upto, from) - __builtin_amdgcn_readlane(held_places, from) + r.block * r.parts + r.part;
    return r;
}

// How more than 64 sequences are dealt, once for all workgroups: of each the units before it, the blocks that are split and the places of their parts, and what is even.
// One workgroup, a run of sequences a lane.
__global__ __launch_bounds__(1024) void k_kv_prompt_deal(Prompt a, uint32_t rows) {
    __shared__ uint64_t works[1024];
    __shared__ uint32_t sums[3][1024];
    const uint32_t each = (a.batch + 1023) / 1024, first = threadIdx.x * each, end = first + each < a.batch ? first + each : a.batch, step = a.batch + 1;
    uint64_t work = 0;
    for (uint32_t b = first; b < end; ++b) { const Work w = work_of(a, b, rows); work += (uint64_t)w.blocks * w.tiles; }
    works[threadIdx.x] = work;
    __syncthreads();
    for (uint32_t x = 512; x; x /= 2) {
        if (threadIdx.x < x) works[threadIdx.x] += works[threadIdx.x + x];
        __syncthreads();
    }
    const uint32_t even = even_of(a, works[0]);
    uint32_t mine[3] = {0, 0, 0};
    for (uint32_t b = first; b < end; ++b) {
        const Work w = work_of(a, b, rows);
        const uint32_t parts = parts_of(a, w.tiles, even);
        mine[0] += w.blocks * parts;
        mine[1] += parts > 1 ? w.blocks : 0;
        mine[2] += parts > 1 ? w.blocks * parts : 0;
    }
    for (int k = 0; k < 3; ++k) sums[k][threadIdx.x] = mine[k];
    __syncthreads();
    for (uint32_t x = 1; x < 1024; x *= 2) {
        uint32_t before[3];
        for (int k = 0; k < 3; ++k) before[k] = threadIdx.x >= x ? sums[k][threadIdx.x - x] : 0;
        __syncthreads();
        for (int k = 0; k < 3; ++k) sums[k][threadIdx.x] += before[k];
        __syncthreads();
    }
    uint32_t run[3];
    for (int k = 0; k < 3; ++k) run[k] = sums[k][threadIdx.x] - mine[k];
    for (uint32_t b = first; b < end; ++b) {
        const Work w = work_of(a, b, rows);
        const uint32_t parts = parts_of(a, w.tiles, even);
        for (int k = 0; k < 3; ++k) a.deal[k * step + b] = run[k];
        run[0] += w.blocks * parts;
        run[1] += parts > 1 ? w.blocks : 0;
        run[2] += parts > 1 ? w.blocks * parts : 0;
    }
    if (threadIdx.x == 0) {
        for (int k = 0; k < 3; ++k) a.deal[k * step + a.batch] = sums[k][1023];
        a.deal[3 * step] = even;
    }
}

template <int BITS, int D, int kWaves> struct Shape {
    static constexpr int kUnits = D <= 32 ? 4 : D <= 64 ? 8 : D <= 128 ? 16 : 32;      // 16-byte units a row of K has room for
    static constexpr int kRowBytes = D * BITS / 8;
    static constexpr int kChunks = kRowBytes / 16, kKeyItems = kTile * kChunks;         // pieces of 16 bytes of codes
    static constexpr int kWords = kRowBytes / 4, kValueItems = kTile / 4 * kWords;      // and of 4 bytes by 4 tokens
    static constexpr int kKeyLoads = (kKeyItems + kWaves * 64 - 1) / (kWaves * 64), kValueLoads = (kValueItems + kWaves * 64 - 1) / (kWaves * 64);
};
// Where in its row a unit is kept: sixteen lanes that read one column of units from rows that follow each other, and those that write it, have sixteen places in the 256
// bytes that LDS gives at once.  Rows of V^T have eight units; lanes that write it are 4 (8 bits) or 8 (4 bits) rows apart.
template <int UNITS> __device__ __forceinline__ uint32_t key_unit(uint32_t t, uint32_t u) { return u ^ (UNITS >= 16 ? t & 15 : UNITS == 8 ? t >> 1 & 7 : t >> 2 & 3); }
__device__ __forceinline__ uint32_t value_unit(uint32_t d, uint32_t u) { return u ^ ((d >> 1 ^ (d >> 4 & 1)) & 7); }

// Code e of a word of keys; of 4 bits in sixteenths (from a turned word, whose upper nibbles have one of their own).
template <int BITS> struct Word {
    uint32_t w, up;
    __device__ __forceinline__ explicit Word(uint32_t x) : w(x), up(0) {
        if (BITS == 4) w = turned(x);
        asm("" : "+v"(w));                                  // (else codes are cut out one by one before they are converted)
        if (BITS == 4) up = upper_nibbles(w);
    }
    __device__ __forceinline__ float code(int e) const { return BITS == 8 ? (float)(int8_t)(w >> (8 * e)) : low_nibble_of(e % 2 ? up : w, e / 2); }
};
constexpr float unit_of(int bits) { return bits == 4 ? 16.0f : 1.0f; }

// What is left to the compiler's own judgement becomes calls, with registers put away around them, in some of the kernels (heads of 160 in 4 bits twice the time).
#define LC_INLINE __attribute__((always_inline))
// f(Number<0>), f(Number<1>) ... of N.
template <int I> struct Number { static constexpr int value = I; };
template <int N, int I = 0, typename F> __device__ __forceinline__ void each(F&& f) {
    if constexpr (I < N) { f(Number<I>{}); each<N, I + 1>(f); }
}

template <int T, int BITS, int D, int kWaves, int PERSIMD>
__global__ __launch_bounds__(kWaves * 64, PERSIMD) void k_kv_prompt(Prompt a) {
    using S = Shape<BITS, D, kWaves>;
    constexpr int kRows = 32 * kWaves;
    constexpr bool HALF = Kind<T>::kHalf, PHALF = Kind<T>::kHalfValues;
    constexpr int NP = Kind<T>::kParts, KS = D / 16, DB = D / 32;
    constexpr int kScaler = kWaves - 3, kPlacer = kWaves - 1;      // the wavefronts that see to scales and to places
    __shared__ __attribute__((aligned(16))) uint16_t sk[2][kTile][S::kUnits * 8];
    __shared__ __attribute__((aligned(16))) uint16_t sv[2][D][kTile];
    __shared__ __attribute__((aligned(16))) float sks[2][kTile], svs[2][kTile];
    __shared__ uint64_t srow[4][8];                         // where each eight tokens of a tile lie, counted in rows
    __shared__ uint32_t snot[4];                            // which of them lie in pages that are not there
    __shared__ int sunit[2];                                // 16-bit types: probabilities times scales are counted in 2^sunit
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), c = lane % 32, h = lane / 32;
    const uint32_t head = blockIdx.x % a.c.heads;
    const Own own = own_of<false>(a, a.first_unit + blockIdx.x / a.c.heads, lane, kRows);
    if (own.count == 0) return;
    const uint32_t b = own.b;
    const int32_t room = (int32_t)(a.table_pages << a.c.page_shift);
    const int32_t len = held(a.lens[b], 0, room);
    const int32_t rows = (int32_t)(own.count * a.group), blocks = (rows + kRows - 1) / kRows;
    const int32_t row0 = (blocks - 1 - (int32_t)own.block) * kRows;  // (the rows that see most first)
    const int32_t row_last = row0 + kRows < rows ? row0 + kRows - 1 : rows - 1;
    const int32_t base = len - own.count;                   // the place of the first new token
    auto place_of = [&](int32_t row) LC_INLINE { return base + (int32_t)a.by_group((uint32_t)row); };
    const int32_t tiles_all = place_of(row_last) >= 0 ? place_of(row_last) / kTile + 1 : 0;
    const int32_t per = (tiles_all + (int32_t)own.parts - 1) / (int32_t)own.parts;
    const int32_t tile0 = (int32_t)own.part * per, tile1 = tile0 + per < tiles_all ? tile0 + per : tiles_all;

    // this lane's row
    const int32_t row = row0 + (int32_t)(32 * wave + c);
    const bool has_row = row < rows;
    const uint32_t rr = (uint32_t)(has_row ? row : rows - 1), qi = a.by_group(rr), qg = rr - qi * a.group;
    const int32_t place = has_row ? base + (int32_t)qi : -1;
    const int32_t wave_row = row0 + 32 * (int32_t)wave;     // the places of the wavefront's first and last rows
    const int32_t wave_first = place_of(wave_row < rows ? wave_row : rows - 1);
    const int32_t wave_end = wave_row < rows ? place_of(wave_row + 31 < rows ? wave_row + 31 : rows - 1) : -1;
    const int32_t wave_tiles = __builtin_amdgcn_readfirstlane(wave_end < 0 ? 0 : wave_end / kTile + 1 < tile1 ? wave_end / kTile + 1 : tile1);     // those that any of them sees
    u32x4 q[KS][NP];
    {
        const uint64_t at = (uint64_t)(own.first + qi) * a.ld_q + (uint64_t)(head * a.group + qg) * D;
        // An infinity is taken as NaN: the score of whatever is seen is infinite or NaN, so the softmax of any set of them is NaN.
        if constexpr (T == LC_F32) {
#pragma unroll
            for (int o = 0; o < KS; ++o) {
                float v[8];
                load_eight<T>(a.q, at + 16 * o + 8 * h, has_row ? 8 : 0, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += v[e] - v[e];
#pragma unroll
                for (int p = 0; p < NP; ++p) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) q[o][p][j] = high_halves(bits_of(v[2 * j]), bits_of(v[2 * j + 1]));
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] -= float_of(bits_of(v[e]) & 0xffff0000u);
                }
                __builtin_amdgcn_sched_barrier(0);          // (else all of q is there three times over)
            }
        } else {
            constexpr uint32_t kTop = HALF ? 0x7c00u : 0x7f80u;     // the exponent of what is not finite
            bool wrong = false;
#pragma unroll
            for (int o = 0; o < KS; ++o) {
                q[o][0] = has_row ? load_once<u32x4>(static_cast<const uint16_t*>(a.q) + at + 16 * o + 8 * h) : u32x4{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < 4; ++j) wrong |= (q[o][0][j] & kTop) == kTop || (q[o][0][j] & kTop << 16) == kTop << 16;
            }
            if (wrong) q[0][0][0] = 0x7fff7fffu;
        }
    }

    // A tile on its way: eight lanes look up where it lies, a tile ahead; codes go to registers and, converted, into LDS.
    const int32_t* table = a.table + b * a.ld_table;
    int32_t page_raw = 0;
    auto token_of = [&](int32_t tile) LC_INLINE {                     // the lane's eight tokens (that begin at a multiple of eight, and so lie together)
        const int32_t t = (tile < tiles_all ? tile : tiles_all - 1) * kTile + 8 * (int32_t)(lane % 8);
        return t < len ? t : (len - 1) & ~7;
    };
    auto look = [&](int32_t tile, uint32_t lanes) LC_INLINE {         // (of several tiles that follow each other, eight lanes each)
        if (wave == kPlacer && lane < lanes) page_raw = table[token_of(tile + (int32_t)lane / 8) >> a.c.page_shift];
    };
    auto place_eights = [&](int32_t tile, uint32_t lanes) LC_INLINE {
        if (wave != kPlacer || lane >= lanes) return;
        tile += (int32_t)lane / 8;
        const bool there = (uint32_t)page_raw < (uint32_t)a.pages;
        srow[tile % 4][lane % 8] = row_of(a.c, there ? page_raw : 0, head, (uint32_t)token_of(tile) & ((1u << a.c.page_shift) - 1));
        const unsigned long long missing = __ballot(!there);
        if (lane % 8 == 0) snot[tile % 4] = (uint32_t)(missing >> lane) & 255u;
    };
    u32x4 keys[S::kKeyLoads];
    uint32_t values[S::kValueLoads][4];
    float key_scale = 0, value_scale = 0;
    auto ask = [&](int32_t tile) LC_INLINE {
        const uint64_t* eights = srow[tile % 4];
#pragma unroll
        for (int l = 0; l < S::kKeyLoads; ++l) {
            const uint32_t i = l * kWaves * 64 + threadIdx.x, t = i / S::kChunks, ch = i % S::kChunks;
            if (S::kKeyItems % (kWaves * 64) == 0 || i < (uint32_t)S::kKeyItems)
                keys[l] = *reinterpret_cast<const u32x4*>(a.c.k + eights[t / 8] * S::kRowBytes + (t % 8 * S::kRowBytes + ch * 16));
        }
#pragma unroll
        for (int l = 0; l < S::kValueLoads; ++l) {
            const uint32_t i = l * kWaves * 64 + threadIdx.x, t = i / S::kWords * 4, w = i % S::kWords;
            if (S::kValueItems % (kWaves * 64) == 0 || i < (uint32_t)S::kValueItems) {
                const uint8_t* from = a.c.v + eights[t / 8] * S::kRowBytes + (t % 8 * S::kRowBytes + w * 4);
#pragma unroll
                for (int r = 0; r < 4; ++r) values[l][r] = *reinterpret_cast<const uint32_t*>(from + r * S::kRowBytes);
            }
        }
        if (wave == kScaler) {
            key_scale = a.c.k_scale[eights[lane / 8] + lane % 8];
            value_scale = a.c.v_scale[eights[lane / 8] + lane % 8];
        }
    };
    int unit = -1000;                                       // 16-bit types: what this wavefront's sums are counted in; and for the one that sees to scales the tiles so far
    int unit_next = -1000;
    const int32_t place_last = place_of(row_last);          // the last place that any row here sees
    auto put_scales = [&](int32_t tile, uint32_t buffer) LC_INLINE {
        if (wave == kScaler) {
            // What no row here sees, behind that place or in a page that is not there, may have any scale, which must not set what products are counted in.
            if (PHALF && (tile * kTile + (int32_t)lane > place_last || (snot[tile % 4] >> lane / 8 & 1))) value_scale = 0;
            // A value that is not finite makes all of a result NaN: as well a key that is not does, and products with the values are left without it.
            const uint32_t size = bits_of(value_scale) & 0x7fffffffu;
            const bool finite = size < 0x7f800000u;
            sks[buffer][lane] = finite ? key_scale * a.scale : __builtin_nanf("");
            if (!finite) value_scale = 0;
            if (PHALF) {
                const uint32_t most = largest_of_wave(finite ? size : 0);
                int e = (int)(most >> 23) - 127 - 10;
                e = e < -100 ? -100 : e;
                unit_next = e > unit_next ? e : unit_next;
                value_scale = ldexpf(value_scale, -unit_next);
                if (lane == 0) sunit[buffer] = unit_next;
            }
            svs[buffer][lane] = value_scale;
        }
    };
    // The conversions of a lane, by pieces: eight codes of a key, or one element of four tokens' values.  Where they go in LDS: a place a load, turned by the piece (units of
    // a row and rows of V^T follow each other in powers of two, so turning and counting do not meet).
    constexpr int kKeyPieces = S::kKeyLoads * (16 / BITS), kPieces = kKeyPieces + S::kValueLoads * (32 / BITS);
    uint32_t key_to[S::kKeyLoads], value_to[S::kValueLoads];
#pragma unroll
    for (int l = 0; l < S::kKeyLoads; ++l) {
        const uint32_t i = l * kWaves * 64 + threadIdx.x, t = i / S::kChunks, ch = i % S::kChunks;
        key_to[l] = t * S::kUnits * 16 + key_unit<S::kUnits>(t, ch * (16 / BITS)) * 16;
    }
#pragma unroll
    for (int l = 0; l < S::kValueLoads; ++l) {
        const uint32_t i = l * kWaves * 64 + threadIdx.x, t = i / S::kWords * 4, d = i % S::kWords * (32 / BITS);
        const uint32_t group = t / 4 % 4, unit = t / 16 * 2 + group % 2, half = group / 2;      // tokens 0-3, 8-11, 4-7, 12-15
        value_to[l] = d * kTile * 2 + value_unit(d, unit) * 16 + half * 8;
    }
    auto put = [&](uint32_t buffer, auto piece_of) LC_INLINE {
        constexpr int piece = decltype(piece_of)::value;
        if constexpr (piece < kKeyPieces) {
            constexpr int l = piece / (16 / BITS), u = piece % (16 / BITS);
            if (S::kKeyItems % (kWaves * 64) && l * kWaves * 64 + threadIdx.x >= (uint32_t)S::kKeyItems) return;
            u32x4 v;
#pragma unroll
            for (int n = 0; n < BITS / 4; ++n) {
                const Word<BITS> w(keys[l][u * BITS / 4 + n]);
#pragma unroll
                for (int j = 0; j < 16 / BITS; ++j) v[n * 2 + j] = pair_of<HALF>(w.code(2 * j), w.code(2 * j + 1));
            }
            uint32_t to = key_to[l];
            asm("" : "+v"(to));                             // (else places are worked out for every piece before the first tile, for which there are no registers)
            *reinterpret_cast<u32x4*>(reinterpret_cast<uint8_t*>(sk[buffer]) + (to ^ (u * 16))) = v;
        } else {
            // (4 bits: the lower nibbles of all bytes first, then the upper ones, for which words are moved on)
            constexpr int l = (piece - kKeyPieces) / (32 / BITS), n = (piece - kKeyPieces) % (32 / BITS), e = BITS == 8 ? n : n % 4 * 2 + n / 4;
            if (S::kValueItems % (kWaves * 64) && l * kWaves * 64 + threadIdx.x >= (uint32_t)S::kValueItems) return;
            float x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                uint32_t& w = values[l][r];
                if (BITS == 4 && n == 0) w = turned(w);
                if (BITS == 4 && n == 4) w = upper_nibbles(w);
                x[r] = BITS == 8 ? (float)(int8_t)(w >> (8 * e)) : low_nibble_of(w, n % 4);
            }
            uint32_t to = value_to[l];
            asm("" : "+v"(to));
            *reinterpret_cast<u32x2*>(reinterpret_cast<uint8_t*>(sv[buffer]) + (to ^ (e / 2 * 16)) + e * kTile * 2) = u32x2{pair_of<PHALF>(x[0], x[1]), pair_of<PHALF>(x[2], x[3])};
        }
    };
    auto put_all = [&](uint32_t buffer) LC_INLINE { each<kPieces>([&](auto piece) LC_INLINE { put(buffer, piece); }); };

    f32x16 acc[DB];
#pragma unroll
    for (int j = 0; j < DB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[j][e] = 0;
    float top = -__builtin_inff(), from = 0, sum = 0;       // the largest score so far (or about that), what probabilities are measured from, their sum

    // A tile: scores, what probabilities are measured from, probabilities, products with the values.
    auto use = [&](int32_t tile, uint32_t buffer) LC_INLINE {         // (and, beside the scores, puts the next one in its place)
        const int32_t tb = tile * kTile;
        const uint32_t missing = __builtin_amdgcn_readfirstlane(snot[tile % 4]);
        const int unit_now = PHALF ? __builtin_amdgcn_readfirstlane(sunit[buffer]) : unit;
        // Scores: keys are read four products ahead, and between those the next tile is converted.  (What is written here one after the other stays so: left to
        // itself the compiler reads each key right before its product, and the matrix unit waits.)
        f32x16 score[2];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int e = 0; e < 16; ++e) score[s][e] = 0;
        uint32_t key_from = c * S::kUnits * 16 + key_unit<S::kUnits>(c, h) * 16 + buffer * (uint32_t)sizeof(sk[0]);
        asm("" : "+v"(key_from));
        auto key_at = [&](int i) LC_INLINE {
            return *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(sk) + (key_from ^ (i % KS * 32)) + i / KS * 32 * S::kUnits * 16);
        };
        u32x4 key[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) key[i] = key_at(i);
        each<2 * KS>([&](auto step) LC_INLINE {
            constexpr int i = decltype(step)::value;
#pragma unroll
            for (int p = NP - 1; p >= 0; --p) score[i / KS] = mfma<HALF>(key[i % 4], q[i % KS][p], score[i / KS]);
            if constexpr (i + 4 < 2 * KS) key[i % 4] = key_at(i + 4);
            each<(i + 1) * kPieces / (2 * KS) - i * kPieces / (2 * KS)>([&](auto n) LC_INLINE { put(buffer ^ 1, Number<i * kPieces / (2 * KS) + decltype(n)::value>{}); });
            __builtin_amdgcn_sched_barrier(0);
        });
        ask(tile + 2);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 ks = *reinterpret_cast<const f32x4*>(&sks[buffer][32 * s + 8 * g + 4 * h]);
#pragma unroll
                for (int r = 0; r < 4; ++r) score[s][4 * g + r] = fmaf(score[s][4 * g + r], ks[r], -from);
            }
        if (tb + kTile - 1 > wave_first || missing) {       // (else every row sees all of it)
            asm volatile("");                               // (a branch, not 64 selections for every tile)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const bool hidden = tb + 32 * s + 8 * (e / 4) + (int32_t)(4 * h) + e % 4 > place || (missing >> (4 * s + e / 4) & 1);
                    score[s][e] = hidden ? -__builtin_inff() : score[s][e];
                }
        }
        float most = -__builtin_inff();
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int e = 0; e < 16; ++e) most = fmaxf(most, score[s][e]);
        // What probabilities are measured from moves only when one would pass 2^kFar, what sums are counted in when a larger scale comes, so sums are seldom rescaled.
        if (__any(most > Kind<T>::kFar || top == -__builtin_inff()) || unit_now != unit) {
            most = fmaxf(fmaxf(most, other_half(most)) + from, top);
            // Products are counted in a unit for all rows, by the largest scale that any of them sees.  A row that does not see it, because its token is later, measures its probabilities from
            // as much lower: its products do not pass 2^11 so, and keep their bits.  (This is the last tile that such a row sees anything of.)
            const bool unlike = PHALF && tb + kTile - 1 > wave_first && unit_now != unit;       // (else all rows see all that set the unit)
            if (unlike && __any(svs[buffer][lane] != 0.0f && fabsf(svs[buffer][lane]) < kNear)) {
                float large = 0;
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x4 vs = *reinterpret_cast<const f32x4*>(&svs[buffer][32 * s + 8 * g + 4 * h]);
#pragma unroll
                        for (int r = 0; r < 4; ++r) large = fmaxf(large, score[s][4 * g + r] == -__builtin_inff() ? 0.0f : fabsf(vs[r]));
                    }
                large = fmaxf(large, other_half(large));
                const int own_unit = (int)(bits_of(large) >> 23) - 127 - 10, below = -(own_unit > unit - unit_now ? own_unit : unit - unit_now);
                most -= large > 0.0f ? (float)(below < kLowest ? below : kLowest) : 0.0f;
            }
            const float then = most == -__builtin_inff() ? 0.0f : most, shrink = __builtin_amdgcn_exp2f(top - then);
            sum *= shrink;
            const float by = PHALF ? ldexpf(shrink, unit - unit_now) : shrink;
#pragma unroll
            for (int j = 0; j < DB; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[j][e] *= by;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int e = 0; e < 16; ++e) score[s][e] -= then - from;
            top = most;
            from = then;
            unit = unit_now;
        }
        // Products with the values, 16 tokens at a time: those of the next 16 are read, and their probabilities worked out, between them.
        uint32_t value_from = c * kTile * 2 + value_unit(c, h) * 16 + buffer * (uint32_t)sizeof(sv[0]);
        asm("" : "+v"(value_from));
        auto value_at = [&](int g, int j) LC_INLINE { return *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(sv) + (value_from ^ (g * 32)) + j * 32 * kTile * 2); };
        u32x4 value[DB], pp[2][NP];
        f32x4 vs[2][2];
        auto scales_at = [&](int g) LC_INLINE {
#pragma unroll
            for (int x = 0; x < 2; ++x) vs[g % 2][x] = *reinterpret_cast<const f32x4*>(&svs[buffer][16 * g + 8 * x + 4 * h]);
        };
        auto probability = [&](int g, int pair) LC_INLINE {           // two of the lane's eight
            float p[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int e = 2 * pair + x;
                p[x] = __builtin_amdgcn_exp2f(score[g / 2][8 * (g % 2) + e]);
                sum += p[x];
                p[x] *= vs[g % 2][e / 4][e % 4];
            }
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                pp[g % 2][k][pair] = k == NP - 1 ? pair_of<PHALF>(p[0], p[1]) : high_halves(bits_of(p[0]), bits_of(p[1]));
                if (k < NP - 1)
#pragma unroll
                    for (int x = 0; x < 2; ++x) p[x] -= float_of(bits_of(p[x]) & 0xffff0000u);
            }
        };
#pragma unroll
        for (int j = 0; j < DB; ++j) value[j] = value_at(0, j);
        scales_at(0);
#pragma unroll
        for (int pair = 0; pair < 4; ++pair) probability(0, pair);
        each<4>([&](auto group) LC_INLINE {
            constexpr int g = decltype(group)::value;
            if constexpr (g < 3) scales_at(g + 1);
            each<DB>([&](auto block) LC_INLINE {
                constexpr int j = decltype(block)::value;
#pragma unroll
                for (int k = NP - 1; k >= 0; --k) acc[j] = mfma<PHALF>(value[j], pp[g % 2][k], acc[j]);
                if constexpr (g < 3) {
                    value[j] = value_at(g + 1, j);
                    each<(j + 1) * 4 / DB - j * 4 / DB>([&](auto n) LC_INLINE { probability(g + 1, j * 4 / DB + decltype(n)::value); });
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    };

    // (Behind the last tile it is asked for once more, into a buffer that nothing reads.)
    if (tile0 < tile1) {
        look(tile0, 24);
        place_eights(tile0, 24);
        __syncthreads();
        ask(tile0);
        put_scales(tile0, 0);
        put_all(0);
        ask(tile0 + 1);
    }
    uint32_t buffer = 0;
    int32_t tile = tile0;
    for (; tile < wave_tiles; ++tile, buffer ^= 1) {
        __syncthreads();
        look(tile + 3, 8);
        put_scales(tile + 1, buffer ^ 1);
        use(tile, buffer);
        place_eights(tile + 3, 8);
    }
    for (; tile < tile1; ++tile, buffer ^= 1) {             // (what only other wavefronts' rows see; they meet as often in this loop as in the one above)
        __syncthreads();
        look(tile + 3, 8);
        put_scales(tile + 1, buffer ^ 1);
        put_all(buffer ^ 1);
        ask(tile + 2);
        place_eights(tile + 3, 8);
    }

    float total = sum + other_half(sum);
    if (!has_row) return;
    const uint64_t at = (uint64_t)(own.first + qi), hd = head * a.group + qg;
    float whole = own.parts > 1 || total == 0.0f ? 1.0f : 1.0f / total;
    whole *= unit_of(BITS);
    if (PHALF) whole = total == 0.0f ? 0.0f : ldexpf(whole, unit);
    if (own.parts > 1) {
        // (A sum of probabilities measured from far below the largest is brought near 1, so that products with large values fit.)
        if (PHALF && total > 0x1p40f) {
            const int e = (int)(bits_of(total) >> 23) - 127;
            top += (float)e;
            total = ldexpf(total, -e);
            whole = ldexpf(whole, -e);
        }
        const uint64_t place_at = ((uint64_t)own.place * a.c.heads + head) * kRows + 32 * wave + c;
        if (h == 0) *reinterpret_cast<f32x2*>(a.stats + 2 * place_at) = f32x2{top, total};
        if (total == 0.0f) return;
        float* to = a.part + place_at * D;
#pragma unroll
        for (int j = 0; j < DB; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 v = {acc[j][4 * g], acc[j][4 * g + 1], acc[j][4 * g + 2], acc[j][4 * g + 3]};
                *reinterpret_cast<f32x4*>(to + 32 * j + 8 * g + 4 * h) = v * whole;
            }
        return;
    }
#pragma unroll
    for (int j = 0; j < DB; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 v = f32x4{acc[j][4 * g], acc[j][4 * g + 1], acc[j][4 * g + 2], acc[j][4 * g + 3]} * whole;
            const uint64_t to = at * a.ld_out + hd * D + 32 * j + 8 * g + 4 * h;
            if (T == LC_F32) *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + to) = v;
            else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + to) = u32x2{pair_of<HALF>(v[0], v[1]), pair_of<HALF>(v[2], v[3])};
        }
}

// The parts of a block of rows, joined, 32 rows a workgroup: first each row's factors, then a lane four elements, eight parts' at once.
constexpr uint32_t kJoined = 32;
template <int T>
__global__ __launch_bounds__(256) void k_kv_prompt_join(Prompt a, uint32_t rows) {
    __shared__ float factor[kJoined][kMostParts + 1];
    const uint32_t head = blockIdx.x % a.c.heads, lane = threadIdx.x % 64;
    __shared__ Own shared_own;
    if (threadIdx.x < 64) {                                 // (most workgroups find that there is nothing for them)
        const Own found = own_of<true>(a, blockIdx.x / a.c.heads, lane, rows);
        if (lane == 0) shared_own = found;
    }
    __syncthreads();
    const Own own = shared_own;
    if (own.count == 0) return;
    const uint32_t all = (uint32_t)own.count * a.group, blocks = (all + rows - 1) / rows, row0 = (blocks - 1 - own.block) * rows + blockIdx.y * kJoined;
    if (row0 >= all) return;
    const uint32_t here = all - row0 < kJoined ? all - row0 : kJoined;
    const uint64_t step = (uint64_t)a.c.heads * rows, first = ((uint64_t)own.place * a.c.heads + head) * rows + blockIdx.y * kJoined;      // from part to part; the first
    for (uint32_t r = threadIdx.x / 32; r < here; r += 8) {             // half a wavefront a row, a lane a part
        const uint32_t p = threadIdx.x % 32;
        f32x2 stat = {-__builtin_inff(), 0};
        if (p < own.parts) stat = *reinterpret_cast<const f32x2*>(a.stats + 2 * (first + r + p * step));
        float m = stat[0];
        for (int x = 16; x; x /= 2) m = fmaxf(m, __shfl_xor(m, x));
        const float f = stat[1] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(stat[0] - m);
        float l = stat[1] == 0.0f ? 0.0f : f * stat[1];
        for (int x = 16; x; x /= 2) l += __shfl_xor(l, x);
        factor[r][p] = l == 0.0f ? 0.0f : f * (1.0f / l);
    }
    static_assert(kMostParts == 32, "a lane a part");
    __syncthreads();
    const uint32_t quads = a.c.dim / 4;
    for (uint32_t i = threadIdx.x; i < here * quads; i += 256) {
        const uint32_t r = i / quads, d = 4 * (i - r * quads), qi = a.by_group(row0 + r), qg = row0 + r - qi * a.group;
        const float* from = a.part + (first + r) * a.c.dim + d;
        f32x4 o = {0, 0, 0, 0};
        for (uint32_t p0 = 0; p0 < own.parts; p0 += 8) {    // (the last again beyond the last)
            f32x4 v[8];
#pragma unroll
            for (uint32_t p = 0; p < 8; ++p) v[p] = *reinterpret_cast<const f32x4*>(from + (p0 + p < own.parts ? p0 + p : own.parts - 1) * step * a.c.dim);
#pragma unroll
            for (uint32_t p = 0; p < 8; ++p) {
                const float f = p0 + p < own.parts ? factor[r][p0 + p] : 0.0f;
                if (f != 0.0f)                              // (else nothing was written there)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = fmaf(f, v[p][e], o[e]);
            }
        }
        store_four<T>(a.out, (uint64_t)(own.first + qi) * a.ld_out + (uint64_t)(head * a.group + qg) * a.c.dim + d, o);
    }
}

// How rows are dealt to workgroups.  Eight wavefronts a workgroup share conversions (2048 of 10000 tokens of 32 / 8 heads 323 us for 355 with four, 512 of 8192 97 for 107) where two
// a SIMD have the registers and rows are many; sequences of few rows leave much of 256 unused (9 of 57 to 517 tokens 155 for 141).  Splitting is left out where rows fill the
// chip: once if all is one sequence, else four times.
struct Deal { uint32_t waves, blocks, share, most_parts; };
uint32_t share_of(uint64_t chip, uint32_t kv_heads) { return (uint32_t)(chip > kv_heads ? chip / kv_heads : 1); }
Deal deal_of(uint64_t tokens, uint64_t batch, uint32_t group, uint32_t kv_heads, bool two) {
    const uint64_t sequences = tokens < batch ? tokens : batch;      // those with new tokens
    Deal d;
    d.waves = two && tokens * group / 256 * kv_heads >= 64 && tokens * group >= 1024 * sequences ? 8 : 4;
    const uint64_t rows = 32 * d.waves, chip = two && d.waves == 4 ? 512 : 256;      // workgroups that are on the chip at once
    d.blocks = (uint32_t)((tokens * group + rows - 1) / rows + sequences);
    d.share = share_of(chip, kv_heads);
    d.most_parts = tokens * group / rows * kv_heads >= chip * (batch == 1 ? 1 : 4) ? 1 : kMostParts;
    return d;
}
bool two_fit(int dtype, uint32_t dim) { return dtype != LC_F32 && dim <= 128; }        // two wavefronts a SIMD have the registers
uint64_t deal_bytes(uint64_t batch) { return batch > 64 ? ((3 * (batch + 1) + 1) * 4 + 255) / 256 * 256 : 0; }
uint64_t places_of(const Deal& d, uint32_t kv_heads) { return d.most_parts == 1 ? 0 : 2ull * d.share * kv_heads; }
uint64_t rows_bytes(uint64_t rows, int dim) { return (rows * 8 + 255) / 256 * 256 + rows * dim * 4; }      // of parts: a maximum and a sum, and dim elements
bool bad_sizes(uint64_t tokens, uint64_t batch, int heads, int kv_heads, int dim) {
    return tokens > (1ull << 24) || batch > 65535 || kv_heads < 1 || kv_heads > 1024 || heads < kv_heads || heads % kv_heads || heads > 4096 || dim < 32 || dim > 256 ||
           dim % 32 || tokens * heads > (1ull << 30);
}

template <int T, int BITS, int D>
void prompt_of(const Prompt& a, const Deal& d, hipStream_t s) {
    constexpr int PERSIMD = T == LC_F32 || D > 128 ? 1 : 2;
    if (a.deal) k_kv_prompt_deal<<<1, 1024, 0, s>>>(a, 32 * (PERSIMD == 2 ? d.waves : 4));
    // (by launches of fewer than 2^32 threads)
    const uint32_t units = d.blocks + (a.most_parts > 1 ? d.share : 0), step = (1u << 31) / 512 / a.c.heads;
    Prompt p = a;
    for (uint32_t u = 0; u < units; u += step) {
        const uint32_t grid = (units - u < step ? units - u : step) * a.c.heads;
        p.first_unit = u;
        if constexpr (PERSIMD == 2)
            if (d.waves == 8) { k_kv_prompt<T, BITS, D, 8, 2><<<grid, 512, 0, s>>>(p); continue; }
        k_kv_prompt<T, BITS, D, 4, PERSIMD><<<grid, 256, 0, s>>>(p);
    }
}
template <int T, int BITS>
void prompt(const Prompt& a, const Deal& d, hipStream_t s) {
    switch (a.c.dim) {
        case 32: prompt_of<T, BITS, 32>(a, d, s); break;
        case 64: prompt_of<T, BITS, 64>(a, d, s); break;
        case 96: prompt_of<T, BITS, 96>(a, d, s); break;
        case 128: prompt_of<T, BITS, 128>(a, d, s); break;
        case 160: prompt_of<T, BITS, 160>(a, d, s); break;
        case 192: prompt_of<T, BITS, 192>(a, d, s); break;
        case 224: prompt_of<T, BITS, 224>(a, d, s); break;
        default: prompt_of<T, BITS, 256>(a, d, s); break;
    }
    if (a.most_parts > 1) {
        const uint32_t blocks = (d.blocks < d.share ? d.blocks : d.share) * a.c.heads;      // (a block that is split has the work of more than one of the chip's)
        k_kv_prompt_join<T><<<dim3(blocks, 32 * d.waves / kJoined), 256, 0, s>>>(a, 32 * d.waves);
    }
}

}  // namespace
}  // namespace serve
}  // namespace lc

using namespace lc::serve;

extern "C" {

size_t lc_kv_prompt_workspace_bytes(uint64_t tokens, uint64_t batch, int heads, int kv_heads, int dim) {
    if (bad_sizes(tokens, batch, heads, kv_heads, dim)) return 0;
    if (tokens == 0 || batch == 0) return 256;
    uint64_t most = 0;                                      // (of both ways there are, whatever the type)
    for (int two = 0; two < 2; ++two) {
        const Deal d = deal_of(tokens, batch, (uint32_t)(heads / kv_heads), (uint32_t)kv_heads, two != 0);
        const uint64_t rows = places_of(d, (uint32_t)kv_heads) * 32 * d.waves;
        most = rows > most ? rows : most;
    }
    return (size_t)(rows_bytes(most, dim) + 256 + deal_bytes(batch));
}

size_t lc_kv_prompt_workspace_most(uint64_t tokens, uint64_t batch, int heads, int kv_heads, int dim) {
    if (bad_sizes(tokens, batch, heads, kv_heads, dim)) return 0;
    if (tokens == 0 || batch == 0) return 256;
    uint64_t most = 0;                                      // (of every way there is to deal rows)
    for (const uint32_t waves : {4u, 8u})
        for (const uint64_t chip : {256u, 512u}) {
            if (waves == 8 && chip > 256) continue;        // (eight are given where one workgroup a compute unit is)
            const uint64_t rows = places_of({waves, 0, share_of(chip, (uint32_t)kv_heads), kMostParts}, (uint32_t)kv_heads) * 32 * waves;
            most = rows > most ? rows : most;
        }
    return (size_t)(rows_bytes(most, dim) + 256 + deal_bytes(batch));
}

int lc_kv_attend_prompt(const lc_kv_cache* cache, const void* q, uint64_t ld_q, uint64_t tokens, int heads, const int32_t* starts, uint64_t batch,
                        const int32_t* table, uint64_t ld_table, uint64_t table_pages, const int32_t* lens, float scale, void* out, uint64_t ld_out, int dtype,
                        void* ws, size_t ws_bytes, void* stream) {
    if (!served_type(dtype) || bad(cache)) return LC_ERR_BADARG;
    const size_t need = lc_kv_prompt_workspace_bytes(tokens, batch, heads, cache->heads, cache->dim);
    if (!need) return LC_ERR_BADARG;
    if (tokens == 0 || batch == 0) return LC_OK;
    const uint64_t width = (uint64_t)heads * cache->dim, step = dtype == LC_F32 ? 4 : 8;
    if (!q || !out || !starts || !lens || off(q, 16) || off(out, 16) || off(starts, 4) || off(lens, 4) || (table_pages && (!table || off(table, 4))) ||
        ld_table > (1ull << 31) || table_pages > (1ull << 30) / cache->page_tokens || (batch > 1 && ld_table < table_pages)) return LC_ERR_BADARG;
    if (ld_q > (1ull << 40) || ld_out > (1ull << 40) || (tokens > 1 && (ld_q < width || ld_out < width || ld_q % step || ld_out % step))) return LC_ERR_BADARG;
    if (!ws || off(ws, 256) || ws_bytes < need) return LC_ERR_WORKSPACE;
    Prompt a = {};
    a.c = described(*cache);
    a.q = q; a.ld_q = ld_q; a.starts = starts; a.table = table; a.ld_table = ld_table; a.table_pages = cache->pages ? table_pages : 0; a.lens = lens;
    a.out = out; a.ld_out = ld_out;
    a.scale = scale * kLog2e * unit_of(cache->bits);
    a.tokens = (uint32_t)tokens; a.batch = (uint32_t)batch; a.heads = (uint32_t)heads; a.group = (uint32_t)(heads / cache->heads);
    a.by_group = FastDiv(a.group);
    a.pages = (int32_t)(cache->pages > 0x7fffffffull ? 0x7fffffff : cache->pages);
    const Deal d = deal_of(tokens, batch, a.group, a.c.heads, two_fit(dtype, a.c.dim));
    a.share = d.share;
    a.most_parts = a.table_pages << a.c.page_shift <= (kLeastTiles + kLeastTiles / 4) * kTile ? 1 : d.most_parts;
    a.deal = batch > 64 ? static_cast<uint32_t*>(ws) : nullptr;
    a.stats = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + deal_bytes(batch));
    a.part = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(a.stats) + (places_of(d, a.c.heads) * 32 * d.waves * 8 + 255) / 256 * 256);
    hipStream_t s = static_cast<hipStream_t>(stream);
#define CALL(T) do { if (cache->bits == 8) prompt<T, 8>(a, d, s); else prompt<T, 4>(a, d, s); } while (0)
    if (dtype == LC_F32) CALL(LC_F32);
    else if (dtype == LC_BF16) CALL(LC_BF16);
    else CALL(LC_F16);
#undef CALL
    return launched();
}

}  // extern "C"
