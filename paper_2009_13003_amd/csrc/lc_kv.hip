// A paged cache of keys and values in 8 or 4 bits: writing, reading back, and the attention over it (include/lc_serve.h).
#include "lc_serve.h"

namespace lc {
namespace serve {
namespace {

struct Cache {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    uint64_t slots;             // pages * page_tokens
    uint32_t page_shift, heads, dim, row_bytes;
};

// Where a head's token lies: the row of codes and the scale, counted in rows.
__device__ __forceinline__ uint64_t row_of(const Cache& c, uint64_t page, uint32_t head, uint32_t token) {
    return ((page * c.heads + head) << c.page_shift) + token;
}

// ---------------------------------------------------------------- writing and reading back
// A lane takes eight elements of a token's head, a power of two of lanes (those behind the last element idle) the whole head; the
// keys are the first half of the grid, the values the second.
template <int T, int BITS, int LANES>
__global__ __launch_bounds__(256) void k_kv_write(Cache c, const void* k, const void* v, uint64_t ld_token, uint64_t ld_head, const int64_t* slots,
                                                  uint32_t items, FastDiv by_heads) {
    const uint32_t item = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, at = 8 * (threadIdx.x % LANES);
    const bool in = item < items;
    const uint32_t token = by_heads(in ? item : 0), head = (in ? item : 0) - token * c.heads;
    const void* from = blockIdx.y ? v : k;
    float x[8];
    load_eight<T>(from, token * ld_token + head * ld_head + at, in && at < c.dim ? 8 : 0, x);
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) { const uint32_t a = bits_of(x[e]) & 0x7fffffffu; most = a > most ? a : most; }
    most = max_of_lanes<LANES>(most);
    constexpr float kMost = BITS == 8 ? 127.0f : 7.0f;
    float s = float_of(most) * (1.0f / kMost), inv = 0.0f;
    if (most >= 0x7f800000u) s = __builtin_nanf("");
    else if (s < kSmallest) s = 0.0f;
    else inv = 1.0f / s;
    if (!in || at >= c.dim) return;
    const int64_t slot = slots[token];
    if (slot < 0 || (uint64_t)slot >= c.slots) return;
    uint32_t q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = rounded(fminf(fmaxf(inv == 0.0f ? 0.0f : x[e] * inv, -kMost), kMost), BITS == 8 ? 0.0f : 8.0f);
    const uint64_t row = row_of(c, (uint64_t)slot >> c.page_shift, head, (uint32_t)slot & ((1u << c.page_shift) - 1));
    uint8_t* to = (blockIdx.y ? c.v : c.k) + row * c.row_bytes + at * BITS / 8;
    if (BITS == 8) {
        u32x2 w = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e / 4] |= (q[e] & 255u) << (8 * (e % 4));
        *reinterpret_cast<u32x2*>(to) = w;
    } else {
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) w |= (q[e] & 15u) << (4 * e);
        *reinterpret_cast<uint32_t*>(to) = w;
    }
    if (at == 0) (blockIdx.y ? c.v_scale : c.k_scale)[row] = s;
}

template <int T, int BITS>
__global__ __launch_bounds__(256) void k_kv_read(Cache c, const int64_t* slots, void* k, void* v, uint64_t ld_token, uint64_t ld_head, uint32_t lanes,
                                                 FastDiv by_row, FastDiv by_heads) {
    const uint32_t lane = blockIdx.x * 256u + threadIdx.x;
    if (lane >= lanes) return;
    const uint32_t item = by_row(lane), at = 8 * (lane - item * by_row.d);
    const uint32_t token = by_heads(item), head = item - token * c.heads;
    const int64_t slot = slots[token];
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (slot >= 0 && (uint64_t)slot < c.slots) {
        const uint64_t row = row_of(c, (uint64_t)slot >> c.page_shift, head, (uint32_t)slot & ((1u << c.page_shift) - 1));
        const uint8_t* from = (blockIdx.y ? c.v : c.k) + row * c.row_bytes + at * BITS / 8;
        const float s = (blockIdx.y ? c.v_scale : c.k_scale)[row];
        if (BITS == 8) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(from);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (float)(int8_t)(w[e / 4] >> (8 * (e % 4))) * s;
        } else {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(from);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (float)((int)(w >> (4 * e) & 15u) - 8) * s;
        }
    }
    store_eight<T>(blockIdx.y ? v : k, token * ld_token + head * ld_head + at, 8, x);
}

// ---------------------------------------------------------------- attention
// The rows that share a head of the cache are the nq * (heads / kv heads) queries of a sequence; a wavefront holds 16 of them (or 32, 64)
// and walks over its part of the sequence 32 tokens at a time, everything in registers:
//   S^T = K Q^T   rows of the matrix instruction are tokens, columns the queries: lane l gets query l % 16, tokens 4 (l / 16) + 0..3
//   O^T += V^T P^T   the same lane's probabilities are its part of the second operand as they stand, with the tokens
//                    in the order 4 h + 0..3, 16 + 4 h + 0..3, in which the values are then loaded too
// so the running maximum, the sum and the factors of the rescaling are one number a lane, and nothing passes through LDS.
// Scales of keys multiply the scores, scales of values the probabilities; codes enter the matrix instructions as whole numbers, exactly.
constexpr int kTile = 32, kWaves = 4;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr uint32_t kMostSplits = 64, kWantBlocks = 1024, kLeastTokens = 128;

struct Attend {
    Cache c;
    const void* q;
    const int32_t* table; uint64_t ld_table; uint64_t table_pages;
    const int32_t* lens;
    const uint64_t* mask;
    void* out;
    float* part;                // [row][split][dim], then the maximum and the sum of each [row][split]
    float* stats;
    float scale;                // times log2(e)
    uint32_t batch, nq, heads, group, rows;     // rows = nq * group of a head of the cache
    uint32_t splits, tiles;                     // 32-token tiles a split
    int32_t pages;
};

template <int T> struct Kind;       // how many 16-bit parts an element of q, and a probability, are given
template <> struct Kind<LC_F32> { static constexpr int kQ = 3, kP = 3; static constexpr bool kHalf = false; };
template <> struct Kind<LC_BF16> { static constexpr int kQ = 1, kP = 2; static constexpr bool kHalf = false; };
template <> struct Kind<LC_F16> { static constexpr int kQ = 1, kP = 2; static constexpr bool kHalf = true; };

template <bool HALF> __device__ __forceinline__ f32x4 mfma_16(u32x4 a, u32x4 b, f32x4 c) { return HALF ? mfma_f16(a, b, c) : mfma_bf16(a, b, c); }

// Two whole numbers of at most 8 bits as an operand's pair: exact in either type.
template <bool HALF> __device__ __forceinline__ uint32_t pair_of(float a, float b) {
    if (HALF) { const auto h = __builtin_amdgcn_cvt_pkrtz(a, b); uint32_t u; __builtin_memcpy(&u, &h, 4); return u; }
    return high_halves(bits_of(a), bits_of(b));
}
// Nibble j of a word of 4-bit codes as a sixteenth of what it stands for: the instruction reads four bits as a two's complement number
// of sixteenths, which the code with its top bit turned round is.
__device__ __forceinline__ uint32_t turned(uint32_t w) { return w ^ 0x88888888u; }
__device__ __forceinline__ float nibble_of(uint32_t w, int j) { return __builtin_amdgcn_cvt_off_f32_i4((int)(w >> (4 * j))); }
template <int BYTE> __device__ __forceinline__ float byte_of(uint32_t w) { return (float)(int8_t)(w >> (8 * BYTE)); }

// A bf16 operand of the values of eight tokens at element j of each token's `w` (4 bits: turned words, and sixteenths).
template <int BITS> __device__ __forceinline__ u32x4 values_at(const uint32_t (&w)[8], int j) {
    u32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a, b;
        if (BITS == 8) { a = (float)(int8_t)(w[2 * e] >> (8 * j)); b = (float)(int8_t)(w[2 * e + 1] >> (8 * j)); }
        else { a = nibble_of(w[2 * e], j); b = nibble_of(w[2 * e + 1], j); }
        r[e] = high_halves(bits_of(a), bits_of(b));
    }
    return r;
}

__device__ __forceinline__ float max_over_quarters(float v) { v = fmaxf(v, __shfl_xor(v, 16)); return fmaxf(v, __shfl_xor(v, 32)); }
__device__ __forceinline__ float sum_over_quarters(float v) { v += __shfl_xor(v, 16); return v + __shfl_xor(v, 32); }

// A tile of 32 tokens as it lies in the cache.
template <int BITS, int DP> struct InCache {
    static constexpr int kKey = DP * BITS / 32 < 16 ? DP * BITS / 32 : 16;      // bytes of a key a lane loads at once
    static constexpr int kKeyLoads = DP * BITS / 32 / kKey, kKeyWords = kKey / 4;
    static constexpr int kDims = DP / 16;                                       // elements of a value a lane holds
    static constexpr int kValue = kDims * BITS / 8, kValueWords = (kValue + 3) / 4, kPerWord = 32 / BITS < kDims ? 32 / BITS : kDims;
    uint32_t key[2][kKeyLoads][kKeyWords];      // of token 16 s + l % 16
    uint32_t value[8][kValueWords];             // of tokens 16 s + 4 (l / 16) + r, at 4 s + r
    f32x4 key_scale[2], value_scale[2];
};

// Sequences lie in pages of a power of two of tokens, at least 8, so eight tokens that begin at a multiple of eight lie together: where
// each eight of a tile lie is the same for all lanes.
struct Eights { uint64_t row[4]; uint32_t there; };

template <int T, int BITS, int DP, int NT>
__global__ __launch_bounds__(kWaves * 64) void k_kv_attend(Attend a) {
    using Raw = InCache<BITS, DP>;
    constexpr bool HALF = Kind<T>::kHalf;
    constexpr int NQ = Kind<T>::kQ, NP = Kind<T>::kP;
    // Keys in 4 bits for 16-bit queries: 16 + c, a nibble put into the mantissa of 16 (two operations for two codes), and 24 times the
    // query's sum taken away, which moves scores by some 2^-24 of 24 sum |q|; for fp32 exact codes instead.
    constexpr bool LIFTED = BITS == 4 && T != LC_F32;
    constexpr int KOPS = DP / 32, VD = Raw::kDims;
    __shared__ float so[kWaves][16][DP + 4];
    __shared__ float sm[kWaves][16], sl[kWaves][16];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), c = lane % 16, h = lane / 16;
    const uint32_t split = blockIdx.x, row_groups = (a.rows + 16 * NT - 1) / (16 * NT);
    const uint32_t head = blockIdx.y / row_groups, row0 = (blockIdx.y - head * row_groups) * 16 * NT, b = blockIdx.z;
    const int32_t room = (int32_t)(a.table_pages << a.c.page_shift);
    // (What all lanes read alike is read by the scalar unit, which counts its loads apart: a vector load of it, waited for, would wait for
    // the keys and values asked for before it as well.)
    typedef const __attribute__((address_space(4))) int32_t* Uniform;
    const int32_t given = ((Uniform)(uintptr_t)a.lens)[b];
    const int32_t len = given < 0 ? 0 : given < room ? given : room;
    const int32_t base = len - (int32_t)a.nq;               // the first drafted token
    const Uniform table = (Uniform)(uintptr_t)(a.table + b * a.ld_table);
    const int32_t first = (int32_t)(split * a.tiles * kTile);
    const int32_t end = first + (int32_t)a.tiles * kTile < len ? first + (int32_t)a.tiles * kTile : len;
    const int32_t own = first + (int32_t)wave * kTile;      // this wavefront's first tile; every kWaves-th is its own
    const int32_t tiles = own < end ? (end - own + kWaves * kTile - 1) / (kWaves * kTile) : 0;

    // this lane's queries, eight elements an operand at the places at which the keys' codes lie
    u32x4 q[NT][KOPS][NQ];
    f32x4 less[NT];                                         // -24 times each query's sum
    uint64_t mask[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint32_t row = row0 + 16 * n + c;
        const bool has_row = row < a.rows;
        const uint32_t qi = (has_row ? row : 0) / a.group, qg = (has_row ? row : 0) - qi * a.group;
        const uint64_t q_at = (((uint64_t)b * a.nq + qi) * a.heads + head * a.group + qg) * a.c.dim;
        mask[n] = a.mask ? a.mask[(uint64_t)b * a.nq + qi] : qi >= 63 ? ~0ull : (2ull << qi) - 1;
        less[n] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int o = 0; o < KOPS; ++o) {
            uint32_t d;
            if (BITS == 8) d = 16 * h + 64 * (o / 2) + 8 * (o % 2);
            else d = 2 * Raw::kKey * h + 8 * Raw::kKey * (o / Raw::kKeyWords) + 8 * (o % Raw::kKeyWords);
            float v[8];
            load_eight<T>(a.q, q_at + d, has_row && d < a.c.dim ? 8 : 0, v);
#pragma unroll
            for (int p = 0; p < NQ; ++p) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float x = BITS == 8 ? v[2 * j] : v[j], y = BITS == 8 ? v[2 * j + 1] : v[j + 4];
                    q[n][o][p][j] = HALF ? f16_of(x) | f16_of(y) << 16 : high_halves(bits_of(x), bits_of(y));
                }
                if (NQ > 1)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] -= float_of(bits_of(v[e]) & 0xffff0000u);
            }
            if (LIFTED) {
                const uint32_t m24 = HALF ? 0xCE00CE00u : 0xC1C0C1C0u;
#pragma unroll
                for (int p = NQ - 1; p >= 0; --p) less[n] = mfma_16<HALF>(u32x4{m24, m24, m24, m24}, q[n][o][p], less[n]);
            }
        }
    }

    auto find = [&](int32_t i) {                            // where this wavefront's tile i lies (beyond the last: the last again)
        Eights e;
        e.there = 0;
        const int32_t tb = own + (i < tiles ? i : tiles - 1) * kWaves * kTile;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int32_t t = tb + 8 * g < len ? tb + 8 * g : (len - 1) & ~7;
            const int32_t page = table[t >> a.c.page_shift];
            const bool there = (uint32_t)page < (uint32_t)a.pages;
            e.row[g] = row_of(a.c, there ? page : 0, head, (uint32_t)t & ((1u << a.c.page_shift) - 1));
            e.there |= there ? 1u << g : 0;
        }
        return e;
    };
    // (Lanes whose elements lie beyond dim read the row's first: their queries are zero there, or their results go nowhere.)
    uint32_t key_off[Raw::kKeyLoads];
#pragma unroll
    for (int l = 0; l < Raw::kKeyLoads; ++l) {
        const uint32_t at = (4 * l + h) * Raw::kKey;
        key_off[l] = (c % 8) * a.c.row_bytes + (at < a.c.row_bytes ? at : 0);
    }
    const uint32_t value_off = (4 * h % 8) * a.c.row_bytes + (c * Raw::kValue < a.c.row_bytes ? c * Raw::kValue : 0);
    auto load = [&](Raw& f, const Eights& e) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint64_t k0 = e.row[2 * s] * a.c.row_bytes, k1 = e.row[2 * s + 1] * a.c.row_bytes;
            const uint8_t* keys = a.c.k + (c < 8 ? k0 : k1);
#pragma unroll
            for (int l = 0; l < Raw::kKeyLoads; ++l) __builtin_memcpy(f.key[s][l], __builtin_assume_aligned(keys + key_off[l], Raw::kKey), Raw::kKey);
            const uint64_t value_row = h < 2 ? e.row[2 * s] : e.row[2 * s + 1];
            f.key_scale[s] = *reinterpret_cast<const f32x4*>(a.c.k_scale + value_row + 4 * h % 8);
            f.value_scale[s] = *reinterpret_cast<const f32x4*>(a.c.v_scale + value_row + 4 * h % 8);
            const uint8_t* values = a.c.v + (h < 2 ? k0 : k1) + value_off;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (Raw::kValue < 4) f.value[4 * s + r][0] = 0;
                __builtin_memcpy(f.value[4 * s + r], __builtin_assume_aligned(values + r * a.c.row_bytes, Raw::kValue < 16 ? Raw::kValue : 16), Raw::kValue);
            }
        }
    };

    f32x4 acc[NT][VD];
    float top[NT], sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        top[n] = -__builtin_inff();
        sum[n] = 0;
#pragma unroll
        for (int j = 0; j < VD; ++j) acc[n][j] = f32x4{0, 0, 0, 0};
    }
    auto use = [&](const Raw& f, const Eights& e, int32_t tb) {
        f32x4 score[NT][2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int n = 0; n < NT; ++n) score[n][s] = LIFTED ? less[n] : f32x4{0, 0, 0, 0};
#pragma unroll
            for (int o = 0; o < KOPS; ++o) {
                u32x4 key;
                if (BITS == 8) {
                    const uint32_t *w = &f.key[s][o / 2][2 * (o % 2)];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        key[2 * i] = pair_of<HALF>(byte_of<0>(w[i]), byte_of<1>(w[i]));
                        key[2 * i + 1] = pair_of<HALF>(byte_of<2>(w[i]), byte_of<3>(w[i]));
                    }
                } else {
                    const uint32_t w = f.key[s][o / Raw::kKeyWords][o % Raw::kKeyWords];
                    uint32_t into = HALF ? 0x03C003C0u : 0x00780078u;
                    asm("" : "+v"(into));                   // (see codes_as_operand of the products)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int up = (HALF ? 6 : 3) - 4 * j;
                        const uint32_t m = up >= 0 ? w << (up & 31) : w >> (-up & 31);
                        key[j] = LIFTED ? (m & into) | (HALF ? 0x4C004C00u : 0x41804180u)
                                        : high_halves(bits_of(nibble_of(turned(w), j)), bits_of(nibble_of(turned(w), j + 4)));
                    }
                }
#pragma unroll
                for (int p = NQ - 1; p >= 0; --p)
#pragma unroll
                    for (int n = 0; n < NT; ++n) score[n][s] = mfma_16<HALF>(key, q[n][o][p], score[n][s]);
            }
        }
        float ks[8], vs[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            ks[i] = f.key_scale[i / 4][i % 4] * (BITS == 4 && !LIFTED ? 16.0f * a.scale : a.scale);
            vs[i] = f.value_scale[i / 4][i % 4];
        }
        const bool whole = tb + kTile <= base && tb + kTile <= end && e.there == 15;      // all of the tile is seen by all
        u32x4 pp[NT][NP];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = score[n][i / 4][i % 4] * ks[i];
            uint32_t seen = 0xff;
            if (!whole) {
                seen = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int32_t t = tb + 16 * (i / 4) + 4 * h + i % 4, j = t - base;
                    const bool there = e.there >> (2 * (i / 4) + h / 2) & 1;
                    if (there && t < end && (j < 0 || (mask[n] >> (j & 63) & 1))) seen |= 1u << i;
                    if (!(seen >> i & 1)) x[i] = -__builtin_inff();
                }
            }
            float most = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
            // What probabilities are measured from moves only when one would pass 2^8, so that the sums are seldom rescaled.
            most = max_over_quarters(most);
            if (__any(most > top[n] + 8.0f)) {
                most = fmaxf(most, top[n]);
                const float shrink = __builtin_amdgcn_exp2f(top[n] - (most == -__builtin_inff() ? 0.0f : most));
                sum[n] *= shrink;
#pragma unroll
                for (int j = 0; j < VD; ++j) acc[n][j] *= shrink;
                top[n] = most;
            }
            const float from = top[n] == -__builtin_inff() ? 0.0f : top[n];
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = __builtin_amdgcn_exp2f(x[i] - from);
                sum[n] += p[i];
                p[i] *= vs[i];
            }
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] = seen >> i & 1 ? p[i] : 0.0f;          // (what is not seen may have any scale)
            }
#pragma unroll
            for (int k = 0; k < NP; ++k) {
#pragma unroll
                for (int i = 0; i < 4; ++i) pp[n][k][i] = high_halves(bits_of(p[2 * i]), bits_of(p[2 * i + 1]));
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] -= float_of(bits_of(p[i]) & 0xffff0000u);
            }
        }
#pragma unroll
        for (int o = 0; o < Raw::kValueWords; ++o) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = BITS == 4 ? turned(f.value[i][o]) : f.value[i][o];
                if (BITS == 4) asm("" : "+v"(w[i]));         // (turned once, not again for every element)
            }
#pragma unroll
            for (int j = 0; j < Raw::kPerWord; ++j) {
                const u32x4 v = values_at<BITS>(w, j);
#pragma unroll
                for (int k = NP - 1; k >= 0; --k)
#pragma unroll
                    for (int n = 0; n < NT; ++n) acc[n][o * Raw::kPerWord + j] = mfma_bf16(v, pp[n][k], acc[n][o * Raw::kPerWord + j]);
            }
        }
    };

    // While a tile is worked on, the next one is on its way into registers of its own, and the places of the one after that are looked up.
    if (tiles > 0) {
        Raw raw[2];
        Eights at[2];
        at[0] = find(0);
        load(raw[0], at[0]);
        at[1] = find(1);
        for (int32_t i = 0; i < tiles; i += 2) {
            load(raw[1], at[1]);
            const Eights two = find(i + 2);
            use(raw[0], at[0], own + i * kWaves * kTile);
            if (i + 1 >= tiles) break;
            load(raw[0], two);
            const Eights three = find(i + 3);
            use(raw[1], at[1], own + (i + 1) * kWaves * kTile);
            at[0] = two;
            at[1] = three;
        }
    }

    // the wavefronts' parts, joined: lane (c, h) holds elements VD (4 h + r) + j of query c
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (n) __syncthreads();
        const float total = sum_over_quarters(sum[n]);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < VD; ++j) so[wave][c][VD * (4 * h + r) + j] = BITS == 4 ? 16.0f * acc[n][j][r] : acc[n][j][r];
        if (h == 0) { sm[wave][c] = top[n]; sl[wave][c] = total; }
        __syncthreads();
        for (uint32_t e = threadIdx.x; e < 16 * a.c.dim; e += kWaves * 64) {
            const uint32_t r = e / a.c.dim, d = e - r * a.c.dim, row = row0 + 16 * n + r;
            if (row >= a.rows) break;
            float m = sm[0][r];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) m = fmaxf(m, sm[w][r]);
            const float from = m == -__builtin_inff() ? 0.0f : m;
            float l = 0, o = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float f = __builtin_amdgcn_exp2f(sm[w][r] - from);
                l += sl[w][r] == 0.0f ? 0.0f : f * sl[w][r];
                o += sl[w][r] == 0.0f ? 0.0f : f * so[w][r][d];
            }
            const uint32_t i = row / a.group, g = row - i * a.group;
            const uint64_t out_row = ((uint64_t)b * a.nq + i) * a.heads + head * a.group + g;
            if (a.splits == 1) store_one<T>(a.out, out_row * a.c.dim + d, l == 0.0f ? 0.0f : o / l);
            else {
                a.part[(out_row * a.splits + split) * a.c.dim + d] = o;
                if (d == 0) { a.stats[2 * (out_row * a.splits + split)] = m; a.stats[2 * (out_row * a.splits + split) + 1] = l; }
            }
        }
    }
}

// The splits of each row, joined: a wavefront a row.
template <int T>
__global__ __launch_bounds__(256) void k_kv_join(const float* part, const float* stats, void* out, uint64_t rows, uint32_t splits, uint32_t dim) {
    const uint64_t row = blockIdx.x * 4ull + threadIdx.x / 64;
    if (row >= rows) return;
    const uint32_t lane = threadIdx.x % 64;
    const bool has = lane < splits;
    const float m = has ? stats[2 * (row * splits + lane)] : -__builtin_inff(), l = has ? stats[2 * (row * splits + lane) + 1] : 0.0f;
    float top = m;
    for (int x = 1; x < 64; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
    const float f = __builtin_amdgcn_exp2f(m - (top == -__builtin_inff() ? 0.0f : top));
    float total = l == 0.0f ? 0.0f : f * l;
    for (int x = 1; x < 64; x *= 2) total += __shfl_xor(total, x);
    float o[4] = {0, 0, 0, 0};
    for (uint32_t s = 0; s < splits; ++s) {
        if (__shfl(l, s) == 0.0f) continue;
        const float w = __shfl(f, s);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 64 * i < dim) o[i] = fmaf(w, part[(row * splits + s) * dim + lane + 64 * i], o[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < dim) store_one<T>(out, row * dim + lane + 64 * i, total == 0.0f ? 0.0f : o[i] / total);
}

// Splits of a sequence: as many as give the chip enough workgroups, whatever its length.
uint32_t most_splits(uint64_t batch, uint32_t nq, uint32_t heads, uint32_t kv_heads) {
    const uint64_t rows = (uint64_t)nq * (heads / kv_heads), blocks = batch * kv_heads * ((rows + 15) / 16);
    const uint64_t s = blocks ? (kWantBlocks + blocks - 1) / blocks : 1;
    return (uint32_t)(s < kMostSplits ? s : kMostSplits);
}

bool bad(const lc_kv_cache* c) {
    if (!c || c->heads < 1 || c->heads > 1024 || c->dim < 32 || c->dim > 256 || c->dim % 32 || (c->bits != 8 && c->bits != 4)) return true;
    if (c->page_tokens < 8 || c->page_tokens > 1024 || (c->page_tokens & (c->page_tokens - 1)) || c->pages > (1ull << 31) / c->page_tokens) return true;
    if (c->pages == 0) return false;
    return !c->k || !c->v || !c->k_scale || !c->v_scale || off(c->k, 16) || off(c->v, 16) || off(c->k_scale, 16) || off(c->v_scale, 16);
}
Cache described(const lc_kv_cache& c) {
    return {static_cast<uint8_t*>(c.k), static_cast<uint8_t*>(c.v), c.k_scale, c.v_scale, c.pages * c.page_tokens,
            (uint32_t)__builtin_ctz((unsigned)c.page_tokens), (uint32_t)c.heads, (uint32_t)c.dim, (uint32_t)(c.dim * c.bits / 8)};
}
int launched() { return hipGetLastError() == hipSuccess ? LC_OK : LC_ERR_HIP; }

bool bad_vectors(const lc_kv_cache* c, const void* k, const void* v, uint64_t ld_token, uint64_t ld_head, const int64_t* slots, uint64_t tokens, int dtype) {
    const uintptr_t size = size_of(dtype);
    return !k || !v || !slots || off(k, size) || off(v, size) || off(slots, 8) || tokens > (1ull << 31) || ld_token > (1ull << 40) || ld_head > (1ull << 40) ||
           (c->heads > 1 && ld_head < (uint64_t)c->dim) || (tokens > 1 && ld_token < (uint64_t)c->dim);
}

template <int T, int BITS>
void write(const Cache& c, const void* k, const void* v, uint64_t ld_token, uint64_t ld_head, const int64_t* slots, uint64_t tokens, hipStream_t s) {
    const uint32_t lanes = c.dim <= 32 ? 4 : c.dim <= 64 ? 8 : c.dim <= 128 ? 16 : 32;
    const uint64_t step = (1ull << 25) / c.heads;                  // items are counted in 25 bits, a launch's lanes in 31
    for (uint64_t t = 0; t < tokens; t += step) {
        const uint32_t items = (uint32_t)((tokens - t < step ? tokens - t : step) * c.heads);
        const uint64_t by = t * ld_token * (T == LC_F32 ? 4 : 2);
        const void *from_k = static_cast<const uint8_t*>(k) + by, *from_v = static_cast<const uint8_t*>(v) + by;
        const dim3 grid((items + 256 / lanes - 1) / (256 / lanes), 2);
        const FastDiv div(c.heads);
        if (lanes == 4) k_kv_write<T, BITS, 4><<<grid, 256, 0, s>>>(c, from_k, from_v, ld_token, ld_head, slots + t, items, div);
        else if (lanes == 8) k_kv_write<T, BITS, 8><<<grid, 256, 0, s>>>(c, from_k, from_v, ld_token, ld_head, slots + t, items, div);
        else if (lanes == 16) k_kv_write<T, BITS, 16><<<grid, 256, 0, s>>>(c, from_k, from_v, ld_token, ld_head, slots + t, items, div);
        else k_kv_write<T, BITS, 32><<<grid, 256, 0, s>>>(c, from_k, from_v, ld_token, ld_head, slots + t, items, div);
    }
}
template <int T, int BITS>
void read(const Cache& c, const int64_t* slots, uint64_t tokens, void* k, void* v, uint64_t ld_token, uint64_t ld_head, hipStream_t s) {
    const uint64_t step = (1ull << 25) / c.heads;
    for (uint64_t t = 0; t < tokens; t += step) {
        const uint32_t lanes = (uint32_t)((tokens - t < step ? tokens - t : step) * c.heads * (c.dim / 8));
        const uint64_t by = t * ld_token * (T == LC_F32 ? 4 : 2);
        k_kv_read<T, BITS><<<dim3((lanes + 255) / 256, 2), 256, 0, s>>>(c, slots + t, static_cast<uint8_t*>(k) + by, static_cast<uint8_t*>(v) + by, ld_token,
                                                                        ld_head, lanes, FastDiv(c.dim / 8), FastDiv(c.heads));
    }
}
template <int T, int BITS, int DP, int NT>
void attend_of(const Attend& a, hipStream_t s) {
    k_kv_attend<T, BITS, DP, NT><<<dim3(a.splits, a.c.heads * ((a.rows + 16 * NT - 1) / (16 * NT)), a.batch), kWaves * 64, 0, s>>>(a);
}
template <int T, int BITS>
void attend(const Attend& a, hipStream_t s) {
    const bool two = a.rows > 16 && T != LC_F32;
    if (a.c.dim <= 64) two ? attend_of<T, BITS, 64, 2>(a, s) : attend_of<T, BITS, 64, 1>(a, s);
    else if (a.c.dim <= 128) two ? attend_of<T, BITS, 128, 2>(a, s) : attend_of<T, BITS, 128, 1>(a, s);
    else attend_of<T, BITS, 256, 1>(a, s);
    const uint64_t rows = (uint64_t)a.batch * a.nq * a.heads;
    if (a.splits > 1) k_kv_join<T><<<(uint32_t)((rows + 3) / 4), 256, 0, s>>>(a.part, a.stats, a.out, rows, a.splits, a.c.dim);
}

}  // namespace
}  // namespace serve
}  // namespace lc

using namespace lc::serve;

#define LC_BY_BITS(call, T, bits) do { if ((bits) == 8) call(T, 8); else call(T, 4); } while (0)
#define LC_BY_TYPE(call, dtype, bits) \
    do { if ((dtype) == LC_F32) LC_BY_BITS(call, LC_F32, bits); else if ((dtype) == LC_BF16) LC_BY_BITS(call, LC_BF16, bits); \
         else LC_BY_BITS(call, LC_F16, bits); } while (0)

extern "C" {

int lc_kv_write(const lc_kv_cache* cache, const void* k, const void* v, uint64_t ld_token, uint64_t ld_head, const int64_t* slots, uint64_t tokens, int dtype,
                void* stream) {
    if (!served_type(dtype) || bad(cache)) return LC_ERR_BADARG;
    if (tokens == 0) return LC_OK;
    if (bad_vectors(cache, k, v, ld_token, ld_head, slots, tokens, dtype)) return LC_ERR_BADARG;
    const Cache c = described(*cache);
    hipStream_t s = static_cast<hipStream_t>(stream);
#define CALL(T, B) write<T, B>(c, k, v, ld_token, ld_head, slots, tokens, s)
    LC_BY_TYPE(CALL, dtype, cache->bits);
#undef CALL
    return launched();
}

int lc_kv_read(const lc_kv_cache* cache, const int64_t* slots, uint64_t tokens, void* k, void* v, uint64_t ld_token, uint64_t ld_head, int dtype, void* stream) {
    if (!served_type(dtype) || bad(cache)) return LC_ERR_BADARG;
    if (tokens == 0) return LC_OK;
    if (bad_vectors(cache, k, v, ld_token, ld_head, slots, tokens, dtype)) return LC_ERR_BADARG;
    const Cache c = described(*cache);
    hipStream_t s = static_cast<hipStream_t>(stream);
#define CALL(T, B) read<T, B>(c, slots, tokens, k, v, ld_token, ld_head, s)
    LC_BY_TYPE(CALL, dtype, cache->bits);
#undef CALL
    return launched();
}

size_t lc_kv_workspace_bytes(uint64_t batch, int nq, int heads, int kv_heads, int dim) {
    if (batch > 65535 || nq < 1 || nq > 64 || kv_heads < 1 || kv_heads > 1024 || heads < kv_heads || heads % kv_heads || heads > 4096 || dim < 32 ||
        dim > 256 || dim % 32) return 0;
    const uint64_t splits = most_splits(batch, (uint32_t)nq, (uint32_t)heads, (uint32_t)kv_heads);
    return splits == 1 ? 256 : (size_t)((batch * nq * heads * splits * (dim + 2) * 4 + 255) / 256 * 256);
}

int lc_kv_attend(const lc_kv_cache* cache, const void* q, uint64_t batch, int nq, int heads, const int32_t* table, uint64_t ld_table, uint64_t table_pages,
                 const int32_t* lens, const uint64_t* mask, float scale, void* out, int dtype, void* ws, size_t ws_bytes, void* stream) {
    if (!served_type(dtype) || bad(cache) || batch > 65535) return LC_ERR_BADARG;
    const size_t need = lc_kv_workspace_bytes(batch, nq, heads, cache->heads, cache->dim);
    if (!need) return LC_ERR_BADARG;
    if (batch == 0) return LC_OK;
    if (!q || !out || !lens || off(q, 16) || off(out, 16) || off(lens, 4) || off(mask, 8) || (table_pages && (!table || off(table, 4))) ||
        ld_table > (1ull << 31) || table_pages > (1ull << 30) / cache->page_tokens || (batch > 1 && ld_table < table_pages)) return LC_ERR_BADARG;
    if (!ws || off(ws, 256) || ws_bytes < need) return LC_ERR_WORKSPACE;
    Attend a = {};
    a.c = described(*cache);
    a.q = q; a.table = table; a.ld_table = ld_table; a.table_pages = cache->pages ? table_pages : 0; a.lens = lens; a.mask = mask; a.out = out;
    a.scale = scale * kLog2e;
    a.batch = (uint32_t)batch; a.nq = (uint32_t)nq; a.heads = (uint32_t)heads; a.group = (uint32_t)(heads / cache->heads); a.rows = a.nq * a.group;
    a.pages = (int32_t)(cache->pages > 0x7fffffffull ? 0x7fffffff : cache->pages);
    // (splits by what the table has room for: the lengths are known on the device only)
    const uint64_t room = a.table_pages << a.c.page_shift, by_room = (room + kLeastTokens - 1) / kLeastTokens;
    uint64_t splits = most_splits(batch, a.nq, a.heads, a.c.heads);
    splits = by_room < splits ? (by_room ? by_room : 1) : splits;
    a.tiles = (uint32_t)((room + splits * kTile - 1) / (splits * kTile));
    a.splits = (uint32_t)splits;
    a.part = static_cast<float*>(ws);
    a.stats = a.part + batch * nq * heads * splits * a.c.dim;
    hipStream_t s = static_cast<hipStream_t>(stream);
#define CALL(T, B) attend<T, B>(a, s)
    LC_BY_TYPE(CALL, dtype, cache->bits);
#undef CALL
    return launched();
}

}  // extern "C"
