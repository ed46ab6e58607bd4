// A paged cache of keys and values in 8 or 4 bits: writing, reading back, and the attention over it (include/lc_serve.h).
#include "lc_serve.h"

#include <atomic>

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
// keys are the first half of the grid, the values the second.  s = max |x| / 127 (or 7) over the head in fp32, q = rint(x (1 / s)).  Bound by memory:
// 2000 tokens of 8 heads of 128 in fp16 to 4 bits 4.7 us, of which 2.3 are the launch; 30011 tokens read back, keys and values by the same lane,
// 26 to 29 us, 5.4 to 6 TB/s, past the caches.
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

template <int N> struct Bits;
template <> struct Bits<16> { typedef uint16_t Type; };
template <> struct Bits<32> { typedef uint32_t Type; };
template <> struct Bits<64> { typedef uint64_t Type; };
// A lane takes 16 bytes' worth of a token's head, keys and values alike.
template <int T, int BITS>
__global__ __launch_bounds__(256) void k_kv_read(Cache c, const int64_t* slots, void* k, void* v, uint64_t ld_token, uint64_t ld_head, uint32_t lanes,
                                                 FastDiv by_row, FastDiv by_heads) {
    const uint32_t lane = blockIdx.x * 256u + threadIdx.x;
    if (lane >= lanes) return;
    constexpr int N = kAtOnce<T>;
    const uint32_t item = by_row(lane), at = N * (lane - item * by_row.d);
    const uint32_t token = by_heads(item), head = item - token * c.heads;
    const int64_t slot = slots[token];
    float x[2][N] = {};
    if (slot >= 0 && (uint64_t)slot < c.slots) {
        typedef typename Bits<N * BITS>::Type Word;
        const uint64_t row = row_of(c, (uint64_t)slot >> c.page_shift, head, (uint32_t)slot & ((1u << c.page_shift) - 1)), from = row * c.row_bytes + at * BITS / 8;
        const float s[2] = {c.k_scale[row], c.v_scale[row]};
        const uint64_t w[2] = {*reinterpret_cast<const Word*>(c.k + from), *reinterpret_cast<const Word*>(c.v + from)};
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                x[n][e] = (BITS == 8 ? (float)(int8_t)(w[n] >> (8 * e)) : (float)((int)(w[n] >> (4 * e) & 15u) - 8)) * s[n];
                if (T == LC_F16) asm("" : "+v"(x[n][e]));    // (else product and conversion become one instruction, with one rounding for the two)
            }
    }
    store_some<T>(k, token * ld_token + head * ld_head + at, N, x[0]);
    store_some<T>(v, token * ld_token + head * ld_head + at, N, x[1]);
}

// ---------------------------------------------------------------- attention
// The rows that share a head of the cache are the nq * (heads / kv heads) queries of a sequence; a wavefront holds 16 of them (or 32, 64)
// and walks over its part of the sequence 32 tokens at a time, everything in registers:
//   S^T = K Q^T   rows of the matrix instruction are tokens, columns the queries: lane l gets query l % 16, tokens 4 (l / 16) + 0..3
//   O^T += V^T P^T   the same lane's probabilities are its part of the second operand as they stand, with the tokens
//                    in the order 4 h + 0..3, 16 + 4 h + 0..3, in which the values are then loaded too
// so the running maximum, the sum and the factors of the rescaling are one number a lane, and nothing passes through LDS.
// Scales of keys multiply the scores, scales of values the probabilities; codes enter the matrix instructions as whole numbers, exactly, and
// probabilities times scales as two bf16 parts (three for fp32), the first cut off and the last rounded to nearest: 2^-16 of each at most, either way.  One
// part alone, 2^-9 of each, would show beside a result in fp16; with the last one cut off as well results were 7e-6 too small on average.
// One token of 16 sequences of up to 4096 tokens of 32 heads (8 bits): 63 to 67 us, 4.4 to 4.7 TB/s of the cache, two thirds of the 7 that a bare read
// reaches (42 us); vector instructions half of its cycles; fp32 68.  The same in 4 bits 50 us (fp32 54), of 8 heads for 32 queries up to 16384 46 (59), where the
// bytes take 21.  Heads of 160, 192 and 256 (16 of them, 8 bits) 50, 55 and 67 us, in 4 bits 40,
// 43 and 44: all are worked on as 256.  24 drafted
// tokens of 5 sequences of up to 8191, 4 queries to a head (4 bits): 43 us for what memory would give in 4 to 6 and products at the rate of large ones in 8: each tile of
// 32 tokens by 32 queries takes 350 vector instructions, half of them to convert codes and half for the softmax, beside 48 of the matrix unit's (16% of the time), and
// three workgroups convert a head's codes each for its own rows; 8 bits 48 us, fp32 66 to 68.  One token of one sequence of 1000: 9 us, latencies in a row: launch 2.3,
// lengths, pages, tiles, and a meeting of the parts.
constexpr int kTile = 32, kWaves = 4;
constexpr float kFar = 8.0f;                                // by how much, in powers of two, a score may pass what probabilities are measured from
constexpr float kLog2e = 1.44269504088896340736f;
// A sequence whose heads and queries alone do not give the chip as many workgroups as fit it at once is split along its tokens, into as many parts at most as
// a wavefront has lanes to look at the parts' marks with, less a few.  (One sequence of 32768 tokens of one head, 8 queries: 60 workgroups, 24 us in 8 bits; of 8
// heads, 480 of them, 30 us.)
constexpr uint32_t kMostSplits = 60, kLeastTokens = kWaves * kTile;

struct Attend {
    Cache c;
    const void* q;
    const int32_t* table; uint64_t ld_table; uint64_t table_pages;
    const int32_t* lens;
    const uint64_t* mask;
    void* out;
    unsigned long long* marks;  // [head and group of rows][slot]: the call's number where that part is done
    float* stats;               // the maximum and the sum of each [slot][query][head]
    float* part;                // [slot][query][head][dim]
    unsigned long long call;
    float scale;                // times log2(e)
    uint32_t batch, nq, heads, group, rows;     // rows = nq * group of a head of the cache
    uint32_t slots;             // parts of all sequences together: batch of them if none is split
    int32_t pages;
    FastDiv by_group;
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
template <int BYTE> __device__ __forceinline__ float byte_of(uint32_t w) { return (float)(int8_t)(w >> (8 * BYTE)); }

// A bf16 operand of the values of eight tokens at element j of each token's `w` (4 bits: turned words, and sixteenths).
template <int BITS> __device__ __forceinline__ u32x4 values_at(const uint32_t (&w)[8], int j) {
    u32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a, b;
        if (BITS == 8) { a = (float)(int8_t)(w[2 * e] >> (8 * j)); b = (float)(int8_t)(w[2 * e + 1] >> (8 * j)); }
        else { a = low_nibble_of(w[2 * e], j); b = low_nibble_of(w[2 * e + 1], j); }
        r[e] = high_halves(bits_of(a), bits_of(b));
    }
    return r;
}

// Over the four lanes of a column (c, c + 16, c + 32, c + 48), in each of them: rows of sixteen lanes change places, without LDS.
__device__ __forceinline__ float max_over_quarters(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(bits_of(v), bits_of(v), false, false);
    v = fmaxf(float_of(a[0]), float_of(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(bits_of(v), bits_of(v), false, false);
    return fmaxf(float_of(b[0]), float_of(b[1]));
}
__device__ __forceinline__ float sum_over_quarters(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(bits_of(v), bits_of(v), false, false);
    v = float_of(a[0]) + float_of(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(bits_of(v), bits_of(v), false, false);
    return float_of(b[0]) + float_of(b[1]);
}
// Over all lanes, as a number that all of them share.
template <bool MAX> __device__ __forceinline__ uint32_t over_wave(uint32_t v) {
#define LC_DPP(ctrl) { const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, false); v = MAX ? (v > o ? v : o) : v + o; }
    LC_DPP(0xB1) LC_DPP(0x4E) LC_DPP(0x141) LC_DPP(0x140)
#undef LC_DPP
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = MAX ? (a[0] > a[1] ? a[0] : a[1]) : a[0] + a[1];
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = MAX ? (b[0] > b[1] ? b[0] : b[1]) : b[0] + b[1];
    return __builtin_amdgcn_readfirstlane(v);
}

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

// What passes between workgroups goes through agent-scope atomic operations, whose completion each waits for before it arrives: a fence
// would write back the L2 of a die from every workgroup (1000 tokens of 16 heads in 8 parts: 37 us with fences).
__device__ __forceinline__ void put_shared(float* p, float x, float y) {
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), (unsigned long long)bits_of(y) << 32 | bits_of(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 get_shared(const float* p) {
    const unsigned long long v = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return f32x2{float_of((uint32_t)v), float_of((uint32_t)(v >> 32))};
}

// Which part of which sequence a workgroup has: its slot, counted over the parts of all sequences.
struct Part { uint32_t b, index, count; int32_t len, first, end; };

// With as many slots as sequences each has one.  With more, all parts are of one length (the last of a sequence may be shorter): about the
// least that the slots suffice for, so that long sequences have more parts than short ones and no part waits for another to
// leave the chip.  The lengths are known on the device only; each wavefront works the division out for itself.
__device__ __forceinline__ int32_t length_of(const Attend& a, uint32_t b, int32_t room) {
    typedef const __attribute__((address_space(4))) int32_t* Uniform;
    const int32_t n = ((Uniform)(uintptr_t)a.lens)[b];
    return n < 0 ? 0 : n < room ? n : room;
}
__device__ __forceinline__ Part part_of(const Attend& a, uint32_t slot, uint32_t lane) {
    const int32_t room = (int32_t)(a.table_pages << a.c.page_shift);
    Part p = {slot, 0, 1, 0, 0, 0};
    if (a.slots == a.batch) {
        p.len = p.end = length_of(a, slot, room);
        return p;
    }
    // In units of kLeastTokens; lengths add up to less than 2^32 of them.
    auto units_of = [&](uint32_t i) {
        int32_t n = i < a.batch ? a.lens[i] : 0;
        n = n < 0 ? 0 : n < room ? n : room;
        return (uint32_t)(n + (int32_t)kLeastTokens - 1) / kLeastTokens;
    };
    uint32_t total = 0, longest = 0;
    for (uint32_t i = lane; i < a.batch; i += 64) {
        const uint32_t n = units_of(i);
        total += n;
        longest = n > longest ? n : longest;
    }
    total = over_wave<false>(total);
    longest = over_wave<true>(longest);
    uint32_t length = (total + a.slots - 1) / a.slots, least = (longest + kMostSplits - 1) / kMostSplits;
    length = length > least ? length : least;
    length = length ? length : 1;
    // Where all are short the meeting of the parts costs more than it saves.  (One sequence, split / not: 250 tokens of 8 heads of 128 11.3 / 9.8 us, 500
    // 11.6 / 11.7, 700 11.7 / 13.5; a tree of 24 over 300 18.2 / 14.6; 8 heads of 256 500 12.9 / 14.5.)
    if (longest <= (a.c.dim <= 128 ? 4 : 2)) length = longest ? longest : 1;
    for (; length < longest; length += 1 + length / 16) {   // (at the longest, if not before, each sequence has one part)
        uint32_t parts = 0;
        for (uint32_t i = lane; i < a.batch; i += 64) { const uint32_t n = units_of(i); parts += n ? (n + length - 1) / length : 1; }
        if (over_wave<false>(parts) <= a.slots) break;
    }
    uint32_t before = 0;
    p.count = 0;                                            // (none: a slot beyond the last part)
    for (uint32_t i0 = 0; i0 < a.batch; i0 += 64) {
        const uint32_t i = i0 + lane, n = units_of(i), own = i < a.batch ? (n ? (n + length - 1) / length : 1) : 0;
        uint32_t upto = own;
        if (a.batch > 1)
            for (int x = 1; x < 64; x *= 2) { const uint32_t o = __shfl_up(upto, x); if (lane >= (uint32_t)x) upto += o; }
        const unsigned long long mine = __ballot(before + upto > slot && before + upto - own <= slot);
        if (mine) {
            const int from = __builtin_ctzll(mine);
            p.b = i0 + from;
            p.count = __builtin_amdgcn_readfirstlane(__shfl(own, from));
            p.index = slot - (before + __builtin_amdgcn_readfirstlane(__shfl(upto, from)) - p.count);
            p.len = length_of(a, p.b, room);
            p.first = (int32_t)(p.index * length * kLeastTokens);
            const uint64_t end = (uint64_t)(p.index + 1) * length * kLeastTokens;
            p.end = end < (uint64_t)p.len ? (int32_t)end : p.len;
            break;
        }
        before += __builtin_amdgcn_readfirstlane(__shfl(upto, 63));
    }
    p.first = __builtin_amdgcn_readfirstlane(p.first);
    p.end = __builtin_amdgcn_readfirstlane(p.end);
    return p;
}

template <int T, int BITS, int DP, int NT, int DEEP, int PERSIMD>
__global__ __launch_bounds__(kWaves * 64, PERSIMD) void k_kv_attend(Attend a) {
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
    // Workgroups go round the eight dies, each with an L2 of its own: those that have different rows of one head follow each other by eights.  (24 drafted
    // tokens as above 45.2 us for 46.2, with 37 MB from beyond the L2s instead of 90.)
    const uint32_t row_groups = (a.rows + 16 * NT - 1) / (16 * NT), by_dies = a.c.heads / 8 * 8 * row_groups;
    const uint32_t x = blockIdx.x < by_dies ? blockIdx.x / 8 : blockIdx.x, over = x / row_groups;
    const uint32_t head = blockIdx.x < by_dies ? over * 8 + blockIdx.x % 8 : over, row0 = (x - over * row_groups) * 16 * NT;
    const uint32_t slot = blockIdx.y;
    const Part part = part_of(a, slot, lane);
    if (part.count == 0) return;
    const uint32_t b = part.b;
    const int32_t len = part.len, first = part.first, end = part.end, base = len - (int32_t)a.nq;      // base: the first drafted token
    // (What all lanes read alike is read by the scalar unit, which counts its loads apart: a vector load of it, waited for, would wait for
    // the keys and values asked for before it as well.)
    typedef const __attribute__((address_space(4))) int32_t* Uniform;
    const Uniform table = (Uniform)(uintptr_t)(a.table + b * a.ld_table);
    const int32_t own = first + (int32_t)wave * kTile;      // this wavefront's first tile; every kWaves-th is its own
    const int32_t tiles = own < end ? (end - own + kWaves * kTile - 1) / (kWaves * kTile) : 0;

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
    auto load_keys = [&](Raw& f, const Eights& e) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint64_t k0 = e.row[2 * s] * a.c.row_bytes, k1 = e.row[2 * s + 1] * a.c.row_bytes;
            const uint8_t* keys = a.c.k + (c < 8 ? k0 : k1);
#pragma unroll
            for (int l = 0; l < Raw::kKeyLoads; ++l) __builtin_memcpy(f.key[s][l], __builtin_assume_aligned(keys + key_off[l], Raw::kKey), Raw::kKey);
        }
    };
    auto load_values = [&](Raw& f, const Eights& e) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint64_t k0 = e.row[2 * s] * a.c.row_bytes, k1 = e.row[2 * s + 1] * a.c.row_bytes;
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
    Raw raw[DEEP];                                          // the tiles under way
    Eights places[DEEP] = {};
    if (tiles > 0) {
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            places[d] = find(d);
            load_keys(raw[d], places[d]);
            load_values(raw[d], places[d]);
        }
    }

    // this lane's queries, eight elements an operand at the places at which the keys' codes lie
    u32x4 q[NT][KOPS][NQ];
    f32x4 less[NT];                                         // -24 times each query's sum
    uint64_t mask[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint32_t row = row0 + 16 * n + c;
        const bool has_row = row < a.rows;
        const uint32_t qi = a.by_group(has_row ? row : 0), qg = (has_row ? row : 0) - qi * a.group;
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
            // An infinity is taken as NaN: the score of whatever is seen is infinite or NaN, so the softmax of any set of them is NaN, and scores that are
            // all minus infinity would look like those of what is not seen.
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += v[e] - v[e];
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

    f32x4 acc[NT][VD];
    float top[NT], from[NT], sum[NT];                       // the largest score so far (or about that), what probabilities are measured from, their sum
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        top[n] = -__builtin_inff();
        from[n] = sum[n] = 0;
#pragma unroll
        for (int j = 0; j < VD; ++j) acc[n][j] = f32x4{0, 0, 0, 0};
    }
    // Keys are spent once the scores are there, values once they are added up: then those of the DEEP-th tile behind are asked for, into the
    // same registers.
    auto use = [&](Raw& f, Eights& at, int32_t i) {
        const int32_t tb = own + i * kWaves * kTile;
        const Eights next = find(i + DEEP);
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
        load_keys(f, next);
        float ks[8], vs[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            ks[i] = f.key_scale[i / 4][i % 4] * (BITS == 4 && !LIFTED ? 16.0f * a.scale : a.scale);
            vs[i] = f.value_scale[i / 4][i % 4];
        }
        const bool whole = tb + kTile <= base && tb + kTile <= end && at.there == 15;      // all of the tile is seen by all
        u32x4 pp[NT][NP];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float p[8], weight[8];                           // scores less what probabilities are measured from, then probabilities
#pragma unroll
            for (int i = 0; i < 8; ++i) { p[i] = fmaf(score[n][i / 4][i % 4], ks[i], -from[n]); weight[i] = vs[i]; }
            if (!whole) {                                    // (what is not seen may have any scale)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int32_t t = tb + 16 * (i / 4) + 4 * h + i % 4, j = t - base;
                    const bool there = at.there >> (2 * (i / 4) + h / 2) & 1, seen = there && t < end && (j < 0 || (mask[n] >> (j & 63) & 1));
                    p[i] = seen ? p[i] : -__builtin_inff();
                    weight[i] = seen ? weight[i] : 0.0f;
                }
            }
            // What probabilities are measured from moves only when one would pass 2^8, so that the sums are seldom rescaled.
            float most = fmaxf(fmaxf(fmaxf(p[0], p[1]), p[2]), fmaxf(fmaxf(fmaxf(p[3], p[4]), p[5]), fmaxf(p[6], p[7])));
            if (__any(most > kFar || top[n] == -__builtin_inff())) {
                most = fmaxf(max_over_quarters(most) + from[n], top[n]);
                const float then = most == -__builtin_inff() ? 0.0f : most, shrink = __builtin_amdgcn_exp2f(top[n] - then);
                sum[n] *= shrink;
#pragma unroll
                for (int j = 0; j < VD; ++j) acc[n][j] *= shrink;
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] -= then - from[n];
                top[n] = most;
                from[n] = then;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = __builtin_amdgcn_exp2f(p[i]);
                sum[n] += p[i];
                p[i] *= weight[i];
            }
#pragma unroll
            for (int k = 0; k < NP; ++k) {
#pragma unroll
                for (int i = 0; i < 4; ++i) pp[n][k][i] = k == NP - 1 ? rounded_halves(p[2 * i], p[2 * i + 1]) : high_halves(bits_of(p[2 * i]), bits_of(p[2 * i + 1]));
                if (k < NP - 1)
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
            for (int half = 0; half < (BITS == 4 ? 2 : 1); ++half) {
                if (half)
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = upper_nibbles(w[i]);
#pragma unroll
                for (int j = 0; j < Raw::kPerWord * BITS / 8; ++j) {
                    const u32x4 v = values_at<BITS>(w, j);
                    const int at = o * Raw::kPerWord + (BITS == 4 ? 2 * j + half : j);
#pragma unroll
                    for (int k = NP - 1; k >= 0; --k)
#pragma unroll
                        for (int n = 0; n < NT; ++n) acc[n][at] = mfma_bf16(v, pp[n][k], acc[n][at]);
                }
            }
        }
        load_values(f, next);
        at = next;
    };
    for (int32_t i = 0; i < tiles; i += DEEP)
#pragma unroll
        for (int d = 0; d < DEEP; ++d)
            if (i + d < tiles) use(raw[d], places[d], i + d);

    // The wavefronts' parts, joined: lane (c, h) holds elements VD (4 h + r) + j of query c.
    const uint64_t heads_of = (uint64_t)a.nq * a.heads;
    auto place = [&](uint32_t row) {                        // of a row of this head, among a sequence's queries and heads
        const uint32_t i = a.by_group(row), g = row - i * a.group;
        return (uint64_t)i * a.heads + head * a.group + g;
    };
    const uint32_t quads = a.c.dim / 4;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (n) __syncthreads();
        const float total = sum_over_quarters(sum[n]);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < VD; j += 4) {
                f32x4 v = {acc[n][j][r], acc[n][j + 1][r], acc[n][j + 2][r], acc[n][j + 3][r]};
                if (BITS == 4) v *= 16.0f;
                *reinterpret_cast<f32x4*>(&so[wave][c][VD * (4 * h + r) + j]) = v;
            }
        if (h == 0) { sm[wave][c] = top[n]; sl[wave][c] = total; }
        __syncthreads();
        if (threadIdx.x < 16) {
            const uint32_t r = threadIdx.x;
            float m = sm[0][r], l = 0, f[kWaves];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) m = fmaxf(m, sm[w][r]);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                f[w] = sl[w][r] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(sm[w][r] - m);      // (where a sum is not zero the maximum is a number, or all is NaN)
                l += sl[w][r] == 0.0f ? 0.0f : f[w] * sl[w][r];
            }
            if (part.count > 1 && row0 + 16 * n + r < a.rows) {
                put_shared(a.stats + 2 * (slot * heads_of + place(row0 + 16 * n + r)), m, l);
            }
            const float whole = part.count > 1 || l == 0.0f ? 1.0f : 1.0f / l;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) sm[w][r] = f[w] * whole;
        }
        __syncthreads();
        for (uint32_t e = threadIdx.x; e < 16 * quads; e += kWaves * 64) {
            const uint32_t r = e / quads, d = 4 * (e - r * quads), row = row0 + 16 * n + r;
            if (row >= a.rows) break;
            f32x4 o = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float f = sm[w][r];
                const f32x4 v = *reinterpret_cast<const f32x4*>(&so[w][r][d]);
                if (f != 0.0f)
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[k] = fmaf(f, v[k], o[k]);
            }
            if (part.count == 1) store_four<T>(a.out, (b * heads_of + place(row)) * a.c.dim + d, o);
            else {
                float* to = a.part + (slot * heads_of + place(row)) * a.c.dim + d;
                put_shared(to, o[0], o[1]);
                put_shared(to + 2, o[2], o[3]);
            }
        }
    }
    if (part.count == 1) return;

    // The last workgroup of a sequence's parts to get here joins them: each marks its part done with the call's number, once what it has
    // written has arrived, and then looks at the marks of all.  Whoever marks last finds them all there; should two find that, both
    // write the same.  Marks are taken back, so that the same call replayed from a graph begins without them; what was there before the
    // call does not matter.
    __shared__ uint32_t is_last;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (wave == 0) {
        unsigned long long* marks = a.marks + (uint64_t)blockIdx.x * a.slots + slot - part.index;
        if (lane == 0) __hip_atomic_store(marks + part.index, a.call, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const bool done = lane >= part.count || __hip_atomic_load(marks + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.call;
        const bool all = __all(done);
        if (lane == 0) is_last = all;
        if (all && lane < part.count) __hip_atomic_store(marks + lane, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!is_last) return;
    f32x2 (*stat)[kMostSplits] = reinterpret_cast<f32x2 (*)[kMostSplits]>(&so[0][0][0]);
    static_assert(sizeof(so) >= 16 * NT * kMostSplits * sizeof(f32x2), "room for every row and part");
    static_assert(kMostSplits <= 64, "a lane a part");
    const uint64_t slot0 = slot - part.index;
    const uint32_t rows_here = a.rows - row0 < 16 * NT ? a.rows - row0 : 16 * NT;
    for (uint32_t e = threadIdx.x; e < rows_here * part.count; e += kWaves * 64) {
        const uint32_t k = e / rows_here, r = e - k * rows_here;
        stat[r][k] = get_shared(a.stats + 2 * ((slot0 + k) * heads_of + place(row0 + r)));
    }
    __syncthreads();
    if (threadIdx.x < rows_here) {
        const uint32_t r = threadIdx.x;
        float m = -__builtin_inff(), l = 0;
        for (uint32_t k = 0; k < part.count; ++k) m = fmaxf(m, stat[r][k][0]);
        for (uint32_t k = 0; k < part.count; ++k) {
            const float sum_k = stat[r][k][1], f = sum_k == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(stat[r][k][0] - m);
            stat[r][k][0] = f;
            l += sum_k == 0.0f ? 0.0f : f * sum_k;
        }
        const float whole = l == 0.0f ? 1.0f : 1.0f / l;
        for (uint32_t k = 0; k < part.count; ++k) stat[r][k][0] *= whole;
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < rows_here * quads; e += kWaves * 64) {
        const uint32_t r = e / quads, d = 4 * (e - r * quads);
        const float* from = a.part + (slot0 * heads_of + place(row0 + r)) * a.c.dim + d;
        f32x4 o = {0, 0, 0, 0};
        for (uint32_t k0 = 0; k0 < part.count; k0 += 8) {                // (the last part again beyond the last: eight loads under way at once)
            f32x2 v[8][2];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float* at = from + (k0 + k < part.count ? k0 + k : part.count - 1) * heads_of * a.c.dim;
                v[k][0] = get_shared(at);
                v[k][1] = get_shared(at + 2);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float f = k0 + k < part.count ? stat[r][k0 + k][0] : 0.0f;
                if (f != 0.0f) o = f32x4{fmaf(f, v[k][0][0], o[0]), fmaf(f, v[k][0][1], o[1]), fmaf(f, v[k][1][0], o[2]), fmaf(f, v[k][1][1], o[3])};
            }
        }
        store_four<T>(a.out, (b * heads_of + place(row0 + r)) * a.c.dim + d, o);
    }
}

// Slots for the parts of all sequences: one a sequence, or as many more as all fit the chip together.
uint64_t slots_of(uint64_t batch, uint32_t kv_heads, uint64_t row_groups, uint32_t want) {
    const uint64_t blocks = kv_heads * row_groups;
    const uint64_t slots = batch * blocks >= want ? batch : want / blocks;
    return slots < batch * kMostSplits ? slots : batch * kMostSplits;
}
struct Scratch { uint64_t stats, part, bytes; };            // where the parts of the scratch memory begin
Scratch scratch_of(uint64_t batch, uint64_t slots, uint64_t groups, uint64_t nq, uint64_t heads, uint64_t dim) {
    if (slots == batch) return {0, 0, 256};
    Scratch s;
    s.stats = (slots * groups * 8 + 255) / 256 * 256;
    s.part = s.stats + (slots * nq * heads * 8 + 255) / 256 * 256;
    s.bytes = (s.part + slots * nq * heads * dim * 4 + 255) / 256 * 256;
    return s;
}
int tiles_of_rows(uint64_t rows, int dim, int dtype) { return rows > 16 && dtype != LC_F32 && dim <= 128 ? 2 : 1; }
// How many workgroups: two a compute unit, which is what most kernels' registers leave room for; three for one tile of rows of 4-bit codes, where that
// pays (one token of 16 sequences of up to 16384 of 8 heads of 128 47.0 us for 50.5, of 40 of up to 2000 of 2 heads of 96 16.1 for 15.6; one over 32000 of
// 16 heads of 64 25.0 for 22.9).
uint32_t workgroups_of(int bits, int dim, int dtype, int tiles) { return bits == 4 && dim > 64 && dim <= 128 && dtype != LC_F32 && tiles == 1 ? 768 : 512; }

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
    const uint64_t step = (1ull << 24) / c.heads;
    for (uint64_t t = 0; t < tokens; t += step) {
        const uint32_t lanes = (uint32_t)((tokens - t < step ? tokens - t : step) * c.heads * (c.dim / kAtOnce<T>));
        const uint64_t by = t * ld_token * (T == LC_F32 ? 4 : 2);
        k_kv_read<T, BITS><<<(lanes + 255) / 256, 256, 0, s>>>(c, slots + t, static_cast<uint8_t*>(k) + by, static_cast<uint8_t*>(v) + by, ld_token,
                                                                        ld_head, lanes, FastDiv(c.dim / kAtOnce<T>), FastDiv(c.heads));
    }
}
template <int T, int BITS, int DP, int NT, int DEEP, int PERSIMD>
void attend_of(const Attend& a, hipStream_t s) {
    k_kv_attend<T, BITS, DP, NT, DEEP, PERSIMD><<<dim3(a.c.heads * ((a.rows + 16 * NT - 1) / (16 * NT)), a.slots), kWaves * 64, 0, s>>>(a);
}
template <int T, int BITS>
void attend(const Attend& a, hipStream_t s) {
    // Two tiles of 16 rows a wavefront where there are more rows than one: codes are converted once for both (24 drafted tokens as above 46 us
    // for 59, in 8 bits 50 for 68, 64 tokens of 4 queries to a head of 64 over 20000 49 for 63).  Two tiles of tokens under way where the registers of
    // two wavefronts a SIMD hold them: not for 8 bits and two tiles of rows (49 us either way), nor from 129 elements on.
    if constexpr (T != LC_F32)
        if (tiles_of_rows(a.rows, (int)a.c.dim, T) == 2) {
            if (a.c.dim <= 64) attend_of<T, BITS, 64, 2, 2, 2>(a, s);
            else attend_of<T, BITS, 128, 2, BITS == 8 ? 1 : 2, 2>(a, s);
            return;
        }
    if (a.c.dim <= 64) attend_of<T, BITS, 64, 1, 2, 3>(a, s);
    else if (a.c.dim <= 128) attend_of<T, BITS, 128, 1, 2, BITS == 4 && T != LC_F32 ? 3 : 2>(a, s);
    else attend_of<T, BITS, 256, 1, 1, 1>(a, s);
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
    uint64_t most = 0;                                      // (of the ways the rows may be grouped and split, whatever the type)
    for (int tiles = 1; tiles <= 2; ++tiles) {
        const uint64_t rows = (uint64_t)nq * (heads / kv_heads), groups = (rows + 16 * tiles - 1) / (16 * tiles);
        for (int bits = 4; bits <= 8; bits += 4) {
            const uint64_t slots = slots_of(batch, (uint32_t)kv_heads, groups, workgroups_of(bits, dim, LC_BF16, tiles));
            const uint64_t bytes = scratch_of(batch, slots, kv_heads * groups, nq, heads, dim).bytes;
            most = bytes > most ? bytes : most;
        }
    }
    return (size_t)most;
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
    a.by_group = FastDiv(a.group);
    a.pages = (int32_t)(cache->pages > 0x7fffffffull ? 0x7fffffff : cache->pages);
    const int tiles = tiles_of_rows(a.rows, cache->dim, dtype);
    const uint64_t groups = (a.rows + 16 * tiles - 1) / (16 * tiles);
    a.slots = (uint32_t)slots_of(batch, a.c.heads, groups, workgroups_of(cache->bits, cache->dim, dtype, tiles));
    if ((a.table_pages << a.c.page_shift) <= kLeastTokens) a.slots = a.batch;      // (nothing to split)
    const Scratch at = scratch_of(batch, a.slots, a.c.heads * groups, nq, heads, a.c.dim);
    a.marks = static_cast<unsigned long long*>(ws);
    a.stats = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + at.stats);
    a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + at.part);
    static std::atomic<unsigned long long> calls{0x5bd1e995};
    a.call = calls.fetch_add(1, std::memory_order_relaxed) * 0x9E3779B97F4A7C15ull | 1;      // (one to one on 63 bits, and never zero)
    hipStream_t s = static_cast<hipStream_t>(stream);
#define CALL(T, B) attend<T, B>(a, s)
    LC_BY_TYPE(CALL, dtype, cache->bits);
#undef CALL
    return launched();
}

}  // extern "C"
