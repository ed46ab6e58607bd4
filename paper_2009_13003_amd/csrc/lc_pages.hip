// The pages of a paged cache, given to sequences and taken back on the device, and where their new tokens go (include/lc_serve.h).
#include "lc_serve.h"

namespace lc {
namespace serve {
namespace {

struct Pages {
    int32_t* table; uint64_t ld_table, table_pages;
    const int32_t* lens;
    int32_t* free_pages;
    const int32_t* free_count;
    uint64_t free_room;
    uint32_t batch, shift;
};
// What is known of a sequence once its place among the others is.
struct Turn { uint64_t rank, start; int32_t len, add; };    // pages and tokens of the sequences before it; its own, cached and new

constexpr uint32_t kHere = 4096;                            // new tokens at most whose places the workgroup that gives pages out writes itself

__device__ __forceinline__ uint64_t pages_of(uint64_t tokens, uint32_t shift) { return (tokens + (1u << shift) - 1) >> shift; }

// The sums over all lanes before this one, and those of all, of two numbers a lane.  Two meetings.
template <uint32_t TURN> __device__ __forceinline__ void sums_before(uint64_t& a, uint64_t& b, uint64_t (*room)[2], uint64_t& all_a, uint64_t& all_b) {
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint64_t x = a, y = b;
    for (int d = 1; d < 64; d *= 2) {
        const uint64_t o = __shfl_up(x, d), p = __shfl_up(y, d);
        if (lane >= (uint32_t)d) { x += o; y += p; }
    }
    __syncthreads();
    if (lane == 63) { room[wave][0] = x; room[wave][1] = y; }
    __syncthreads();
    uint64_t before_a = 0, before_b = 0;
    all_a = all_b = 0;
    for (uint32_t w = 0; w < TURN / 64; ++w) {
        if (w < wave) { before_a += room[w][0]; before_b += room[w][1]; }
        all_a += room[w][0];
        all_b += room[w][1];
    }
    a = before_a + x - a;
    b = before_b + y - b;
}

__device__ __forceinline__ int32_t held_count(const Pages& p) {
    const int32_t n = p.free_count[0];
    return n < 0 ? 0 : (uint64_t)n > p.free_room ? (int32_t)p.free_room : n;
}

// The last of `count` turns whose number is at most n.
template <uint64_t Turn::*FIELD> __device__ __forceinline__ uint32_t turn_of(const Turn* turns, uint32_t count, uint64_t n) {
    uint32_t lo = 0, hi = count;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (turns[mid].*FIELD <= n) lo = mid; else hi = mid;
    }
    return lo;
}

// One workgroup, as many sequences at a time as it has lanes: sums of pages and tokens over those before give each its pages on the stack and its first token's number, and the
// first that does not fit ends the giving out.  Then a lane a page, and of few tokens a lane a token, whose sequences it finds by halving, so that each of the two takes
// one wait for the stack however pages and tokens are shared out.  Latencies in a row bound it: the loads of the lengths, two meetings, the stack's entries (48 tokens 3.6 us, of which
// a launch is 2.3; 300 prompts, 4000 pages, 6.6, and their 40000 slots 3 to 4 in a launch of their own; a wavefront a sequence took 6.0 and 10.9).  Everything is
// read before the meetings that anything is written behind, so lengths and count may be written where they are read.
template <uint32_t TURN>
__global__ __launch_bounds__(TURN) void k_kv_extend(Pages p, const int32_t* add, uint64_t room, int32_t* new_lens, int32_t* new_count, int32_t* starts,
                                                    int64_t* slots, int32_t* places, int32_t* owners, uint32_t here) {
    __shared__ uint64_t sums[TURN / 64][2];
    __shared__ uint32_t first_out[2];
    __shared__ Turn turns[TURN];
    const uint64_t count = (uint64_t)held_count(p);
    uint64_t rank = 0, start = 0;                           // of the first sequence of the turn
    uint32_t over = 0xffffffffu;                            // the first that did not fit
    for (uint32_t b0 = 0, turn = 0; b0 < p.batch; b0 += TURN, ++turn) {
        const uint32_t b = b0 + threadIdx.x;
        const bool in = b < p.batch;
        const int32_t was = in ? p.lens[b] : 0, len = was < 0 ? 0 : was;
        int32_t more = in ? add[b] : 0;
        more = more < 0 ? 0 : more;
        const uint64_t have = pages_of(len, p.shift), want = pages_of((uint64_t)len + more, p.shift);
        uint64_t r = more ? want - have : 0, s = more, all_r, all_s;
        const uint64_t need = r;
        if (threadIdx.x == 0) first_out[turn % 2] = 0xffffffffu;
        sums_before<TURN>(r, s, sums, all_r, all_s);
        const bool fits = more == 0 || (rank + r + need <= count && start + s + more <= room && want <= p.table_pages);
        if (!fits) atomicMin(&first_out[turn % 2], b);
        __syncthreads();
        over = over < first_out[turn % 2] ? over : first_out[turn % 2];
        if (b >= over) more = 0;
        turns[threadIdx.x] = {rank + r, start + s, len, more};
        __syncthreads();
        const uint32_t turns_here = p.batch - b0 < TURN ? p.batch - b0 : TURN;
        uint32_t given = turns_here;                        // sequences of this turn before the end of the giving out
        uint64_t end = start + all_s, pages = rank + all_r;
        if (over < b0 + turns_here) {                       // (behind it sums stand still)
            given = over < b0 ? 0 : over - b0;
            end = over < b0 ? start : turns[given].start;
            pages = over < b0 ? rank : turns[given].rank;
        }
        if (in) {
            starts[b] = (int32_t)(start + s < end ? start + s : end);
            new_lens[b] = more ? len + more : was;
        }
        if (given) {
            for (uint64_t n = rank + threadIdx.x; n < pages; n += TURN) {
                const uint32_t i = turn_of<&Turn::rank>(turns, given, n);
                p.table[(b0 + i) * p.ld_table + pages_of(turns[i].len, p.shift) + (n - turns[i].rank)] = p.free_pages[count - 1 - n];
            }
            if (here)
                for (uint64_t n = start + threadIdx.x; n < end; n += TURN) {
                    const uint32_t i = turn_of<&Turn::start>(turns, given, n);
                    const Turn t = turns[i];
                    const uint64_t place = (uint64_t)t.len + (n - t.start), j = place >> p.shift, had = pages_of(t.len, p.shift);
                    const int64_t page = j < had ? p.table[(b0 + i) * p.ld_table + j] : p.free_pages[count - 1 - t.rank - (j - had)];
                    slots[n] = page * (1 << p.shift) + (int64_t)(place & ((1u << p.shift) - 1));
                    if (places) places[n] = (int32_t)place;
                    if (owners) owners[n] = (int32_t)(b0 + i);
                }
        }
        rank = pages;
        start = end;
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        starts[p.batch] = (int32_t)start;
        new_count[0] = (int32_t)(count - rank);
    }
    if (here)
        for (uint64_t t = start + threadIdx.x; t < room; t += TURN) {
            slots[t] = -1;
            if (places) places[t] = -1;
            if (owners) owners[t] = -1;
        }
}

// Where each of many new tokens goes, a lane a token, from what k_kv_extend left: its sequence by halving.
__global__ __launch_bounds__(256) void k_kv_slots(Pages p, const int32_t* new_lens, const int32_t* starts, uint64_t room, int64_t* slots, int32_t* places,
                                                  int32_t* owners) {
    const uint64_t t = blockIdx.x * 256ull + threadIdx.x;
    if (t >= room) return;
    int64_t slot = -1;
    int32_t place = -1, owner = -1;
    if (t < (uint64_t)starts[p.batch]) {
        uint32_t lo = 0, hi = p.batch;                      // the last sequence that begins at t or before
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if ((uint64_t)starts[mid] <= t) lo = mid; else hi = mid;
        }
        owner = (int32_t)lo;
        place = new_lens[lo] - (starts[lo + 1] - (int32_t)t);
        slot = (int64_t)p.table[lo * p.ld_table + ((uint32_t)place >> p.shift)] * (1 << p.shift) + (place & ((1 << p.shift) - 1));
    }
    slots[t] = slot;
    if (places) places[t] = place;
    if (owners) owners[t] = owner;
}

// Pages behind what is kept go back, the last one of the last sequence first: sums over the sequences before give each its place, counted from the end of
// what comes back, which takes a walk over all of them first where they are more than the workgroup has lanes.
template <uint32_t TURN>
__global__ __launch_bounds__(TURN) void k_kv_trim(Pages p, const int32_t* keep, int32_t* new_lens, int32_t* new_count) {
    __shared__ uint64_t sums[TURN / 64][2];
    __shared__ Turn turns[TURN];
    const uint64_t count = (uint64_t)held_count(p);
    uint64_t back = 0;                                      // pages that come back, all together
    auto seen = [&](uint32_t b, int32_t& len, int32_t& kept) {
        len = b < p.batch ? p.lens[b] : 0;
        const uint64_t most = p.table_pages << p.shift;
        len = len < 0 ? 0 : (uint64_t)len > most ? (int32_t)most : len;
        kept = b < p.batch ? keep[b] : 0;
        kept = kept < 0 ? 0 : kept > len ? len : kept;
        return pages_of(len, p.shift) - pages_of(kept, p.shift);
    };
    if (p.batch > TURN)
        for (uint32_t b0 = 0; b0 < p.batch; b0 += TURN) {
            int32_t len, kept;
            uint64_t r = seen(b0 + threadIdx.x, len, kept), none = 0, all, x;
            sums_before<TURN>(r, none, sums, all, x);
            back += all;
        }
    uint64_t rank = 0;
    for (uint32_t b0 = 0; b0 < p.batch; b0 += TURN) {
        const uint32_t b = b0 + threadIdx.x;
        int32_t len, kept;
        uint64_t r = seen(b, len, kept), none = 0, all, x;
        sums_before<TURN>(r, none, sums, all, x);
        if (p.batch <= TURN) back = all;
        turns[threadIdx.x] = {rank + r, 0, len, kept};
        __syncthreads();
        if (b < p.batch) new_lens[b] = kept;
        const uint32_t turns_here = p.batch - b0 < TURN ? p.batch - b0 : TURN;
        for (uint64_t n = rank + threadIdx.x; n < rank + all; n += TURN) {
            const uint32_t i = turn_of<&Turn::rank>(turns, turns_here, n);
            const uint64_t at = count + back - 1 - n;
            if (at < p.free_room) p.free_pages[at] = p.table[(b0 + i) * p.ld_table + pages_of(turns[i].add, p.shift) + (n - turns[i].rank)];
        }
        rank += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) new_count[0] = (int32_t)(count + back < p.free_room ? count + back : p.free_room);
}

bool bad(const lc_kv_pages* p) {
    if (!p || p->batch > 65535 || p->page_tokens < 8 || p->page_tokens > 1024 || (p->page_tokens & (p->page_tokens - 1))) return true;
    if (p->table_pages > (1ull << 30) / p->page_tokens || p->free_room > 0x7fffffffull || p->ld_table > (1ull << 31)) return true;
    if (!p->free_count || off(p->free_count, 4) || (p->free_room && (!p->free_pages || off(p->free_pages, 4)))) return true;
    if (p->batch == 0) return false;
    return !p->lens || off(p->lens, 4) || (p->table_pages && (!p->table || off(p->table, 4))) || (p->batch > 1 && p->ld_table < p->table_pages);
}
Pages described(const lc_kv_pages& p) {
    return {p.table, p.ld_table, p.table_pages, p.lens, p.free_pages, p.free_count, p.free_room, (uint32_t)p.batch, (uint32_t)__builtin_ctz((unsigned)p.page_tokens)};
}

}  // namespace
}  // namespace serve
}  // namespace lc

using namespace lc::serve;

extern "C" {

int lc_kv_extend(const lc_kv_pages* pages, const int32_t* add, uint64_t room, int32_t* new_lens, int32_t* new_count, int32_t* starts, int64_t* slots,
                 int32_t* places, int32_t* owners, void* stream) {
    if (bad(pages) || room > 0x7fffffffull || !new_count || !starts || off(new_count, 4) || off(starts, 4)) return LC_ERR_BADARG;
    if ((pages->batch && (!add || !new_lens || off(add, 4) || off(new_lens, 4))) || (room && (!slots || off(slots, 8))) || off(places, 4) || off(owners, 4))
        return LC_ERR_BADARG;
    const Pages p = described(*pages);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool here = room <= kHere;
    // (48 sequences of a token each 3.5 us with 256 lanes, 6.0 with 1024; 300 prompts, whose many pages take turns, 6.6 with 1024.)
    if (p.batch <= 256 && room <= 1024) k_kv_extend<256><<<1, 256, 0, s>>>(p, add, room, new_lens, new_count, starts, slots, places, owners, here);
    else k_kv_extend<1024><<<1, 1024, 0, s>>>(p, add, room, new_lens, new_count, starts, slots, places, owners, here);
    if (!here) k_kv_slots<<<(uint32_t)((room + 255) / 256), 256, 0, s>>>(p, new_lens, starts, room, slots, places, owners);
    return launched();
}

int lc_kv_trim(const lc_kv_pages* pages, const int32_t* keep, int32_t* new_lens, int32_t* new_count, void* stream) {
    if (bad(pages) || !new_count || off(new_count, 4) || (pages->batch && (!keep || !new_lens || off(keep, 4) || off(new_lens, 4)))) return LC_ERR_BADARG;
    const Pages p = described(*pages);
    hipStream_t s = static_cast<hipStream_t>(stream);
    k_kv_trim<1024><<<1, 1024, 0, s>>>(p, keep, new_lens, new_count);
    return launched();
}

}  // extern "C"
