// Drafted tokens judged against the model's probabilities, and the token behind them drawn (include/lc_serve.h).
#include "lc_serve.h"

#include <atomic>

namespace lc {
namespace serve {
namespace {

// The path hangs on a few probabilities, which every workgroup of a sequence looks up for itself, a lane a node; what is read at length is the row behind its
// end, once for the sums and, the slice in which the drawn token lies, once more.  A sequence's row is dealt to up to 64 workgroups in slices; each leaves its slice's
// sum and a mark, and the one that finds all marks there finds the slice and, in it, the token.  Sums are held in 64 bits: products of two 32-bit
// numbers and differences of probabilities are exact in them or nearly, and which token is drawn must not hang on the order of a sum.
// One sequence of 5 nodes over 32000 tokens: 10 us, waits in a row: launch 2.3, tokens, their probabilities, the row, the meeting, the slice again.  48 sequences of 9 over 50257: 18 us
// for 19 MB, which a bare read takes 2.7 for: the same waits, longer, since each is the first look at another page of memory.  (Two sums, of p as well: 19.4; slices twice as long: 19.0.)
constexpr uint32_t kMostSlices = 64, kThreads = 256, kEach = 8, kStep = kThreads * kEach;      // elements a lane takes, and a workgroup at once

struct Draft {
    const void* target; uint64_t ld_batch, ld_row;
    const void* draft; uint64_t ld_draft_batch, ld_draft_row;
    const int32_t *tokens, *parent, *count;
    const float* uniform;
    int32_t *path, *length, *next;
    unsigned long long* marks;  // [batch][slices]
    double* sums;               // [batch][slices], of what is left
    unsigned long long call;
    uint32_t nodes, vocab, slices, slice;       // slice: elements of each, a multiple of kStep
};

__device__ __forceinline__ double weight(float p) { return p > 0.0f && p < __builtin_inff() ? (double)p : 0.0; }

__device__ __forceinline__ double get_shared(const double* p) {
    return __builtin_bit_cast(double, __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
__device__ __forceinline__ void put_shared(double* p, double v) {
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), __builtin_bit_cast(unsigned long long, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// Lane i's number, the same i in all lanes, without a way through LDS.
__device__ __forceinline__ double lane_value(double v, uint32_t i) {
    const unsigned long long b = __builtin_bit_cast(unsigned long long, v);
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)b, i), hi = __builtin_amdgcn_readlane((uint32_t)(b >> 32), i);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
// The sum over a wavefront, in every lane.
__device__ __forceinline__ double sum_of_wave(double v) {
#define LC_DPP(ctrl) { \
    const unsigned long long b = __builtin_bit_cast(unsigned long long, v); \
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, ctrl, 0xf, 0xf, false), hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(b >> 32), ctrl, 0xf, 0xf, false); \
    v += __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo); }
    LC_DPP(0xB1) LC_DPP(0x4E) LC_DPP(0x141) LC_DPP(0x140)     // of sixteen lanes
#undef LC_DPP
    return lane_value(v, 0) + lane_value(v, 16) + (lane_value(v, 32) + lane_value(v, 48));
}

// A lane's eight weights of what is left, from element `at` on: p less q, if there is one, and without what was refused.
template <int T>
__device__ __forceinline__ void left_of(const Draft& d, uint64_t p_row, const void* draft, uint64_t q_row, const int32_t* gone, uint32_t n_gone, uint32_t at, double rest[kEach]) {
    const int valid = at < d.vocab ? (int)(d.vocab - at < kEach ? d.vocab - at : kEach) : 0;
    float p[kEach], q[kEach];
    load_eight<T>(d.target, p_row + at, valid, p);
    if (draft) load_eight<T>(draft, q_row + at, valid, q);
#pragma unroll
    for (uint32_t e = 0; e < kEach; ++e) rest[e] = draft ? fmax(weight(p[e]) - weight(q[e]), 0.0) : weight(p[e]);
    for (uint32_t g = 0; g < n_gone; ++g) {
        const uint32_t o = (uint32_t)gone[g] - at;
        if (o < kEach)
#pragma unroll
            for (uint32_t e = 0; e < kEach; ++e) if (e == o) rest[e] = 0.0;
    }
}

template <int T>
__global__ __launch_bounds__(kThreads) void k_draft_verify(Draft d) {
    __shared__ int32_t gone[64];
    __shared__ uint32_t s_cur, s_gone, s_refused, is_last, s_slice, found, any;
    __shared__ double s_sum[kThreads / 64], s_target, s_before;
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, b = blockIdx.y, slice = blockIdx.x;
    if (wave == 0) {                                        // the path
        const uint64_t at = (uint64_t)b * d.nodes;
        uint32_t count = d.nodes;
        if (d.count) { const int32_t n = d.count[b]; count = n < 1 ? 1 : (uint32_t)n < count ? (uint32_t)n : count; }
        const bool node = lane >= 1 && lane < count;
        const int32_t token = node ? d.tokens[at + lane] : -1;
        const int32_t above = node ? (d.parent ? d.parent[at + lane] : (int32_t)lane - 1) : -1;
        const float u = lane < d.nodes ? d.uniform[at + lane] : 0.0f;
        const bool known = node && (uint32_t)token < d.vocab && (uint32_t)above < lane;
        const double p = known ? weight(load_one<T>(d.target, b * d.ld_batch + above * d.ld_row + token)) : 0.0;
        const double q = known && d.draft ? weight(load_one<T>(d.draft, b * d.ld_draft_batch + (lane - 1) * d.ld_draft_row + token)) : 0.0;
        uint32_t cur = 0, length = 1, n_gone = 0, refused = 0;
        int32_t place = lane == 0 ? 0 : -1;                 // this node's place on the path
        if (!d.parent && d.draft) {                         // one behind the other: up to the first that is not taken
            const unsigned long long no = __ballot(node && !((double)u * q < p));
            cur = no ? (uint32_t)__builtin_ctzll(no) - 1 : count - 1;
            length = cur + 1;
            refused = no != 0;
            place = lane <= cur ? (int32_t)lane : -1;
        } else {
            double rest = 1.0;
            unsigned long long out = 0;                     // the nodes refused below the path's end
            for (uint32_t i = 1; i < count; ++i) {
                if ((uint32_t)__builtin_amdgcn_readlane(above, i) != cur) continue;
                const int32_t t = __builtin_amdgcn_readlane(token, i);
                const bool again = __ballot((out >> lane & 1) && token == t) != 0;
                const double pi = again ? 0.0 : lane_value(p, i), ui = (double)float_of(__builtin_amdgcn_readlane(bits_of(u), i));
                if (ui * rest < pi) {
                    if (lane == i) place = (int32_t)length;
                    cur = i;
                    ++length;
                    rest = 1.0;
                    out = 0;
                } else {
                    rest -= pi;
                    out |= 1ull << i;
                }
            }
            if (out >> lane & 1) gone[__builtin_popcountll(out & ((1ull << lane) - 1))] = token;
            n_gone = (uint32_t)__builtin_popcountll(out);
        }
        if (lane == 0) { s_cur = cur; s_gone = n_gone; s_refused = refused; found = 0xffffffffu; any = 0; }
        if (slice == 0) {
            if (lane < d.nodes && lane >= length) d.path[at + lane] = -1;
            if (place >= 0) d.path[at + place] = (int32_t)lane;
            if (lane == 0) d.length[b] = (int32_t)length;
        }
    }
    __syncthreads();
    uint32_t n_gone = s_gone;
    const uint64_t p_row = b * d.ld_batch + s_cur * d.ld_row, q_row = b * d.ld_draft_batch + s_cur * d.ld_draft_row;
    const void* draft = s_refused ? d.draft : nullptr;      // (that of node s_cur + 1, which was refused)
    double rest[kEach];
    // The sum of the elements from `first` to before `end`, in every lane.
    auto sum_of = [&](uint32_t first, uint32_t end) {
        double sum = 0;
        for (uint32_t at = first; at < end && at < d.vocab; at += kStep) {
            left_of<T>(d, p_row, draft, q_row, gone, n_gone, at + threadIdx.x * kEach, rest);
#pragma unroll
            for (uint32_t e = 0; e < kEach; ++e) sum += rest[e];
        }
        sum = sum_of_wave(sum);
        __syncthreads();
        if (lane == 0) s_sum[wave] = sum;
        __syncthreads();
        sum = 0;
        for (uint32_t w = 0; w < kThreads / 64; ++w) sum += s_sum[w];
        return sum;
    };
    const double sum = sum_of(slice * d.slice, (slice + 1) * d.slice);
    const uint64_t row = (uint64_t)b * d.slices;
    const double u = (double)d.uniform[(uint64_t)b * d.nodes];
    if (wave == 0) {
        // The last one to get here goes on: each marks its slice done with the call's number, once its sum has arrived, and looks at the marks of all;
        // whoever marks last finds them all there (should two find that, both write the same).  Marks are taken back, so that a replayed call begins without them.
        if (lane == 0) put_shared(d.sums + row + slice, sum);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        unsigned long long* marks = d.marks + row;
        if (lane == 0) __hip_atomic_store(marks + slice, d.call, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const bool here = lane >= d.slices || __hip_atomic_load(marks + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == d.call;
        const bool done = __all(here);
        if (lane == 0) is_last = done;
        if (done) {
            if (lane < d.slices) __hip_atomic_store(marks + lane, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            const double own = lane < d.slices ? get_shared(d.sums + row + lane) : 0.0;
            // one after the other, so that the sums before a slice and behind the one before it are the same number
            double total = 0, before = 0;
            for (uint32_t i = 0; i < d.slices; ++i) {
                if (i == lane) before = total;
                total += lane_value(own, i);
            }
            const double want = u * total;
            const unsigned long long holds = __ballot(own > 0), past = __ballot(own > 0 && before + own > want);
            // (where rounding leaves no sum above what is wanted: the last slice that holds anything)
            const int at = past ? __builtin_ctzll(past) : holds ? 63 - __builtin_clzll(holds) : 0;
            if (lane == 0) {
                s_slice = holds ? (uint32_t)at : 0xffffffffu;
                s_target = want;
            }
            if ((int)lane == at) s_before = before;
        }
    }
    __syncthreads();
    if (!is_last) return;
    double want = s_target, before = s_before;
    uint32_t begin = s_slice * d.slice, end = begin + d.slice;
    if (s_slice == 0xffffffffu) {                           // nothing is left: of p, all of it
        draft = nullptr;
        n_gone = 0;
        begin = 0;
        end = d.vocab;
        const double total = sum_of(begin, end);
        if (!(total > 0)) {
            if (threadIdx.x == 0) d.next[b] = -1;
            return;
        }
        want = u * total;
        before = 0;
    }
    // Once more, up to the element at which the running sum passes what is wanted.
    for (uint32_t at = begin; at < end && at < d.vocab; at += kStep) {
        left_of<T>(d, p_row, draft, q_row, gone, n_gone, at + threadIdx.x * kEach, rest);
        double own = 0;
#pragma unroll
        for (uint32_t e = 0; e < kEach; ++e) own += rest[e];
        double upto = own;
        for (int x = 1; x < 64; x *= 2) { const double o = __shfl_up(upto, x); if (lane >= (uint32_t)x) upto += o; }
        __syncthreads();
        if (lane == 63) s_sum[wave] = upto;
        __syncthreads();
        double run = before;
        for (uint32_t w = 0; w < kThreads / 64; ++w) {
            if (w < wave) run += s_sum[w];
            before += s_sum[w];
        }
        run += upto - own;
        uint32_t hit = 0xffffffffu, last = 0;
#pragma unroll
        for (uint32_t e = 0; e < kEach; ++e) {
            run += rest[e];
            if (rest[e] > 0 && run > want && hit == 0xffffffffu) hit = at + threadIdx.x * kEach + e;
            if (rest[e] > 0) last = at + threadIdx.x * kEach + e + 1;
        }
        if (hit != 0xffffffffu) atomicMin(&found, hit);
        if (last) atomicMax(&any, last);
        __syncthreads();
        if (found != 0xffffffffu) break;
    }
    if (threadIdx.x == 0) d.next[b] = (int32_t)(found != 0xffffffffu ? found : any - 1);
}

constexpr uint64_t kMarks = kMostSlices * 8, kSums = kMostSlices * 8;

}  // namespace
}  // namespace serve
}  // namespace lc

using namespace lc::serve;

extern "C" {

size_t lc_draft_workspace_bytes(uint64_t batch) { return batch > 65535 ? 0 : (size_t)((batch * (kMarks + kSums) + 255) / 256 * 256 + 256); }

int lc_draft_verify(const void* target, uint64_t ld_batch, uint64_t ld_row, uint64_t batch, int nodes, uint64_t vocab, const int32_t* tokens, const void* draft,
                    uint64_t ld_draft_batch, uint64_t ld_draft_row, const int32_t* parent, const int32_t* count, const float* uniform, int dtype,
                    int32_t* path, int32_t* length, int32_t* next, void* ws, size_t ws_bytes, void* stream) {
    if (!served_type(dtype) || batch > 65535 || nodes < 1 || nodes > 64 || vocab < 1 || vocab > (1ull << 24) || (draft && parent)) return LC_ERR_BADARG;
    if (batch == 0) return LC_OK;
    const uintptr_t size = size_of(dtype);
    if (!target || !tokens || !uniform || !path || !length || !next || off(target, size) || off(draft, size) || off(tokens, 4) || off(parent, 4) || off(count, 4) ||
        off(uniform, 4) || off(path, 4) || off(length, 4) || off(next, 4)) return LC_ERR_BADARG;
    if (ld_row > (1ull << 40) || ld_batch > (1ull << 40) || ld_draft_row > (1ull << 40) || ld_draft_batch > (1ull << 40)) return LC_ERR_BADARG;
    if (!ws || off(ws, 256) || ws_bytes < lc_draft_workspace_bytes(batch)) return LC_ERR_WORKSPACE;
    Draft d = {};
    d.target = target; d.ld_batch = ld_batch; d.ld_row = ld_row;
    d.draft = nodes > 1 ? draft : nullptr; d.ld_draft_batch = ld_draft_batch; d.ld_draft_row = ld_draft_row;
    d.tokens = tokens; d.parent = parent; d.count = count; d.uniform = uniform; d.path = path; d.length = length; d.next = next;
    d.nodes = (uint32_t)nodes; d.vocab = (uint32_t)vocab;
    // Slices of a step of a workgroup each, or of as many as leave eight workgroups a compute unit, which is what fits.
    const uint32_t steps = (d.vocab + kStep - 1) / kStep, want = batch >= 2048 ? 1 : (uint32_t)(2048 / batch);
    uint32_t slices = want < kMostSlices ? want : kMostSlices;
    slices = slices < steps ? slices : steps;
    d.slice = (steps + slices - 1) / slices * kStep;
    d.slices = (d.vocab + d.slice - 1) / d.slice;
    d.marks = static_cast<unsigned long long*>(ws);
    d.sums = reinterpret_cast<double*>(static_cast<uint8_t*>(ws) + batch * kMarks);
    static std::atomic<unsigned long long> calls{0x2545f491};
    d.call = calls.fetch_add(1, std::memory_order_relaxed) * 0x9E3779B97F4A7C15ull | 1;      // (one to one on 63 bits, and never zero)
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 grid(d.slices, (uint32_t)batch);
    if (dtype == LC_F32) k_draft_verify<LC_F32><<<grid, kThreads, 0, s>>>(d);
    else if (dtype == LC_BF16) k_draft_verify<LC_BF16><<<grid, kThreads, 0, s>>>(d);
    else k_draft_verify<LC_F16><<<grid, kThreads, 0, s>>>(d);
    return launched();
}

}  // extern "C"
