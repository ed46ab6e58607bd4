// The paged cache as the kernels that read and write it see it (lc_kv.hip, lc_prompt.hip).
#pragma once
#include "lc_serve.h"

namespace lc {
namespace serve {

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

inline bool bad(const lc_kv_cache* c) {
    if (!c || c->heads < 1 || c->heads > 1024 || c->dim < 32 || c->dim > 256 || c->dim % 32 || (c->bits != 8 && c->bits != 4)) return true;
    if (c->page_tokens < 8 || c->page_tokens > 1024 || (c->page_tokens & (c->page_tokens - 1)) || c->pages > (1ull << 31) / c->page_tokens) return true;
    if (c->pages == 0) return false;
    return !c->k || !c->v || !c->k_scale || !c->v_scale || off(c->k, 16) || off(c->v, 16) || off(c->k_scale, 16) || off(c->v_scale, 16);
}
inline Cache described(const lc_kv_cache& c) {
    return {static_cast<uint8_t*>(c.k), static_cast<uint8_t*>(c.v), c.k_scale, c.v_scale, c.pages * c.page_tokens,
            (uint32_t)__builtin_ctz((unsigned)c.page_tokens), (uint32_t)c.heads, (uint32_t)c.dim, (uint32_t)(c.dim * c.bits / 8)};
}

}  // namespace serve
}  // namespace lc
