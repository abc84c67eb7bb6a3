// The 8-bit key/value cache of include/abft_eb.h as the kernels see it.
#pragma once
#include <stdint.h>

#include "../../include/abft_eb.h"
#include "abft_internal.h"

namespace abft {

constexpr int kKvGroup = 16;   // tokens that stand side by side in v_codes
constexpr int kKvTile = 64;    // tokens that attention takes at a time

inline int kv_columns(int head_dim) { return (head_dim + 63) / 64 * 64; }
// null, or what is wrong with the sizes
inline const char* kv_wrong_sizes(const abft_kv_cache_t* c) {
    if (!c) return "null cache";
    if (c->n_blocks < 1 || c->heads < 1) return "a cache needs blocks and heads";
    if (c->head_dim < 1 || c->head_dim > 256) return "head_dim must be 1..256";
    if (c->block_tokens != 16 && c->block_tokens != 32 && c->block_tokens != 64 && c->block_tokens != 128) return "block_tokens must be 16, 32, 64 or 128";
    return nullptr;
}
inline const char* kv_wrong(const abft_kv_cache_t* c) {
    if (const char* w = kv_wrong_sizes(c)) return w;
    if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale) return "null pointer in the cache";
    if ((reinterpret_cast<uintptr_t>(c->k_codes) | reinterpret_cast<uintptr_t>(c->v_codes)) & 15) return "codes must be 16-byte aligned";
    if (c->heads > 65535) return "too many heads";
    return nullptr;
}

}  // namespace abft
