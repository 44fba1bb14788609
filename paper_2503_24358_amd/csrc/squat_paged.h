// What the calls on a paged store share: its checks on the host, and where a token's codes lie.
#pragma once

#include "squat_internal.h"

namespace squat {

// SQUAT_OK, or what is wrong with a store (every call on one checks this first).
inline int check_store(const squat_paged_store* s) {
    if (!s) return SQUAT_E_NULLPTR;
    if (s->d != kD || (s->bits != 2 && s->bits != 4 && s->bits != 8)) return SQUAT_E_BADSHAPE;
    if (s->group != 32 && s->group != 64 && s->group != 128) return SQUAT_E_BADSHAPE;
    const int p = s->page_tokens;
    if (p < 16 || p > 1024 || (p & (p - 1))) return SQUAT_E_BADSHAPE;
    // (a launch has a workgroup's worth of threads per head; page numbers are 32-bit)
    if (s->n_kv_heads < 1 || s->n_kv_heads > 65535 || s->n_pages < 1 || s->n_pages > 0x7FFFFFFF) return SQUAT_E_BADSHAPE;
    if (!s->key_codes || !s->key_meta || !s->value_codes || !s->value_meta) return SQUAT_E_NULLPTR;
    if (!aligned(s->key_codes, 16) || !aligned(s->value_codes, 16) || !aligned(s->key_meta, 16) || !aligned(s->value_meta, 16))
        return SQUAT_E_ALIGN;
    return SQUAT_OK;
}

}  // namespace squat
