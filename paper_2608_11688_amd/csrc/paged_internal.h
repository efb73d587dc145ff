// What the paged-cache entry points share: the checks of a pool.
#pragma once

#include "common.h"

namespace apex {

inline bool power_of_two(int v) { return v > 0 && (v & (v - 1)) == 0; }

inline int log2_of(int v) {
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
}

inline apex_status check_page_sizes(const char *fn, int page_size, int n_pages) {
    APEX_REQUIRE(power_of_two(page_size) && page_size >= 16 && page_size <= 1024,
                 "%s: page_size=%d must be a power of two from 16 to 1024", fn, page_size);
    APEX_REQUIRE(n_pages >= 1, "%s: n_pages=%d must be >= 1", fn, n_pages);
    if (int64_t(n_pages) * page_size >= (int64_t(1) << 31))
        return fail(APEX_E_UNSUPPORTED, "%s: %d pages of %d positions: 2^31 or more positions", fn,
                    n_pages, page_size);
    return APEX_OK;
}

// The sizes of a pool and, with `pointers`, its addresses.
inline apex_status check_paged_cache(const char *fn, const apex_paged_cache *c, bool pointers) {
    APEX_REQUIRE(c, "%s: NULL cache", fn);
    APEX_REQUIRE(c->format == APEX_KV_BF16 || c->format == APEX_KV_FP8_E4M3,
                 "%s: unknown cache format %d", fn, c->format);
    APEX_REQUIRE(c->G >= 1, "%s: G=%d must be >= 1", fn, c->G);
    APEX_REQUIRE(c->hd == 64 || c->hd == 128, "%s: head size %d must be 64 or 128", fn, c->hd);
    if (c->G > 1024) return fail(APEX_E_UNSUPPORTED, "%s: G=%d exceeds 1024", fn, c->G);
    const apex_status st = check_page_sizes(fn, c->page_size, c->n_pages);
    if (st != APEX_OK || !pointers) return st;
    APEX_REQUIRE(c->k_pages && c->v_pages, "%s: NULL pages", fn);
    APEX_REQUIRE(aligned16(c->k_pages) && aligned16(c->v_pages), "%s: pages must be 16-byte aligned",
                 fn);
    if (c->format == APEX_KV_FP8_E4M3) {
        APEX_REQUIRE(c->k_scales && c->v_scales, "%s: E4M3 pages need scales", fn);
        APEX_REQUIRE(aligned16(c->k_scales) && aligned16(c->v_scales),
                     "%s: scales must be 16-byte aligned", fn);
    } else {
        APEX_REQUIRE(!c->k_scales && !c->v_scales, "%s: bf16 pages have no scales", fn);
    }
    return APEX_OK;
}

// Rows of `n` values of an apex_type at a stride: 16-byte loads stay aligned and in the row.
inline apex_status check_rows(const char *fn, const char *what, int dtype, int64_t stride, int64_t n) {
    const int per = dtype == APEX_TYPE_FP32 ? 4 : 8;   // values in 16 bytes
    APEX_REQUIRE(stride >= n && stride % per == 0,
                 "%s: %s_stride=%lld must be a multiple of %d and at least %lld", fn, what,
                 static_cast<long long>(stride), per, static_cast<long long>(n));
    return APEX_OK;
}

}  // namespace apex
