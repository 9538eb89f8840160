// The paged key/value cache as its kernels see it (device code and launchers of fbq_cache.hip, fbq_attend_*.hip).
#ifndef FBQ_CACHE_H
#define FBQ_CACHE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fbq.h"

namespace fbq {

struct CacheArgs {
    unsigned char *pool;
    int32_t *table, *lengths, *refs;
    long page_bytes;             // of one layer
    long layer_bytes;
    int pages, layers, log_ps, max_pages, rows, kv_heads, D;
};

inline CacheArgs cache_args(const fbq_cache &c)
{
    CacheArgs a{};
    const fbq_cache_desc &d = c.desc;
    a.pool = (unsigned char *)c.pool;
    a.table = c.table; a.lengths = c.lengths; a.refs = c.refs;
    a.log_ps = __builtin_ctz(d.page_size);
    a.page_bytes = 4L * d.kv_heads * d.page_size * d.head_dim;
    a.layer_bytes = a.page_bytes * d.pages;
    a.pages = d.pages; a.layers = d.layers; a.max_pages = c.max_pages; a.rows = c.rows; a.kv_heads = d.kv_heads; a.D = d.head_dim;
    return a;
}

// FBQ_OK, or what is wrong with the cache itself (`refs` whether the call uses them).  Host only.
fbq_status check_cache(const fbq_cache *c, bool refs);

inline bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// Sum over this lane and those before it in the wave; the last lane has all.  (Six additions of neighbours' registers; by way of LDS each would wait for it.)
__device__ __forceinline__ int wave_scan(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // within 16 lanes, by 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // lane 15's to the second 16 of each 32
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // lane 31's to the second 32
    return x;
}

// How many of its tokens a row is taken to have, whatever its length says.
__device__ __forceinline__ int tokens_of(int length, int max_tokens) { return min(max(length, 0), max_tokens); }

// The row b whose q_start[b] <= t < q_start[b + 1] (ascending; rows without tokens are passed over), -1 if there is none.
__device__ __forceinline__ int row_of_token(const int32_t *__restrict__ q_start, int rows, int t)
{
    if (t < q_start[0] || t >= q_start[rows]) return -1;
    int lo = 0, hi = rows;                                    // q_start[lo] <= t < q_start[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (q_start[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

}  // namespace fbq

#endif
