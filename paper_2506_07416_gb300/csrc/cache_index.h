// Where a cached token lies: page and slot of a position, and the checks that
// keep every access to the pool inside it. Plain C++, so that the host tests
// compile it too.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define LVS_HD __host__ __device__ __forceinline__
#else
#define LVS_HD inline
#endif

namespace lvs {

// Tokens of the longest request that a call takes; as a chunk's length: all keys, the last of such a request among
// them (a multiple of the 64 that every chunk is one of).
constexpr int32_t kMostKeys = 1 << 30;

// Where the chunk of keys from k0 on ends, of the `seen` keys there are (at or below k0: the chunk is empty).
LVS_HD int32_t chunk_end(int32_t seen, int32_t k0, int32_t chunk)
{
    return seen - k0 < chunk ? seen : k0 + chunk;
}

// First tile of 128 rows of request b, `rows` of whose batch stand before it, where every request's tiles follow the
// last one's: a request of n rows has at most floor((rows + n) / 128) - floor(rows / 128) + 1. Of the batch's end: the
// tiles of all.
LVS_HD int64_t tile_at(int64_t rows, int64_t b) { return rows / 128 + b; }

// Tokens of a request that the kernels may touch: its length cut to
// [0, limit]. `bad` tells that the length was outside.
LVS_HD int cache_len(int32_t len, int32_t limit, bool& bad)
{
    bad = len < 0 || len > limit;
    return len < 0 ? 0 : (len > limit ? limit : len);
}

// Pool page of position pos (>= 0) of request b, or -1 where the position lies
// behind the table's row or the table names no page of the pool.
LVS_HD int32_t cache_page(const int32_t* table, int32_t width, int32_t num_pages, int32_t page_shift, int64_t b,
                          int64_t pos)
{
    const int64_t i = pos >> page_shift;
    if (i >= width) return -1;
    const int32_t p = table[b * width + i];
    return p >= 0 && p < num_pages ? p : -1;
}

// Row of (page, head, slot) in an array of [num_pages][heads][page_size] rows
// (64 bits: a pool's bytes pass 2^32).
LVS_HD int64_t cache_row(int64_t page, int32_t heads, int32_t head, int32_t page_shift, int64_t slot)
{
    return (((page * heads + head) << page_shift) + slot);
}

}  // namespace lvs
