// Places in a paged cache of keys and values.
#pragma once

#include <hip/hip_runtime.h>

#include "stream_internal.h"

namespace fqvit {
namespace cache {

// Number of keys of sequence b, within what its table can name.
__device__ __forceinline__ int keys_of(const CacheView& c, int b) {
    return min(max(c.length[b], 0), c.max_pages << c.log2_page);
}

// Place of the first of n (<= 2^20) new tokens of sequence b, its last keys: below 0 or beyond
// the table where the length says so.  No key lies beyond 2^20, so a length of 2^30 stands for
// all above it, and 0 for all below.
__device__ __forceinline__ int first_new(const CacheView& c, int b, int n) {
    return min(max(c.length[b], 0), 1 << 30) - n;
}

// The page at place `at` (< max_pages) of sequence b's table.  An id that is no
// page of the cache reads as page 0: never a place outside the cache.
__device__ __forceinline__ int page_at(const int32_t* table, int max_pages, int pages, int b, int at) {
    const int id = table[(int64_t)b * max_pages + at];
    return (uint32_t)id < (uint32_t)pages ? id : 0;
}

// First byte of (page, head) among the keys or the values: both hold page * d.
__device__ __forceinline__ int64_t head_base(const CacheView& c, int page, int h) {
    return ((int64_t)page * c.Hkv + h) * ((int64_t)c.d << c.log2_page);
}

}  // namespace cache
}  // namespace fqvit
