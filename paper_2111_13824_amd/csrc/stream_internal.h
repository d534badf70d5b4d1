// Arguments and launchers of a step over a stream of tokens: the root-mean-square
// norm, the paged cache of keys and values, attention over it, eviction from it.
// Weak, as in layers_internal.h: a host-only build of the C ABI may leave these
// launchers out.
#pragma once

#include "fqvit_internal.h"

namespace fqvit {

struct RmsArgs {
    const int8_t* x;        // nullable [T, C]: the branch
    const uint8_t* alpha;   // nullable [C]
    int32_t zp_x, K;
    float m_x;              // s_x / s_r
    const int16_t* r;       // [T, C]: the stream
    const float* gamma;     // [C]
    int64_t T;
    int32_t C;
    float eps;              // in steps of the stream, squared
    float s_out;            // one scale (scales null)
    int32_t zp_out, bits;
    int16_t* h;             // [T, C] out (may be r)
    int8_t* y;              // [T, C] out
    float* scales;          // nullable [T]: a scale for each row
};

__attribute__((weak)) hipError_t launch_rmsnorm(const RmsArgs& a, hipStream_t stream);

// A cache: pages of `page` keys (a power of two), a table of them for each sequence.
struct CacheView {
    int8_t* k;              // [pages, Hkv, page, d]
    int8_t* v;              // [pages, Hkv, d, page]
    int64_t* weight;        // nullable [pages, Hkv, page]
    const int32_t* table;   // [B, max_pages]
    const int32_t* length;  // [B]
    int32_t pages, max_pages, log2_page;
    int32_t B, Hkv, d;
};

struct AppendArgs {
    CacheView c;
    const int8_t* k;        // [B, Hkv, L, d]
    const int8_t* v;
    const int32_t* n_new;   // nullable [B]
    int32_t L;
};

__attribute__((weak)) hipError_t launch_kv_append(const AppendArgs& a, hipStream_t stream);

struct PagedArgs {
    CacheView c;
    const int8_t* q;        // [B, Hq, L, d]
    const int32_t* n_new;   // nullable [B]
    int32_t Hq, L, group;   // group = Hq / Hkv
    int32_t zp_q, zp_v, causal;
    LisConsts k;
    int32_t* out;           // [B, Hq, L, d]
    void* workspace;
};

// Bytes that a call with these sizes needs (0: none).
__attribute__((weak)) size_t lis_paged_workspace(int32_t B, int32_t Hq, int32_t Hkv, int32_t L,
                                                 int32_t d, int64_t max_keys);
__attribute__((weak)) hipError_t launch_lis_paged(const PagedArgs& a, hipStream_t stream);

struct EvictArgs {
    CacheView c;            // the pages that are read (and written, through table_out)
    const int32_t* table_out;   // [B, max_out]; c.table: in place
    int32_t max_out;
    int32_t keep, recent;
    int32_t* length_out;    // [B] (may be c.length)
    int32_t* kept;          // [B, Hkv, keep]
};

__attribute__((weak)) hipError_t launch_kv_evict(const EvictArgs& a, hipStream_t stream);

}  // namespace fqvit
