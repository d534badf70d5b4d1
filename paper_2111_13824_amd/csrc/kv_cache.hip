// The paged cache of keys and values for gfx950: new tokens written into it, and
// eviction from it by accumulated attention weight.
//
// A page holds `page` keys of every head: keys as rows [page, d], values with their
// channels as rows [d, page].  16 keys of a channel are then 16 neighbouring bytes,
// what a lane feeds to the int8 matrix cores as its operand of P V: the attention
// reads values with the same wide loads as keys and transposes nothing, and the
// transposition is paid once, when a token is written.
#include "cache_device.h"
#include "fqvit_launch.h"

namespace fqvit {
namespace {

using cache::head_base;
using cache::keys_of;
using cache::page_at;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 256;
constexpr int kSpan = 64;       // keys a workgroup of the append takes

// ---------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------

// New tokens of sequence b: token i < n goes to place first + i.
struct NewKeys {
    int first, n;
};

// Tokens whose place would lie before the first or beyond the table are left out.
__device__ __forceinline__ NewKeys new_keys(const AppendArgs& a, int b) {
    const int n = a.n_new ? min(max(a.n_new[b], 0), a.L) : a.L;
    return NewKeys{cache::first_new(a.c, b, n), n};
}

__device__ __forceinline__ bool in_table(const CacheView& c, int place) {
    return place >= 0 && place < (c.max_pages << c.log2_page);
}

// Few new tokens a sequence: a thread takes 16 channels of one token's key and value.
// Bound by its launch (one token of 64 sequences, 4 heads of 64: 7.4 us a call).
__global__ __launch_bounds__(kBlock) void append_tokens_kernel(AppendArgs a) {
    const CacheView& c = a.c;
    const int chunks = c.d >> 4;
    const int64_t all = (int64_t)c.B * c.Hkv * a.L * chunks;
    const int64_t step = (int64_t)gridDim.x * kBlock;
    for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < all; at += step) {
        const int ch = (int)(at % chunks);
        const int64_t tok = at / chunks;        // (b, h, i)
        const int i = (int)(tok % a.L);
        const int h = (int)(tok / a.L % c.Hkv);
        const int b = (int)(tok / a.L / c.Hkv);
        const NewKeys nk = new_keys(a, b);
        const int place = nk.first + i;
        if (i >= nk.n || !in_table(c, place)) continue;
        const int id = c.table[(int64_t)b * c.max_pages + (place >> c.log2_page)];
        if ((uint32_t)id >= (uint32_t)c.pages) continue;
        const int page = 1 << c.log2_page, slot = place & (page - 1);
        const int64_t base = head_base(c, id, h);
        const u32x4 kw = *reinterpret_cast<const u32x4*>(a.k + tok * c.d + 16 * ch);
        const u32x4 vw = *reinterpret_cast<const u32x4*>(a.v + tok * c.d + 16 * ch);
        *reinterpret_cast<u32x4*>(c.k + base + (int64_t)slot * c.d + 16 * ch) = kw;
        int8_t* dst = c.v + base + (int64_t)(16 * ch) * page + slot;
#pragma unroll
        for (int e = 0; e < 16; ++e) dst[(int64_t)e * page] = (int8_t)(vw[e >> 2] >> (8 * (e & 3)));
        if (c.weight && ch == 0) c.weight[((int64_t)id * c.Hkv + h) * page + slot] = 0;
    }
}

// Many new tokens: a workgroup takes the places [64 n, 64 n + 64) of one sequence
// and head.  Keys are copied; values go through LDS, a thread turns 4 channels of
// 16 keys, one 16-byte store a channel.  (16 sequences of up to 577 tokens, 16 heads of 64,
// 20 MB read and written: 7.3 us, of which a copy of as much would take 3.8.)
__global__ __launch_bounds__(kBlock) void append_span_kernel(AppendArgs a) {
    __shared__ uint32_t lds[kSpan * 33];        // [key][d / 4 + 1], d <= 128
    const CacheView& c = a.c;
    const int b = blockIdx.z, h = blockIdx.y;
    const NewKeys nk = new_keys(a, b);
    const int lo = max(nk.first, 0);
    const int hi = min(nk.first + nk.n, c.max_pages << c.log2_page);
    const int span0 = ((lo >> 6) + (int)blockIdx.x) * kSpan;
    if (lo >= hi || span0 >= hi) return;
    const int page = 1 << c.log2_page, d = c.d, chunks = d >> 4, ld = (d >> 2) + 1;
    const int64_t src = ((int64_t)b * c.Hkv + h) * a.L;
    for (int at = threadIdx.x; at < kSpan * chunks; at += kBlock) {
        const int j = at / chunks, ch = at - j * chunks;
        const int place = span0 + j;
        if (place < lo || place >= hi) continue;
        const int64_t row = (src + place - nk.first) * d + 16 * ch;
        const u32x4 vw = *reinterpret_cast<const u32x4*>(a.v + row);
#pragma unroll
        for (int e = 0; e < 4; ++e) lds[j * ld + 4 * ch + e] = vw[e];
        const int id = c.table[(int64_t)b * c.max_pages + (place >> c.log2_page)];
        if ((uint32_t)id >= (uint32_t)c.pages) continue;
        const int slot = place & (page - 1);
        *reinterpret_cast<u32x4*>(c.k + head_base(c, id, h) + (int64_t)slot * d + 16 * ch) =
            *reinterpret_cast<const u32x4*>(a.k + row);
        if (c.weight && ch == 0) c.weight[((int64_t)id * c.Hkv + h) * page + slot] = 0;
    }
    __syncthreads();
    // (4 channels, 16 keys) of a thread; the keys of a group lie in one page
    for (int at = threadIdx.x; at < (d >> 2) * (kSpan / 16); at += kBlock) {
        const int grp = at / (d >> 2), c4 = at - grp * (d >> 2);
        const int place = span0 + 16 * grp;
        if (place + 16 <= lo || place >= hi) continue;
        const int id = c.table[(int64_t)b * c.max_pages + (place >> c.log2_page)];
        if ((uint32_t)id >= (uint32_t)c.pages) continue;
        int8_t* dst = c.v + head_base(c, id, h) + (int64_t)(4 * c4) * page + (place & (page - 1));
        uint32_t w[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j] = lds[(16 * grp + j) * ld + c4];
        if (place >= lo && place + 16 <= hi) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                u32x4 o;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t s = 0x0c0c0400u + 0x0101u * e;     // byte e of both
                    const uint32_t x = __builtin_amdgcn_perm(w[4 * q + 1], w[4 * q], s);
                    const uint32_t y = __builtin_amdgcn_perm(w[4 * q + 3], w[4 * q + 2], s);
                    o[q] = x | (y << 16);
                }
                *reinterpret_cast<u32x4*>(dst + (int64_t)e * page) = o;
            }
        } else {        // keys that are not new keep their values
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (place + j >= lo && place + j < hi)
                    for (int e = 0; e < 4; ++e) dst[(int64_t)e * page + j] = (int8_t)(w[j] >> (8 * e));
        }
    }
}

}  // namespace

hipError_t launch_kv_append(const AppendArgs& a, hipStream_t stream) {
    const CacheView& c = a.c;
    if (a.L < 16) {
        const int64_t all = (int64_t)c.B * c.Hkv * a.L * (c.d >> 4);
        const int64_t blocks = (all + kBlock - 1) / kBlock;
        launch_kernel(append_tokens_kernel, dim3((uint32_t)(blocks < (1 << 20) ? blocks : (1 << 20))),
                      dim3(kBlock), 0, stream, a);
    } else {
        // L tokens from any place touch at most this many aligned spans
        launch_kernel(append_span_kernel, dim3((a.L + 2 * kSpan - 2) / kSpan, c.Hkv, c.B), dim3(kBlock), 0,
                      stream, a);
    }
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Eviction
// ---------------------------------------------------------------------------

namespace {

constexpr int kSelect = 1024;
constexpr int kSelectWaves = kSelect / 64;
constexpr int kCopies = 8;

// Order of signed weights as unsigned numbers.
__device__ __forceinline__ uint64_t rank_of(int64_t w) { return (uint64_t)w ^ (1ull << 63); }

__device__ __forceinline__ const int64_t* weight_slot(const CacheView& c, int b, int h, int place) {
    const int id = page_at(c.table, c.max_pages, c.pages, b, place >> c.log2_page);
    return c.weight + (((int64_t)id * c.Hkv + h) << c.log2_page) + (place & ((1 << c.log2_page) - 1));
}

// The places that stay, one workgroup for each sequence and head.  A thread holds ITEMS
// neighbouring weights (ITEMS 0: reads runs of 8 again in each pass).  The m-th heaviest of the
// old keys is found digit by digit (8 bits, a histogram in LDS, whose sums from the top
// one wavefront takes) from the first bit in which the weights differ; then one scan
// over the threads places what is heavier and as many of its equals, from the lowest
// place on, as are missing.  (A histogram that one thread walks takes 10 us a digit.)
// Bound by latency, of three loads in a row and of the digits' passes: 128 units of up to 8192
// weights, 5 MB, 11.8 us (12.3 where all digits are looked at, 14.5 with one histogram, whose
// first bins' additions, weights of all sizes in them, wait for each other).
template <int ITEMS>
__global__ __launch_bounds__(kSelect) void evict_select_kernel(EvictArgs a) {
    __shared__ uint32_t hist[kCopies][257];     // copies begin in different banks
    __shared__ uint64_t wide[kSelectWaves];
    __shared__ uint32_t part[2][kSelectWaves];
    __shared__ uint64_t bound;
    __shared__ int missing;
    constexpr int kHeld = ITEMS ? ITEMS : 8;
    const CacheView& c = a.c;
    const int b = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = keys_of(c, b);
    int32_t* kept = a.kept + ((int64_t)b * c.Hkv + h) * a.keep;
    if (n <= a.keep) {
        for (int j = tid; j < a.keep; j += kSelect) kept[j] = j < n ? j : -1;
        return;
    }
    const int old = n - a.recent, m = a.keep - a.recent;       // m < old
    for (int j = tid; j < a.recent; j += kSelect) kept[m + j] = old + j;
    if (m == 0) return;

    // f(first place, weights) for the thread's runs; the places at `old` and behind do not count
    uint64_t held[kHeld];
    const auto fetch = [&](int place, uint64_t* w) {
        if (place >= old) return;
        const int64_t* p = weight_slot(c, b, h, place);         // 8 places lie in one page
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = rank_of(p[e]);
    };
    if (ITEMS)
#pragma unroll
        for (int g = 0; g < kHeld; g += 8) fetch(tid * ITEMS + g, held + g);
    const int runs = (old + 8 * kSelect - 1) / (8 * kSelect);
    const auto each = [&](auto&& f) {
        if (ITEMS) {
#pragma unroll
            for (int e = 0; e < kHeld; ++e)
                if (tid * ITEMS + e < old) f(held[e]);
        } else {
            for (int r = 0; r < runs; ++r) {
                const int place = 8 * (r * kSelect + tid);
                fetch(place, held);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (place + e < old) f(held[e]);
            }
        }
    };

    const uint64_t w0 = rank_of(*weight_slot(c, b, h, 0));
    uint64_t diff = 0;
    each([&](uint64_t w) { diff |= w ^ w0; });
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) diff |= __shfl_xor(diff, o);
    if (lane == 0) wide[wave] = diff;
    __syncthreads();
    diff = 0;
    for (int i = 0; i < kSelectWaves; ++i) diff |= wide[i];
    // bits [0, top) differ; the others are w0's
    const int top = diff ? 64 - __clzll((long long)diff) : 0;
    uint64_t prefix = top < 64 ? w0 >> top << top : 0;
    int need = m;
    for (int hi = top; hi > 0 && need > 0;) {
        const int lo = max(hi - 8, 0);
        const uint32_t mask = (1u << (hi - lo)) - 1;
        for (int i = tid; i < kCopies * 257; i += kSelect) (&hist[0][0])[i] = 0;
        __syncthreads();
        each([&](uint64_t w) {
            if (hi == 64 || (w >> hi) == (prefix >> hi)) atomicAdd(&hist[lane % kCopies][(uint32_t)(w >> lo) & mask], 1u);
        });
        __syncthreads();
        if (wave == 0) {        // the digit of the need-th heaviest: lane l holds the bins 255 - 4 l and below
            uint32_t v[4], sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = 0;
#pragma unroll
                for (int i = 0; i < kCopies; ++i) v[e] += hist[i][255 - 4 * lane - e];
                sum += v[e];
            }
            uint32_t before = sum;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const uint32_t x = __shfl_up(before, o);
                before += lane >= o ? x : 0;
            }
            before -= sum;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if ((uint32_t)need > before && (uint32_t)need <= before + v[e]) {
                    const uint64_t at = prefix | ((uint64_t)(255 - 4 * lane - e) << lo);
                    const int left = need - (int)before;
                    // all of this bin stay: what is heavier than the weight below it
                    const bool all = (uint32_t)left == v[e] && at != 0;
                    bound = all ? at - 1 : at;
                    missing = all ? 0 : left;
                }
                before += v[e];
            }
        }
        __syncthreads();
        prefix = bound;
        need = missing;
        hi = lo;
    }
    // heavier than `prefix`: m - need of them; of its equals the first `need`
    int done_heavy = 0, done_equal = 0;
    for (int r = 0; r < (ITEMS ? 1 : runs); ++r) {
        const int place = ITEMS ? tid * ITEMS : 8 * (r * kSelect + tid);
        if (!ITEMS) fetch(place, held);
        uint32_t nh = 0, ne = 0;
#pragma unroll
        for (int e = 0; e < kHeld; ++e)
            if (place + e < old) {
                nh += held[e] > prefix;
                ne += held[e] == prefix;
            }
        uint32_t sh = nh, se = ne;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t xh = __shfl_up(sh, o), xe = __shfl_up(se, o);
            sh += lane >= o ? xh : 0;
            se += lane >= o ? xe : 0;
        }
        __syncthreads();
        if (lane == 63) {
            part[0][wave] = sh;
            part[1][wave] = se;
        }
        __syncthreads();
        int heavies = done_heavy + (int)(sh - nh), equals = done_equal + (int)(se - ne);
        for (int i = 0; i < kSelectWaves; ++i) {
            if (i < wave) {
                heavies += (int)part[0][i];
                equals += (int)part[1][i];
            }
            done_heavy += (int)part[0][i];
            done_equal += (int)part[1][i];
        }
#pragma unroll
        for (int e = 0; e < kHeld; ++e)
            if (place + e < old) {
                if (held[e] > prefix) kept[heavies++ + min(equals, need)] = place + e;
                else if (held[e] == prefix) {
                    if (equals < need) kept[heavies + equals] = place + e;
                    ++equals;
                }
            }
    }
}

// Keys, values and weights of the places that stay, to the places [0, keep) of the
// pages of table_out.  The places are ascending, so kept[j] >= j, and a tile of
// places that is read whole before any of it is written may be written in place when
// the tiles come in order: a tile's sources lie at or behind it, what it overwrites
// is no later tile's source.  A sequence whose first page stays its first one is moved
// so, by the workgroups z = 0; in other pages the order does not matter.  A workgroup
// moves the keys (x = 0), 16 channels of the values, or the weights (the last x) of one
// sequence and head.  Bound by memory: of a quarter of the keys nearly all lines of the
// values come in (128 units, 2048 of up to 8192 keys of 64: 69 MB read and 34 written in
// 31 us, a copy of as much would take 20; writing four keys as one word changed nothing).
// In place one workgroup a part walks the tiles one after another, and a key that stays where it
// is is written again: 16 such sequences take 15 us more, one sequence of 131072 keys cut to
// 32768 307 us in all, in other pages 33.
constexpr int kMoveUnits = 8;       // 16-byte units a thread holds

__global__ __launch_bounds__(kBlock) void evict_move_kernel(EvictArgs a) {
    const CacheView& c = a.c;
    const int parts = 2 + (c.d >> 4);
    const int part = blockIdx.x % parts, h = blockIdx.x / parts, b = blockIdx.y;
    const int32_t* kept = a.kept + ((int64_t)b * c.Hkv + h) * a.keep;
    const int page = 1 << c.log2_page, d = c.d, most = (c.max_pages << c.log2_page) - 1;
    const bool here = a.table_out[(int64_t)b * a.max_out] == c.table[(int64_t)b * c.max_pages];
    if (here && blockIdx.z > 0) return;
    const int zs = here ? 1 : gridDim.z;
    // the length is read by nothing else here: it may be written in place
    if (part == 0 && h == 0 && blockIdx.z == 0 && threadIdx.x == 0) a.length_out[b] = min(keys_of(c, b), a.keep);
    // place that j comes from; behind the last that stays: none
    const auto from = [&](int j) { return j < a.keep ? min(kept[j], most) : -1; };
    // the page that place j goes to; none: nothing is written
    const auto target = [&](int j) {
        const int id = a.table_out[(int64_t)b * a.max_out + (j >> c.log2_page)];
        return (uint32_t)id < (uint32_t)c.pages ? id : -1;
    };
    const auto source = [&](int j) { return page_at(c.table, c.max_pages, c.pages, b, j >> c.log2_page); };
    if (part == 0) {
        const int chunks = d >> 4, tile = kBlock * kMoveUnits / chunks;       // keys
        for (int j0 = blockIdx.z * tile; j0 < a.keep; j0 += zs * tile) {
            u32x4 w[kMoveUnits];
            bool live[kMoveUnits];
#pragma unroll
            for (int u = 0; u < kMoveUnits; ++u) {
                const int at = threadIdx.x + kBlock * u, j = j0 + at / chunks, ch = at % chunks;
                const int s = at < tile * chunks ? from(j) : -1;
                live[u] = s >= 0;
                if (live[u])
                    w[u] = *reinterpret_cast<const u32x4*>(c.k + head_base(c, source(s), h) +
                                                           (int64_t)(s & (page - 1)) * d + 16 * ch);
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kMoveUnits; ++u) {
                const int at = threadIdx.x + kBlock * u, j = j0 + at / chunks, ch = at % chunks;
                const int to = live[u] ? target(j) : -1;
                if (to >= 0)
                    *reinterpret_cast<u32x4*>(c.k + head_base(c, to, h) + (int64_t)(j & (page - 1)) * d +
                                              16 * ch) = w[u];
            }
        }
    } else if (part < parts - 1) {
        // 256 keys of 16 channels a tile: a lane holds 16 channels of one key
        const int c0 = 16 * (part - 1);
        for (int j0 = blockIdx.z * kBlock; j0 < a.keep; j0 += zs * kBlock) {
            const int j = j0 + threadIdx.x, s = from(j);
            int8_t w[16];
            if (s >= 0) {
                const int8_t* src = c.v + head_base(c, source(s), h) + (int64_t)c0 * page + (s & (page - 1));
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = src[(int64_t)e * page];
            }
            __syncthreads();
            const int to = s >= 0 ? target(j) : -1;
            if (to >= 0) {
                int8_t* dst = c.v + head_base(c, to, h) + (int64_t)c0 * page + (j & (page - 1));
#pragma unroll
                for (int e = 0; e < 16; ++e) dst[(int64_t)e * page] = w[e];
            }
        }
    } else {
        for (int j0 = blockIdx.z * kBlock; j0 < a.keep; j0 += zs * kBlock) {
            const int j = j0 + threadIdx.x, s = from(j);
            int64_t w = 0;
            if (s >= 0) w = *weight_slot(c, b, h, s);
            __syncthreads();
            const int to = s >= 0 ? target(j) : -1;
            if (to >= 0) c.weight[(((int64_t)to * c.Hkv + h) << c.log2_page) + (j & (page - 1))] = w;
        }
    }
}

}  // namespace

hipError_t launch_kv_evict(const EvictArgs& a, hipStream_t stream) {
    const CacheView& c = a.c;
    const LaunchEvents ev = launch_events();
    set_launch_events(ev.start, nullptr);
    const int64_t most = (int64_t)c.max_pages << c.log2_page;
    const dim3 units(c.Hkv, c.B);
    if (most <= 8 * kSelect) launch_kernel(evict_select_kernel<8>, units, dim3(kSelect), 0, stream, a);
    else if (most <= 32 * kSelect) launch_kernel(evict_select_kernel<32>, units, dim3(kSelect), 0, stream, a);
    else launch_kernel(evict_select_kernel<0>, units, dim3(kSelect), 0, stream, a);
    set_launch_events(nullptr, ev.stop);
    const int tiles = a.table_out == c.table ? 1 : (a.keep + kBlock - 1) / kBlock;      // (in place: z = 0)
    launch_kernel(evict_move_kernel, dim3((2 + (c.d >> 4)) * c.Hkv, c.B, tiles < 16 ? tiles : 16),
                  dim3(kBlock), 0, stream, a);
    return hipGetLastError();
}

}  // namespace fqvit
