// Attention of new tokens over a paged cache, integer-only, for gfx950: the int8
// product Q K^T, Log-Int-Softmax and the BitShift product with V (Sec. 3.1, 3.3;
// Supplement A.2), with logits and codes kept on chip.
//
// Layout.  The product is taken transposed: D = K Q^T of the 16x16x64 int8 matrix
// instruction gives a lane (r, g) = (lane % 16, lane / 16) four keys of query r.  Row
// m of the K operand of instruction t (0..3) is key 16 (m / 4) + 4 t + m % 4 of a tile
// of 64, so that lane (r, g) holds the 16 neighbouring keys 16 g .. 16 g + 15 of query
// r: a row's maximum, sum and thresholds belong to one register of its lane, its codes
// need no exchange, and the 16 weights P of a lane are, as bytes, its operand of the
// second product D = V^T P^T.  The V^T operand is 16 neighbouring keys of a channel:
// the cache holds values with their channels in rows.  No operand goes through LDS.
//
// A weight P = 2^m, m = (2^b - 1) - code in [0, 15], is not an int8: it is taken as
// -256 hi - lo with hi, lo in {0, -1, -2, .. -128}, two products with the same V
// operand, exact in int32.
//
// The row's maximum is needed before the first I-Exp, its exact sum before the first
// code: three passes over the keys.  The matrix cores are far from busy (a logit costs
// them less than one vector instruction), so each pass takes the logits again; a call
// of at most 16 rows a key head, which the keys' bytes bound, stores them instead.
//
// Codes without I-Exp.  e(u), u = max - logit, does not increase with u (the host
// checks the one place where rounding could make it, the end of an octave), so
// code >= k, c_k e(u) <= 2 S (c_1 = 3, c_k = 3 2^(k-1) - 1), is u >= U_k for 2^b - 1
// integers U_k of the row.  They are found exactly, once a row.  U_(k+1) - U_k is at
// least q_ln2 for k >= 2 and above q_ln2 / 2 for k = 1, while U_k is not 0: buckets of
// 2^shift <= q_ln2 / 2 values of u hold at most one threshold behind their first
// value, and one word in LDS for each row and bucket, E = 2^24 (2^b - 1 - c) + th - 1
// with c the code at the bucket's first u and th its threshold (or its end), gives
// m = (E - u) >> 24.  A code costs five vector instructions and one LDS read where the
// I-Exp and comparisons with S take about thirty.
#include "cache_device.h"
#include "fqvit_launch.h"
#include "lis_device.h"
#include "lis_paged_plan.h"

namespace fqvit {
namespace {

using cache::head_base;
using cache::keys_of;
using cache::page_at;
using paged::kTile;
using paged::kWaves;
using paged::Plan;
using paged::Shape;

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 64 * kWaves;

// Passes of a launch: all of them, or one where the keys are divided.
enum Pass { kAll, kMax, kSum, kOut };

// Row rho of a sequence and head is query (token rho / group, head rho % group).
__device__ __forceinline__ int64_t query_of(const PagedArgs& a, int b, int h, int rho) {
    const int i = rho / a.group, g = rho - i * a.group;
    return ((int64_t)b * a.Hq + h * a.group + g) * a.L + i;
}

__device__ __forceinline__ int limit_of(const PagedArgs& a, int len, int fresh, int rho) {
    return a.causal ? min(max(len - fresh + rho / a.group + 1, 0), len) : len;
}

template <int KS>
struct Operand {
    i32x4 w[KS];
};

// The keys and values of one sequence and head.
template <int KS>
struct Keys {
    const PagedArgs& a;
    int b, h, len, lane;

    // first byte of the 16 keys that hold place `at` (a multiple of 16), in k or v
    __device__ __forceinline__ int64_t base(int at, int& off) const {
        at = min(at, (len - 1) & ~15);          // behind the last key: its block again
        off = at & ((1 << a.c.log2_page) - 1);
        return head_base(a.c, page_at(a.c.table, a.c.max_pages, a.c.pages, b, at >> a.c.log2_page), h);
    }

    __device__ __forceinline__ const int8_t* k_rows(int key0) const {
        const int m = lane & 15;
        int off;
        const int64_t at = base(key0 + 16 * (m >> 2), off);
        return a.c.k + at + (int64_t)(off + (m & 3)) * a.c.d + 16 * (lane >> 4);
    }

    __device__ __forceinline__ void load_k(const int8_t* p, Operand<KS> (&k)[4]) const {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int s = 0; s < KS; ++s)
                k[t].w[s] = 64 * s + 16 * (lane >> 4) < a.c.d
                                ? *reinterpret_cast<const i32x4*>(p + 4 * t * a.c.d + 64 * s)
                                : i32x4{0, 0, 0, 0};
    }

    // channels 16 ct + lane % 16 of the keys 16 (lane / 16) .. + 15 of the tile
    template <int NV>
    __device__ __forceinline__ void load_v(int key0, i32x4 (&v)[NV]) const {
        int off;
        const int64_t at = base(key0 + 16 * (lane >> 4), off);
        const int page = 1 << a.c.log2_page;
        const int8_t* p = a.c.v + at + off;
#pragma unroll
        for (int ct = 0; ct < NV; ++ct) {
            const int ch = 16 * ct + (lane & 15);
            v[ct] = ch < a.c.d ? *reinterpret_cast<const i32x4*>(p + (int64_t)ch * page) : i32x4{0, 0, 0, 0};
        }
    }
};

__device__ __forceinline__ i32x4 mfma(i32x4 x, i32x4 y, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(x, y, c, 0, 0, 0);
}

__device__ __forceinline__ i32x4 splat(int v) { return i32x4{v, v, v, v}; }

template <int RS, int KS>
struct Queries {
    Operand<KS> q[RS];
    int zp0, zp1;           // -zp_q in two terms that are bytes

    __device__ __forceinline__ void load(const PagedArgs& a, int b, int h, int row0, int rows, int lane) {
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            const int rho = min(row0 + 16 * s + (lane & 15), rows - 1);
            const int8_t* p = a.q + query_of(a, b, h, rho) * a.c.d;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int at = 64 * k + 16 * (lane >> 4);
                q[s].w[k] = at < a.c.d ? *reinterpret_cast<const i32x4*>(p + at) : i32x4{0, 0, 0, 0};
            }
        }
        zp0 = min(-a.zp_q, 127);
        zp1 = -a.zp_q - zp0;        // 128 = 127 + 1
    }

    // logits of 64 keys plus the row's `add`: acc[s][t][i] is key 16 (lane / 16) + 4 t + i
    // of row lane % 16
    __device__ __forceinline__ void logits(const Operand<KS> (&k)[4], const i32x4 (&add)[RS],
                                           i32x4 (&acc)[RS][4]) const {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int s = 0; s < RS; ++s) {
                acc[s][t] = add[s];
#pragma unroll
                for (int x = 0; x < KS; ++x) acc[s][t] = mfma(k[t].w[x], q[s].w[x], acc[s][t]);
            }
        }
        if (zp0) {
            const i32x4 z0 = splat((zp0 & 0xFF) * 0x01010101), z1 = splat(zp1 * 0x01010101);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int s = 0; s < RS; ++s)
#pragma unroll
                    for (int x = 0; x < KS; ++x) {
                        acc[s][t] = mfma(k[t].w[x], z0, acc[s][t]);
                        if (zp1) acc[s][t] = mfma(k[t].w[x], z1, acc[s][t]);
                    }
        }
    }
};

// Whether a row of this limit sees key 4 t + i of the lane's 16 keys of a tile.
__device__ __forceinline__ bool seen(int key0, int t, int i, int limit, int lane) {
    return key0 + 16 * (lane >> 4) + 4 * t + i < limit;
}

// ---------------------------------------------------------------------------
// Thresholds
// ---------------------------------------------------------------------------

// U_k: the least u in [0, n d] with c_k e(u) <= 2 S; n d + 1 where there is none.
// With u = z d + rho, e = ((q_b - rho)^2 + q_c) 2^(n - z): the octave z is the first whose
// last value satisfies it, the place in it an integer square root.
__device__ int threshold(uint64_t S2, int k, const LisConsts& c) {
    const uint32_t ck = k == 1 ? 3u : (3u << (k - 1)) - 1u;
    const uint32_t wl = c.qb - c.d_ln2 + 1, last = wl * wl + c.qc, first = c.qb * c.qb + c.qc;
    const auto fits = [&](int z) { return (uint64_t)last * ck <= (S2 >> (c.n - z)); };
    // an estimate of z, then exactly
    const float f = (float)S2 / ((float)last * (float)ck);
    int z = min(max(c.n - ((int)(__float_as_uint(f) >> 23) - 127), 0), c.n);
    while (z < c.n && !fits(z)) ++z;
    while (z > 0 && fits(z - 1)) --z;
    const uint64_t X = S2 >> (c.n - z);
    if (z == c.n) return (uint64_t)first * ck <= X ? c.n * (int)c.d_ln2 : c.n * (int)c.d_ln2 + 1;
    if ((uint64_t)first * ck <= X) return z * (int)c.d_ln2;
    // (q_b - rho)^2 <= floor(X / c_k) - q_c; X < first c_k < 2^40, and X / c_k lies at
    // least 1 / c_k below the next integer: its binary64 quotient has the right floor
    const uint32_t y = (uint32_t)((double)X / (double)ck) - c.qc;
    uint32_t w = (uint32_t)sqrtf((float)y);
    while (w * w > y) --w;
    while ((w + 1) * (w + 1) <= y) ++w;
    return z * (int)c.d_ln2 + (int)(c.qb - w);
}

// The words of a row's buckets, by the threads of a workgroup: bucket j >= 1 holds
// u in ((j - 1) 2^shift, j 2^shift], bucket 0 u = 0.  They are stored backwards, so that
// -u >> shift is the distance from the end; rows are 16 words apart.
constexpr int kMaxTop = 15;

__device__ __forceinline__ void fill_buckets(const int* U, int k, int top, int shift, int buckets,
                                             uint32_t* words) {
    // bucket j's code at its first u is the number of thresholds up to it: k for the
    // buckets from the first whose first u reaches U_k to the one before U_(k+1)'s
    const int u0 = k == 0 ? 0 : U[k - 1], u1 = k == top ? INT_MAX : U[k];
    const auto from = [&](int u) { return u <= 0 ? 0 : (int)(((uint32_t)(u - 1) + (1u << shift) - 1) >> shift) + 1; };
    const int end = u1 == INT_MAX ? buckets : min(from(u1), buckets);
    for (int j = k == 0 ? 0 : from(u0); j < end; ++j) {
        const int stop = (j << shift) + 1;          // behind the bucket's last u
        words[16 * (buckets - 1 - j)] = ((uint32_t)(top - k) << 24) + (uint32_t)(min(u1, stop) - 1);
    }
}

// ---------------------------------------------------------------------------
// The three passes
// ---------------------------------------------------------------------------

// Exact row sum from values e 2^-n held in binary32: the 16 values of a tile are added
// in binary64 to 2^(52 - n), whose unit is 2^-n; the sum's low bits are then their sum
// as an integer (16 2^24 2^n < 2^52: n <= 23; deeper clamps take the general path).
template <bool FAST>
struct RowAdder {
    uint64_t sum = 0;

    // P0: the I-Exp needs no pre-shift (q_ln2 above 512)
    template <bool P0>
    __device__ __forceinline__ void fast(const i32x4 (&acc)[4], const PagedArgs& a, bool edge, int key0,
                                         int limit, int lane) {
        const double unit = __longlong_as_double((int64_t)(1023 + 52 - a.k.n) << 52);
        double s0 = unit, s1 = unit;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t e = lis::screen_iexp<P0>(acc[t][i], 0, a.k);       // the row's offset is in acc
                if (edge) e = seen(key0, t, i, limit, lane) ? e : 0u;
                if (i & 1) s1 += (double)__uint_as_float(e);
                else s0 += (double)__uint_as_float(e);
            }
        const uint64_t m = (1ull << 52) - 1;
        sum += ((uint64_t)__double_as_longlong(s0) & m) + ((uint64_t)__double_as_longlong(s1) & m);
    }

    __device__ __forceinline__ void add(const i32x4 (&acc)[4], int mx, const PagedArgs& a, bool edge,
                                        int key0, int limit, int lane) {
        if constexpr (FAST) {
            if (a.k.s_pre == 0) fast<true>(acc, a, edge, key0, limit, lane);
            else fast<false>(acc, a, edge, key0, limit, lane);
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t z;
                    const uint32_t qL = lis::iexp_qL(acc[t][i], mx, a.k, z);
                    sum += !edge || seen(key0, t, i, limit, lane) ? (uint64_t)qL << (a.k.n - (int)z) : 0;
                }
        }
    }
};

// Bytes 0..3 of the result: byte 3 of each word.
__device__ __forceinline__ uint32_t top_bytes(uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) {
    return __builtin_amdgcn_perm(x1, x0, 0x0c0c0703u) | __builtin_amdgcn_perm(x3, x2, 0x07030c0cu);
}

// Four weights 2^m from the bytes m: their operands hi and lo.
__device__ __forceinline__ void digits(uint32_t m, uint32_t& hi, uint32_t& lo) {
    const uint32_t v = __builtin_amdgcn_perm(0x80C0E0F0u, 0xF8FCFEFFu, m & 0x07070707u);
    const uint32_t up = __builtin_amdgcn_perm(0u, 0x0000FF00u, (m >> 3) & 0x01010101u);
    hi = v & up;
    lo = v & ~up;
}

template <int RS, int KS, int NV, Pass PASS, bool STORED, bool FAST, bool WEIGHT>
__global__ __launch_bounds__(kBlock, 2) void lis_paged_kernel(PagedArgs a, Shape sh) {
    constexpr int kRows = 16 * RS;
    extern __shared__ uint32_t dyn[];               // buckets, then the workgroup's out
    __shared__ int row_max[kRows * kWaves];
    __shared__ unsigned long long row_sum[kRows * kWaves];
    __shared__ int U[kRows * kWaves][kMaxTop];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int RG = sh.row_groups, KG = kWaves / RG;
    const int rg = wave / KG, kg = wave - rg * KG;
    const int tile_rows = RG * kRows;
    // fewer than 2^24 workgroups: 32-bit divisions
    const uint32_t block = (uint32_t)lis::xcd_remap(blockIdx.x, gridDim.x);
    const uint32_t wg = block / (uint32_t)sh.splits;
    const int split = (int)(block - wg * (uint32_t)sh.splits);
    const int64_t unit = wg / (uint32_t)sh.tiles;
    const int tile = sh.tiles - 1 - (int)(wg - (uint32_t)unit * (uint32_t)sh.tiles);    // the rows that see most come first
    const int b = (int)((uint32_t)unit / (uint32_t)a.c.Hkv), h = (int)unit - b * a.c.Hkv;
    const int len = keys_of(a.c, b);
    const int fresh = a.n_new ? min(max(a.n_new[b], 0), a.L) : a.L;
    const int rows = fresh * a.group;
    const int first = tile * tile_rows;             // the workgroup's first row
    if (first >= rows) return;
    const int row0 = first + rg * kRows;            // the wavefront's
    const bool idle = row0 >= rows;

    int limit[RS];
#pragma unroll
    for (int s = 0; s < RS; ++s) limit[s] = limit_of(a, len, fresh, min(row0 + 16 * s + (lane & 15), rows - 1));
    // keys that some row of the wavefront sees, that every one does, and that some row of the workgroup does
    const int full = limit_of(a, len, fresh, min(row0, rows - 1));
    const int all = limit_of(a, len, fresh, min(first + tile_rows, rows) - 1);
    const int per = ((all + kTile - 1) / kTile + sh.splits - 1) / sh.splits * kTile;
    const int from = min(split * per, all);
    const int to = idle ? 0 : min(from + per, limit_of(a, len, fresh, min(row0 + kRows, rows) - 1));
    const int key_first = from + kg * kTile, key_step = KG * kTile;

    Queries<RS, KS> q;
    const Keys<KS> keys{a, b, h, len, lane};
    if (!STORED || PASS != kOut) q.load(a, b, h, min(row0, rows - 1), rows, lane);
    int32_t* lg = nullptr;
    if (STORED) lg = sh.logits + (unit * sh.rows + min(lane & 15, sh.rows - 1)) * sh.keys + 16 * (lane >> 4);

    // body(key0, logits + add, edge) for each of the wavefront's tiles
    const auto walk = [&](const i32x4 (&add)[RS], auto&& body) {
        if (key_first >= to) return;
        Operand<KS> k[4];
        const int8_t* next = keys.k_rows(key_first);
        keys.load_k(next, k);
        next = keys.k_rows(key_first + key_step);
        for (int key0 = key_first; key0 < to; key0 += key_step) {
            Operand<KS> kn[4];
            keys.load_k(next, kn);
            next = keys.k_rows(key0 + 2 * key_step);
            i32x4 acc[RS][4];
            q.logits(k, add, acc);
            body(key0, acc, key0 + kTile > full);
#pragma unroll
            for (int t = 0; t < 4; ++t) k[t] = kn[t];
        }
    };

    const int64_t part0 = ((unit * sh.tiles + tile) * sh.splits) * tile_rows;
    i32x4 add[RS];

    // --- maximum
    for (int i = threadIdx.x; i < tile_rows; i += kBlock) {
        row_max[i] = INT_MIN;
        row_sum[i] = 0;
    }
    __syncthreads();
    if (PASS == kAll || PASS == kMax) {
        int mx[RS];
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            mx[s] = INT_MIN;
            add[s] = splat(0);
        }
        walk(add, [&](int key0, const i32x4 (&acc)[RS][4], bool edge) {
#pragma unroll
            for (int s = 0; s < RS; ++s)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    if (!edge) {
                        mx[s] = max(max(max(mx[s], acc[s][t][0]), acc[s][t][1]), max(acc[s][t][2], acc[s][t][3]));
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            mx[s] = max(mx[s], seen(key0, t, i, limit[s], lane) ? acc[s][t][i] : INT_MIN);
                    }
                    if (STORED && s == 0 && (lane & 15) < sh.rows)
                        *reinterpret_cast<i32x4*>(lg + key0 + 4 * t) = acc[s][t];
                }
        });
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            const int m = lis::row4_max(mx[s]);
            if (lane < 16) atomicMax(&row_max[rg * kRows + 16 * s + lane], m);
        }
        __syncthreads();
        if (PASS == kMax) {
            for (int i = threadIdx.x; i < tile_rows; i += kBlock)
                sh.part_max[part0 + (int64_t)split * tile_rows + i] = row_max[i];
            if (split == 0)         // the parts of the last pass add to it
                for (int at = threadIdx.x; at < tile_rows * (a.c.d >> 2); at += kBlock) {
                    const int r = at / (a.c.d >> 2), ch = at - r * (a.c.d >> 2);
                    if (first + r < rows)
                        *reinterpret_cast<i32x4*>(a.out + query_of(a, b, h, first + r) * a.c.d + 4 * ch) = splat(0);
                }
            return;
        }
    } else {
        for (int at = threadIdx.x; at < tile_rows * sh.splits; at += kBlock)
            atomicMax(&row_max[at % tile_rows], sh.part_max[part0 + at]);
        __syncthreads();
    }

    // --- sum
    int mx[RS];
#pragma unroll
    for (int s = 0; s < RS; ++s) mx[s] = row_max[rg * kRows + 16 * s + (lane & 15)];
    if (PASS == kAll || PASS == kSum) {
        RowAdder<FAST> sum[RS];
#pragma unroll
        for (int s = 0; s < RS; ++s) add[s] = splat(FAST ? -lis::screen_c(mx[s], a.k) : 0);
        walk(add, [&](int key0, const i32x4 (&acc)[RS][4], bool edge) {
#pragma unroll
            for (int s = 0; s < RS; ++s) {
                if (edge) sum[s].add(acc[s], mx[s], a, true, key0, limit[s], lane);
                else sum[s].add(acc[s], mx[s], a, false, key0, limit[s], lane);
            }
        });
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            const uint64_t v = lis::row4_sum(sum[s].sum);
            if (lane < 16) atomicAdd(&row_sum[rg * kRows + 16 * s + lane], (unsigned long long)v);
        }
        __syncthreads();
        if (PASS == kSum) {
            for (int i = threadIdx.x; i < tile_rows; i += kBlock)
                sh.part_sum[part0 + (int64_t)split * tile_rows + i] = row_sum[i];
            return;
        }
    } else {
        for (int at = threadIdx.x; at < tile_rows * sh.splits; at += kBlock)
            atomicAdd(&row_sum[at % tile_rows], (unsigned long long)sh.part_sum[part0 + at]);
        __syncthreads();
    }

    // --- thresholds
    const int out_at = FAST ? tile_rows * sh.buckets : 0;
    const bool shared_out = KG > 1 || PASS == kOut;
    int32_t* wg_out = reinterpret_cast<int32_t*>(dyn + out_at);
    if (shared_out)
        for (int i = threadIdx.x; i < tile_rows * a.c.d; i += kBlock) wg_out[i] = 0;
    lis::RowSum rs[RS];
    if (FAST) {
        for (int at = threadIdx.x; at < tile_rows * a.k.top; at += kBlock) {
            const int r = at % tile_rows, k = at / tile_rows;
            U[r][k] = threshold(2 * row_sum[r], k + 1, a.k);
        }
        __syncthreads();
        for (int at = threadIdx.x; at < tile_rows * (a.k.top + 1); at += kBlock) {
            const int r = at % tile_rows, k = at / tile_rows;
            fill_buckets(U[r], k, a.k.top, sh.shift, sh.buckets, dyn + (r >> 4) * (16 * sh.buckets) + (r & 15));
        }
    } else {
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            rs[s].S2 = 2 * row_sum[rg * kRows + 16 * s + (lane & 15)];
            rs[s].rc = (63 - __clzll((long long)rs[s].S2)) - 31 - a.k.n;
        }
    }
    __syncthreads();

    // --- codes and product
    i32x4 hi[RS][NV] = {}, lo[RS][NV] = {}, ph[RS] = {}, pl[RS] = {};
    const i32x4 ones = splat(0x01010101);
    const int cap = min(a.k.n, a.k.top) * (int)a.k.d_ln2;
    const auto product = [&](int key0, const i32x4 (&acc)[RS][4], bool edge) {
        i32x4 v[NV];
        keys.load_v(key0, v);
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            uint32_t m[4];
            const uint32_t* end = dyn + (rg * RS + s) * (16 * sh.buckets) + 16 * (sh.buckets - 1) + (lane & 15);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                uint32_t x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (FAST) {
                        // -u; a key that the row does not see may lie above its maximum
                        int u;
                        asm("v_med3_i32 %0, %1, %2, 0" : "=v"(u) : "v"(acc[s][t][i]), "s"(-cap));
                        x[i] = end[(u >> sh.shift) * 16] + (uint32_t)u;
                    } else {
                        uint32_t z;
                        const uint32_t qL = lis::iexp_qL(acc[s][t][i], mx[s], a.k, z);
                        x[i] = (uint32_t)(a.k.top - lis::lis_code(qL, z, rs[s], a.k)) << 24;
                    }
                }
                m[t] = top_bytes(x[0], x[1], x[2], x[3]);
            }
            i32x4 wh, wl;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                uint32_t dh, dl;
                digits(m[t], dh, dl);
                if (edge) {
                    uint32_t keep = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        keep |= seen(key0, t, i, limit[s], lane) ? 0xFFu << (8 * i) : 0u;
                    dh &= keep;
                    dl &= keep;
                }
                wh[t] = (int)dh;
                wl[t] = (int)dl;
            }
#pragma unroll
            for (int ct = 0; ct < NV; ++ct) {
                hi[s][ct] = mfma(v[ct], wh, hi[s][ct]);
                lo[s][ct] = mfma(v[ct], wl, lo[s][ct]);
            }
            if (a.zp_v) {
                ph[s] = mfma(ones, wh, ph[s]);
                pl[s] = mfma(ones, wl, pl[s]);
            }
            if (WEIGHT) {
                const bool mine = row0 + 16 * s + (lane & 15) < rows;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int8_t bh = (int8_t)((uint32_t)wh[e >> 2] >> (8 * (e & 3)));
                    const int8_t bl = (int8_t)((uint32_t)wl[e >> 2] >> (8 * (e & 3)));
                    int p = mine ? -(256 * bh + bl) : 0;
#pragma unroll
                    for (int o = 1; o < 16; o <<= 1) p += __shfl_xor(p, o);
                    const int key = key0 + 16 * (lane >> 4) + e;
                    if ((lane & 15) == e && key < len && p) {
                        const int id = page_at(a.c.table, a.c.max_pages, a.c.pages, b, key >> a.c.log2_page);
                        atomicAdd(reinterpret_cast<unsigned long long*>(a.c.weight) +
                                      (((int64_t)id * a.c.Hkv + h) << a.c.log2_page) +
                                      (key & ((1 << a.c.log2_page) - 1)),
                                  (unsigned long long)p);
                    }
                }
            }
        }
    };
#pragma unroll
    for (int s = 0; s < RS; ++s) add[s] = splat(FAST ? -mx[s] : 0);
    if (STORED && PASS == kOut) {
        for (int key0 = key_first; key0 < to; key0 += key_step) {
            i32x4 acc[RS][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                acc[0][t] = *reinterpret_cast<const i32x4*>(lg + key0 + 4 * t);
                if (FAST) acc[0][t] += add[0];
            }
            product(key0, acc, key0 + kTile > full);
        }
    } else {
        walk(add, product);
    }

    // --- out
#pragma unroll
    for (int s = 0; s < RS; ++s) {
        const int rho = row0 + 16 * s + (lane & 15);
        if (rho >= rows) continue;
        int32_t* out = a.out + query_of(a, b, h, rho) * a.c.d;
#pragma unroll
        for (int ct = 0; ct < NV; ++ct) {
            const int ch = 16 * ct + 4 * (lane >> 4);
            if (ch >= a.c.d) continue;
            i32x4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                o[i] = a.zp_v * (ph[s][i] * 256 + pl[s][i]) - (hi[s][ct][i] * 256 + lo[s][ct][i]);
            if (shared_out) {
#pragma unroll
                for (int i = 0; i < 4; ++i) atomicAdd(&wg_out[(rho - first) * a.c.d + ch + i], o[i]);
            } else {
                *reinterpret_cast<i32x4*>(out + ch) = o;
            }
        }
    }
    if (!shared_out) return;
    __syncthreads();
    for (int at = threadIdx.x; at < tile_rows * a.c.d; at += kBlock) {
        const int r = at / a.c.d, ch = at - r * a.c.d;
        if (first + r >= rows) break;
        int32_t* out = a.out + query_of(a, b, h, first + r) * a.c.d + ch;
        if (PASS == kOut) atomicAdd(out, wg_out[at]);
        else *out = wg_out[at];
    }
}

// Sums of a part of the stored logits: a wavefront takes 256 keys of a row at a time,
// every lane four of them.
template <bool FAST>
__global__ __launch_bounds__(kBlock) void lis_paged_sum_kernel(PagedArgs a, Shape sh) {
    __shared__ int row_max[16];
    __shared__ unsigned long long row_sum[16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t block = (uint32_t)lis::xcd_remap(blockIdx.x, gridDim.x);
    const int64_t unit = block / (uint32_t)sh.splits;
    const int split = (int)(block - (uint32_t)unit * (uint32_t)sh.splits);
    const int b = (int)((uint32_t)unit / (uint32_t)a.c.Hkv);
    const int len = keys_of(a.c, b);
    const int fresh = a.n_new ? min(max(a.n_new[b], 0), a.L) : a.L;
    const int rows = fresh * a.group;
    if (rows == 0) return;
    const int all = limit_of(a, len, fresh, rows - 1);
    const int per = ((all + kTile - 1) / kTile + sh.splits - 1) / sh.splits * kTile;
    const int from = min(split * per, all), to = min(from + per, all);
    const int64_t part0 = unit * sh.splits * 16;
    if (threadIdx.x < 16) {
        row_max[threadIdx.x] = INT_MIN;
        row_sum[threadIdx.x] = 0;
    }
    __syncthreads();
    for (int at = threadIdx.x; at < 16 * sh.splits; at += kBlock)
        atomicMax(&row_max[at % 16], sh.part_max[part0 + at]);
    __syncthreads();
    const int runs = (to - from + 255) / 256;
    for (int at = wave; at < rows * runs; at += kWaves) {
        const int r = at / runs, key0 = from + 256 * (at - r * runs) + 4 * lane;
        const int end = min(to, limit_of(a, len, fresh, r));
        uint64_t sum = 0;
        if (key0 < end) {
            const i32x4 v = *reinterpret_cast<const i32x4*>(sh.logits + (unit * sh.rows + r) * sh.keys + key0);
            const int c = lis::screen_c(row_max[r], a.k);
            const double unit_n = __longlong_as_double((int64_t)(1023 + 52 - a.k.n) << 52);
            double s = unit_n;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (FAST) {
                    const uint32_t e = key0 + i < end ? lis::screen_iexp(v[i], c, a.k) : 0u;
                    s += (double)__uint_as_float(e);
                } else {
                    uint32_t z;
                    const uint32_t qL = lis::iexp_qL(v[i], row_max[r], a.k, z);
                    sum += key0 + i < end ? (uint64_t)qL << (a.k.n - (int)z) : 0;
                }
            }
            if (FAST) sum = (uint64_t)__double_as_longlong(s) & ((1ull << 52) - 1);
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
        if (lane == 0) atomicAdd(&row_sum[r], (unsigned long long)sum);
    }
    __syncthreads();
    if (threadIdx.x < 16) sh.part_sum[part0 + (int64_t)split * 16 + threadIdx.x] = row_sum[threadIdx.x];
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------

// Whether the thresholds and the binary32 I-Exp hold for these constants: q_L below
// 2^24 (which keeps d below 2^11), e(u) not increasing over an octave's end, buckets of
// at least 8 values, and the sums of a tile below 2^52.
bool fast_path(const LisConsts& k) {
    const uint64_t first = (uint64_t)k.qb * k.qb + k.qc;
    const uint64_t w = k.qb - k.d_ln2 + 1, last = w * w + k.qc;
    return first < (1u << 24) && 2 * last >= first && k.d_ln2 >= 16 && k.n <= 23;
}

template <int RS, int KS, int NV, Pass PASS, bool STORED>
void enqueue(const PagedArgs& a, const Shape& sh, const Plan& p, bool fast, hipStream_t stream) {
    const bool last = PASS == kAll || PASS == kOut;
    const bool shared_out = last && (p.row_groups < kWaves || PASS == kOut);
    const size_t lds = 4 * ((last && fast ? (size_t)p.tile_rows() * sh.buckets : 0) +
                            (shared_out ? (size_t)p.tile_rows() * a.c.d : 0));
    constexpr bool kWeight = PASS == kAll || PASS == kOut;
    const bool weight = kWeight && a.c.weight;
    launch_kernel(fast ? (weight ? lis_paged_kernel<RS, KS, NV, PASS, STORED, true, kWeight>
                                 : lis_paged_kernel<RS, KS, NV, PASS, STORED, true, false>)
                       : (weight ? lis_paged_kernel<RS, KS, NV, PASS, STORED, false, kWeight>
                                 : lis_paged_kernel<RS, KS, NV, PASS, STORED, false, false>),
                  dim3((uint32_t)(p.units * p.tiles * p.splits)), dim3(kBlock), lds, stream, a, sh);
}

// RS: sets of rows a wavefront holds where there are more than 16 rows
template <int RS, int KS, int NV>
void launch(const PagedArgs& a, const Shape& sh, const Plan& p, hipStream_t stream) {
    const bool fast = fast_path(a.k);
    if (p.splits == 1) {
        if (p.sets == 1) enqueue<1, KS, NV, kAll, false>(a, sh, p, fast, stream);
        else enqueue<RS, KS, NV, kAll, false>(a, sh, p, fast, stream);
        return;
    }
    const LaunchEvents ev = launch_events();
    set_launch_events(ev.start, nullptr);
    if (p.stored) enqueue<1, KS, NV, kMax, true>(a, sh, p, fast, stream);
    else enqueue<RS, KS, NV, kMax, false>(a, sh, p, fast, stream);
    set_launch_events(nullptr, nullptr);
    if (p.stored)
        launch_kernel(fast ? lis_paged_sum_kernel<true> : lis_paged_sum_kernel<false>,
                      dim3((uint32_t)(p.units * p.splits)), dim3(kBlock), 0, stream, a, sh);
    else enqueue<RS, KS, NV, kSum, false>(a, sh, p, fast, stream);
    set_launch_events(nullptr, ev.stop);
    if (p.stored) enqueue<1, KS, NV, kOut, true>(a, sh, p, fast, stream);
    else enqueue<RS, KS, NV, kOut, false>(a, sh, p, fast, stream);
}

}  // namespace

#if defined(FQ_PAGED_32)
void launch_lis_paged_32(const PagedArgs& a, const paged::Shape& sh, const paged::Plan& p, hipStream_t s) { launch<2, 1, 2>(a, sh, p, s); }
#elif defined(FQ_PAGED_64)
void launch_lis_paged_64(const PagedArgs& a, const paged::Shape& sh, const paged::Plan& p, hipStream_t s) { launch<2, 1, 4>(a, sh, p, s); }
#elif defined(FQ_PAGED_128)
void launch_lis_paged_128(const PagedArgs& a, const paged::Shape& sh, const paged::Plan& p, hipStream_t s) { launch<1, 2, 8>(a, sh, p, s); }
#else
void launch_lis_paged_32(const PagedArgs& a, const paged::Shape& sh, const paged::Plan& p, hipStream_t s);
void launch_lis_paged_64(const PagedArgs& a, const paged::Shape& sh, const paged::Plan& p, hipStream_t s);
void launch_lis_paged_128(const PagedArgs& a, const paged::Shape& sh, const paged::Plan& p, hipStream_t s);

size_t lis_paged_workspace(int32_t B, int32_t Hq, int32_t Hkv, int32_t L, int32_t d,
                           int64_t max_keys) {
    return paged::plan(B, Hq, Hkv, L, d, max_keys).bytes();
}

hipError_t launch_lis_paged(const PagedArgs& a, hipStream_t stream) {
    const Plan p = paged::plan(a.c.B, a.Hq, a.c.Hkv, a.L, a.c.d, (int64_t)a.c.max_pages << a.c.log2_page);
    Shape sh{};
    sh.splits = p.splits;
    sh.row_groups = p.row_groups;
    sh.tiles = p.tiles;
    sh.rows = p.rows;
    sh.keys = p.keys;
    // the sums first: they need the largest alignment
    sh.part_sum = static_cast<uint64_t*>(a.workspace);
    sh.part_max = reinterpret_cast<int32_t*>(sh.part_sum + p.partials());
    sh.logits = sh.part_max + (p.partials() + 3) / 4 * 4;
    while ((2u << sh.shift) * 2 <= a.k.d_ln2) ++sh.shift;       // 2^shift <= q_ln2 / 2
    const int cap = (a.k.n < a.k.top ? a.k.n : a.k.top) * (int)a.k.d_ln2;
    sh.buckets = ((cap - 1) >> sh.shift) + 2;
    if (a.c.d <= 32) launch_lis_paged_32(a, sh, p, stream);
    else if (a.c.d <= 64) launch_lis_paged_64(a, sh, p, stream);
    else launch_lis_paged_128(a, sh, p, stream);
    return hipGetLastError();
}
#endif

}  // namespace fqvit
