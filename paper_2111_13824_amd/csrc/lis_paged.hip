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
// the cache holds values with their channels in rows.
//
// Tiles of keys and values come into LDS in the order of memory, a stage of a few tiles at
// a time: two stages there, two more on their way in registers.  A workgroup's wavefronts
// share them.  (Loaded straight into the operands' registers, 16 neighbouring lanes read 16
// rows: 8 chunks of 16 heads over up to 4096 keys took 214 us, 167 so; vector
// instructions were a third of the former.)
//
// A weight P = 2^m, m = (2^b - 1) - code in [0, 15], is not an int8: it is taken as
// -256 hi - lo with hi, lo in {0, -1, -2, .. -128}, two products with the same V
// operand, exact in int32.
//
// The row's maximum is needed before the first I-Exp, its exact sum before the first
// code: three passes over the keys.  The matrix cores are far from busy (a logit costs
// them less than one vector instruction), so each pass takes the logits again; a call
// of at most 16 rows a key head, which the keys' bytes bound, stores them instead where
// they fit.
//
// Measured.  Chunks (8 of up to 512 tokens and 16 heads of 64, 4096 keys): 139 to 158 us by
// their lengths, 36 GOP; bound by vector instructions, 45 million, which are 73 us of issue:
// about half of the time, as the shorter sequences' workgroups end before the
// longest.  One token of 64 streams (4096 keys, 4 key heads
// of 64): 29 us, 3.5 TB/s of the 5.2 that a copy reaches; workgroups of one compute unit
// read at the same time and then compute at the same time.  One token of a stream of 197 keys:
// 10 us, a chain of loads and barriers.  One token of 131072 keys (4 key heads of 128): 45 us,
// three launches of 18, 7 and 20.
//
// Codes without I-Exp.  e(u), u = max - logit, does not increase with u (the host
// checks the one place where rounding could make it, the end of an octave), so
// code >= k, c_k e(u) <= 2 S (c_1 = 3, c_k = 3 2^(k-1) - 1), is u >= U_k for 2^b - 1
// integers U_k of the row.  They are found exactly, once a row.  U_1 exists, and
// U_(k+1) - U_k is at least q_ln2 for k >= 2 where U_k is not 0 (e(u + q_ln2) = e(u) / 2,
// c_(k+1) = 2 c_k + 1).  Buckets of 2^shift <= q_ln2 values of u from U_1 on hold
// at most one threshold behind their first value (the first one U_2, the others none
// closer), and one word of a bucket, E = 2^24 (2^b - 1 - c) + th - U_1 with c the code at its
// first u and th the next threshold (or the bucket's end), gives m = (E + U_1 - 1 - u) >> 24.
// U_1 - 1 - max is in the product's accumulators from the start; a code is a clamp, two
// steps of an address, an LDS read and an addition, where the I-Exp and comparisons with S
// are about thirty instructions.  Every lane has words of its own in its own LDS bank (one
// table for a row's four lanes met five cycles of bank conflicts a read, and LDS bound
// the pass).
#include <algorithm>

#include "cache_device.h"
#include "fqvit_launch.h"
#include "lis_device.h"
#include "lis_paged_plan.h"

namespace fqvit {
namespace {

using cache::first_new;
using cache::head_base;
using cache::keys_of;
using cache::page_at;
using paged::kTile;
using paged::Plan;
using paged::Shape;

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 256;         // of the sums over stored logits

// Passes of a launch: all of them, or one where the keys are divided.
enum Pass { kAll, kMax, kSum, kOut };
// Arithmetic: 64-bit steps of any constants; thresholds and the binary32 I-Exp; the same
// without its pre-shift (q_ln2 above 512).
enum Mode { kGeneral, kShifted, kPlain };

// Row rho of a sequence and head is query (token rho / group, head rho % group).
__device__ __forceinline__ int64_t query_of(const PagedArgs& a, int b, int h, int rho) {
    const int i = rho / a.group, g = rho - i * a.group;
    return ((int64_t)b * a.Hq + h * a.group + g) * a.L + i;
}

// Keys that row rho sees, of `len`; `past`: the place of the first new token.
__device__ __forceinline__ int limit_of(const PagedArgs& a, int len, int past, int rho) {
    return a.causal ? min(max(past + rho / a.group + 1, 0), len) : len;
}

// What a workgroup works on.  Its unit, a sequence's key head, runs on one XCD, whose L2
// then holds the keys that the unit's workgroups share; eight units in a row go to the
// eight XCDs, and the longest sequences come first (of at most 64): the last workgroups to
// start are short ones.  (Units in order, a run of them an XCD, left the XCD of the longest
// sequence alone for the last third of the time; always in the same direction, the
// first XCDs had the longer ones of each eight: 8 chunks over up to 4096 keys 144 us for 140.)
struct Place {
    int split, tile, b, h;
    int64_t unit;
};

// FEW: at most 16 rows, whose workgroups start together or nearly; of divided keys a unit's
// parts, which add to the same few results, stay on one or two XCDs.
template <bool FEW>
__device__ __forceinline__ Place place_of(const PagedArgs& a, const Shape& sh, int lane) {
    // fewer than 2^24 workgroups: 32-bit divisions
    if (FEW) {
        const uint32_t block = (uint32_t)lis::xcd_remap(blockIdx.x, gridDim.x);
        const uint32_t u = block / (uint32_t)sh.splits;
        Place p;
        p.split = (int)(block - u * (uint32_t)sh.splits);
        p.tile = 0;
        p.h = (int)(u / (uint32_t)a.c.B);
        p.b = (int)(u - (uint32_t)p.h * (uint32_t)a.c.B);
        p.unit = (int64_t)p.b * a.c.Hkv + p.h;
        return p;
    }
    const uint32_t units = (uint32_t)a.c.B * (uint32_t)a.c.Hkv, per = (uint32_t)sh.tiles * (uint32_t)sh.splits;
    const uint32_t even = units & ~7u, block = blockIdx.x;
    uint32_t u, part;
    if (block < even * per) {
        const uint32_t i = block >> 3;
        u = i / per;
        part = i - u * per;
        u = 8 * u + (u & 1 ? 7 - (block & 7) : (block & 7));     // there and back: as much for each XCD
    } else {
        const uint32_t i = block - even * per;
        u = i / per;
        part = i - u * per;
        u += even;
    }
    Place p;
    const uint32_t tile = part / (uint32_t)sh.splits;
    p.split = (int)(part - tile * (uint32_t)sh.splits);
    p.tile = sh.tiles - 1 - (int)tile;          // the rows that see most come first
    int b = (int)(u / (uint32_t)a.c.Hkv);
    p.h = (int)(u - (uint32_t)b * (uint32_t)a.c.Hkv);
    if (a.c.B > 1 && a.c.B <= 64) {             // the sequence with b longer ones
        const int mine = lane < a.c.B ? a.c.length[lane] : INT_MIN;
        int rank = 0;
        for (int i = 0; i < a.c.B; ++i) {
            const int other = __builtin_amdgcn_readlane(mine, i);
            rank += other > mine || (other == mine && i < lane) ? 1 : 0;
        }
        const uint64_t is = __ballot(lane < a.c.B && rank == b);
        b = __ffsll((unsigned long long)is) - 1;
    }
    p.b = b;
    p.unit = (int64_t)b * a.c.Hkv + p.h;
    return p;
}

template <int KS>
struct Operand {
    i32x4 w[KS];
};

// What the workgroup's wavefronts wrote to LDS is there, what they read is free.  (Loads
// from global memory stay on their way.)
__device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Stages of KG tiles of 64 keys in LDS.  A key's row there has 4 KS units of 16 bytes; the
// unit of channels c lies at place c ^ f(key), so that 16 lanes that read one unit of the
// operand's 16 rows find it in 16 different columns of a 256-byte line; a channel's row
// of values has 4 units of 16 keys, at place p ^ (channel / 4) % 4.  Units that a head of
// d channels does not have hold others': they meet zeros of the query, or are not stored.
// Wavefront w loads part w % RG of tile w / RG.
template <int RG, int KG, int KS, int NV>
struct Stage {
    static constexpr int kKeyBytes = 4096 * KS, kValueBytes = 1024 * NV;    // of a tile
    static constexpr int kKeyLoads = 4 * KS / RG, kValueLoads = NV / RG;    // of a wavefront
    static_assert(kKeyLoads * RG == 4 * KS && kValueLoads * RG == NV, "parts are whole loads");

    // Pages of the tile's blocks of 16 keys and the blocks' first slots in them (pages of 64
    // keys and more: the first block's, which hold for all): uniform values.
    struct Blocks {
        int id[4], off[4];
    };

    const PagedArgs& a;
    int b, h, len, from, lane, wave;
    bool whole;                 // a page holds whole tiles
    int64_t head;               // bytes before the head in a page
    uint32_t stride;            // bytes of a page (at most 2^27)
    // Pages of 16 stages, block lane % 4 of stage lane / 4: the first ones, those that loads
    // are sent for, and the next.  (Scalar loads of a stage's, which the compiler moved to
    // right before their use: one token of 64 streams of 4096 keys 32.3 us, 30.3 so.)
    int first, now, then;

    __device__ __forceinline__ int key_of(int n) const { return from + 64 * (KG * n + wave / RG); }

    // an id that is no page of the cache reads as page 0
    __device__ __forceinline__ int ids(int n) const {
        const int at = min(key_of(n + (lane >> 2)) + 16 * (lane & 3), (len - 1) & ~15);     // behind the last: it again
        const int id = a.c.table[(int64_t)b * a.c.max_pages + (at >> a.c.log2_page)];
        return (uint32_t)id < (uint32_t)a.c.pages ? id : 0;
    }
    __device__ __forceinline__ void begin() {
        now = first;
        then = ids(16);
    }
    // n from 0 on, one after another
    __device__ __forceinline__ Blocks blocks(int n) {
        if (n > 0 && (n & 15) == 0) {
            now = then;
            then = ids(n + 16);
        }
        const int mask = (1 << a.c.log2_page) - 1, key0 = key_of(n), i = 4 * (n & 15);
        Blocks t;
        if (whole) {
            t.id[0] = __builtin_amdgcn_readlane(now, i);
            t.off[0] = min(key0, (len - 1) & ~63) & mask;
        } else {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                t.id[p] = __builtin_amdgcn_readlane(now, i + p);
                t.off[p] = min(key0 + 16 * p, (len - 1) & ~15) & mask;
            }
        }
        return t;
    }
    // the head's first byte in a page
    __device__ __forceinline__ int64_t base(int id) const { return head + (int64_t)((uint64_t)(uint32_t)id * stride); }

    // A stage on its way.
    struct Loads {
        i32x4 k[kKeyLoads], v[kValueLoads];
    };

    template <bool K, bool V>
    __device__ __forceinline__ void load(const Blocks& t, Loads& r) const {
        const int units = a.c.d >> 4, part = wave % RG;
        // the lane's unit of each load, less the place of the load's first key
        uint32_t k_at[kKeyLoads], v_at[kValueLoads];
#pragma unroll
        for (int i = 0; i < kKeyLoads; ++i) {
            const int j = part * kKeyLoads + i;
            const int row = KS == 1 ? lane >> 2 : 8 * (j & 1) + (lane >> 3);
            const int unit = KS == 1 ? (lane & 3) ^ j : (lane & 7) ^ (((lane >> 4) & 1) | ((j >> 1) << 1));
            k_at[i] = (uint32_t)(row * a.c.d + 16 * min(unit, units - 1));
        }
        const int p = (lane & 3) ^ ((lane >> 4) & 3);
#pragma unroll
        for (int i = 0; i < kValueLoads; ++i)
            v_at[i] = (uint32_t)min(16 * (part * kValueLoads + i) + (lane >> 2), a.c.d - 1) << a.c.log2_page;
        if (whole) {
            const int64_t page = base(t.id[0]);
            const int8_t* k = a.c.k + page + t.off[0] * a.c.d;
            const int8_t* v = a.c.v + page + t.off[0];
            if (K)
#pragma unroll
                for (int i = 0; i < kKeyLoads; ++i)
                    r.k[i] = *reinterpret_cast<const i32x4*>(
                        k + (k_at[i] + (uint32_t)((part * kKeyLoads + i) / KS * 16 * a.c.d)));
            if (V)
#pragma unroll
                for (int i = 0; i < kValueLoads; ++i)
                    r.v[i] = *reinterpret_cast<const i32x4*>(v + (v_at[i] + 16u * (uint32_t)p));
        } else {
            int64_t page[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) page[q] = base(t.id[q]);
            if (K)
#pragma unroll
                for (int i = 0; i < kKeyLoads; ++i) {
                    const int q = (part * kKeyLoads + i) / KS;
                    const int64_t even = q & 2 ? page[2] + t.off[2] * a.c.d : page[0] + t.off[0] * a.c.d;
                    const int64_t odd = q & 2 ? page[3] + t.off[3] * a.c.d : page[1] + t.off[1] * a.c.d;
                    r.k[i] = *reinterpret_cast<const i32x4*>(a.c.k + (q & 1 ? odd : even) + k_at[i]);
                }
            if (V) {
                const int64_t even = p & 2 ? page[2] + t.off[2] : page[0] + t.off[0];
                const int64_t odd = p & 2 ? page[3] + t.off[3] : page[1] + t.off[1];
                const int64_t v = p & 1 ? odd : even;
#pragma unroll
                for (int i = 0; i < kValueLoads; ++i)
                    r.v[i] = *reinterpret_cast<const i32x4*>(a.c.v + v + v_at[i]);
            }
        }
    }

    template <bool K, bool V>
    __device__ __forceinline__ void store(const Loads& r, int8_t* keys, int8_t* values) const {
        const int part = wave % RG, tile = wave / RG;
        if (K)
#pragma unroll
            for (int i = 0; i < kKeyLoads; ++i)
                *reinterpret_cast<i32x4*>(keys + kKeyBytes * tile + 1024 * (part * kKeyLoads + i) + 16 * lane) = r.k[i];
        if (V)
#pragma unroll
            for (int i = 0; i < kValueLoads; ++i)
                *reinterpret_cast<i32x4*>(values + kValueBytes * tile + 1024 * (part * kValueLoads + i) + 16 * lane) = r.v[i];
    }

    __device__ __forceinline__ void read_k(const int8_t* keys, Operand<KS> (&k)[4]) const {
        const int m = lane & 15, g = lane >> 4;
        const int f = KS == 1 ? m >> 2 : ((m >> 1) & 1) | ((m >> 2) << 1);
        const int8_t* p = keys + kKeyBytes * (wave / RG) + (16 * (m >> 2) + (m & 3)) * 64 * KS;
#pragma unroll
        for (int x = 0; x < KS; ++x)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                k[t].w[x] = *reinterpret_cast<const i32x4*>(p + 16 * ((4 * x + g) ^ f) + 256 * KS * t);
    }
    __device__ __forceinline__ void read_v(const int8_t* values, i32x4 (&v)[NV]) const {
        const int m = lane & 15, g = lane >> 4;
        const int8_t* p = values + kValueBytes * (wave / RG) + 64 * m + 16 * (g ^ (m >> 2));
#pragma unroll
        for (int ct = 0; ct < NV; ++ct) v[ct] = *reinterpret_cast<const i32x4*>(p + 1024 * ct);
    }
};

__device__ __forceinline__ i32x4 mfma(i32x4 x, i32x4 y, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(x, y, c, 0, 0, 0);
}

__device__ __forceinline__ i32x4 splat(int v) { return i32x4{v, v, v, v}; }

template <int RS, int KS>
struct Queries {
    Operand<KS> q[RS];
    int z0[KS], z1[KS];     // bytes of -zp_q in two terms, 0 behind the head's channels

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
        const int zp0 = min(-a.zp_q, 127), zp1 = -a.zp_q - zp0;    // 128 = 127 + 1
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const bool in = 64 * k + 16 * (lane >> 4) < a.c.d;
            z0[k] = in ? (zp0 & 0xFF) * 0x01010101 : 0;
            z1[k] = in ? zp1 * 0x01010101 : 0;
        }
    }

    // logits of 64 keys plus the row's `add`: acc[s][t][i] is key 16 (lane / 16) + 4 t + i
    // of row lane % 16.  SIMPLE: zp_q is not -128, and its term is taken whether it is 0 or
    // not: the matrix cores have time, a branch would part the products from what uses them.
    template <bool SIMPLE>
    __device__ __forceinline__ void logits(const Operand<KS> (&k)[4], const i32x4 (&add)[RS],
                                           i32x4 (&acc)[RS][4]) const {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int s = 0; s < RS; ++s) {
                acc[s][t] = add[s];
#pragma unroll
                for (int x = 0; x < KS; ++x) {
                    acc[s][t] = mfma(k[t].w[x], splat(z0[x]), acc[s][t]);
                    if (!SIMPLE) acc[s][t] = mfma(k[t].w[x], splat(z1[x]), acc[s][t]);
                    acc[s][t] = mfma(k[t].w[x], q[s].w[x], acc[s][t]);
                }
            }
    }
};

// How many of the lane's 16 keys of a tile a row of this limit sees (the first ones).
__device__ __forceinline__ int seen(int key0, int limit, int lane) {
    return min(max(limit - (key0 + 16 * (lane >> 4)), 0), 16);
}

// ---------------------------------------------------------------------------
// Thresholds
// ---------------------------------------------------------------------------

// U_k: the least u in [0, n d] with c_k e(u) <= 2 S; kNever where there is none.
// With u = z d + rho, e = q_L(rho) 2^(n - z), q_L(rho) = (q_b - rho)^2 + q_c: the octave z is
// the first whose last value satisfies it, n - z = floor(log2(2 S / (c_k q_L(d - 1)))),
// settled by one comparison.  In it q_b - rho = floor(sqrt(X / c_k - q_c)), X =
// floor(2 S / 2^(n - z)): from binary32 values that come within 2^-9 of it (q_L below
// 2^24, c_k below 2^16: three roundings), so that the next integer is tried, exactly.
constexpr int kNever = 1 << 20;         // above n d

__device__ __forceinline__ int threshold(uint64_t S2, int k, const LisConsts& c) {
    const uint32_t ck = k == 1 ? 3u : (3u << (k - 1)) - 1u;
    const uint32_t wl = c.qb - c.d_ln2 + 1, last = wl * wl + c.qc, first = c.qb * c.qb + c.qc;
    const uint64_t Q = (uint64_t)last * ck;
    int j = __clzll((long long)Q) - __clzll((long long)S2);         // msb(S2) - msb(Q)
    j = j >= 0 && (Q << j) > S2 ? j - 1 : j;
    const int z = c.n - min(max(j, 0), c.n);
    const uint64_t X = S2 >> (c.n - z);
    // the first value of the octave (of the last one, z = n, there is no other)
    if ((uint64_t)first * ck <= X) return z * (int)c.d_ln2;
    if (z == c.n) return kNever;
    float w = (float)X * __builtin_amdgcn_rcpf((float)ck) - (float)c.qc;
    w = __builtin_amdgcn_sqrtf(fmaxf(w, 0.0f));
    uint32_t i = (uint32_t)(w + 0.5f);      // floor or one more
    if (((uint64_t)(i * i + c.qc)) * ck > X) --i;
    return z * (int)c.d_ln2 + (int)(c.qb - i);
}

// Words of the buckets of rows whose U lies in LDS: bucket 0 holds u < U_1, bucket j >= 1
// u in [U_1 + (j - 1) 2^shift, U_1 + j 2^shift).  They lie backwards, so that
// (U_1 - 1 - u) >> shift counts from the end; a bucket's words are the 64 lanes', row
// r's at r, r + 16, r + 32, r + 48.
constexpr int kMaxTop = 15;

// Those whose first u has code k.
__device__ __forceinline__ void fill_buckets(const int* U, int k, int top, int shift, int buckets,
                                             uint32_t* words) {
    const int u1 = U[0], next = k == top ? INT_MAX : U[k];
    // the first bucket whose first u reaches u
    const auto from = [&](int u) { return u <= u1 ? 1 : ((u - u1 - 1) >> shift) + 2; };
    const int end = k == top ? buckets : min(from(next), buckets);
    for (int j = k == 0 ? 0 : from(U[k - 1]); j < (k == 0 ? 1 : end); ++j) {
        const uint32_t e = ((uint32_t)(top - k) << 24) + (j == 0 ? 0u : (uint32_t)min(next - u1, j << shift));
        uint32_t* w = words + 64 * (buckets - 1 - j);
#pragma unroll
        for (int g = 0; g < 4; ++g) w[16 * g] = e;
    }
}

// ---------------------------------------------------------------------------
// The three passes
// ---------------------------------------------------------------------------

// Exact row sum from values e 2^-n held in binary32: the 16 values of a tile are added
// in binary64 to 2^(52 - n), whose unit is 2^-n; the sum's low bits are then their sum
// as an integer (16 2^24 2^n < 2^52: n <= 23; deeper clamps take the general path).
template <Mode MODE>
struct RowAdder {
    uint64_t sum = 0;

    // a key that is not seen holds the lowest value here, is clamped to e = q_L(0) 2^-n, and
    // `unseen` of them are taken off again
    __device__ __forceinline__ void add(const i32x4 (&acc)[4], int mx, const PagedArgs& a) {
        if constexpr (MODE != kGeneral) {
            const double unit = __longlong_as_double((int64_t)(1023 + 52 - a.k.n) << 52);
            double s0 = unit, s1 = unit;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // the row's offset is in acc
                    const uint32_t e = lis::screen_iexp<MODE == kPlain>(acc[t][i], 0, a.k);
                    if (i & 1) s1 += (double)__uint_as_float(e);
                    else s0 += (double)__uint_as_float(e);
                }
            const uint64_t m = (1ull << 52) - 1;
            sum += ((uint64_t)__double_as_longlong(s0) & m) + ((uint64_t)__double_as_longlong(s1) & m);
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t z;
                    const uint32_t qL = lis::iexp_qL(acc[t][i], mx, a.k, z);
                    sum += (uint64_t)qL << (a.k.n - (int)z);
                }
        }
    }
    __device__ __forceinline__ void take_off(int unseen, const PagedArgs& a) {
        sum -= (uint64_t)unseen * (a.k.qb * a.k.qb + a.k.qc);
    }
};

// The middle one of three integers, in a form that the compiler takes as one instruction.  (Not
// inline asm: it would not wait for a matrix instruction that is still writing x.)
__device__ __forceinline__ int median(int x, int lo, int hi) {
    return max(min(x, lo), min(max(x, lo), hi));
}

// Bytes 0..3 of the result: byte 3 of each word.
__device__ __forceinline__ uint32_t top_bytes(uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) {
    return __builtin_amdgcn_perm(x1, x0, 0x0c0c0703u) | __builtin_amdgcn_perm(x3, x2, 0x07030c0cu);
}

// Four weights 2^m from the bytes m: their operands hi and lo; 0 where `keep` has no bits.
__device__ __forceinline__ void digits(uint32_t m, uint32_t keep, uint32_t& hi, uint32_t& lo) {
    const uint32_t v = __builtin_amdgcn_perm(0x80C0E0F0u, 0xF8FCFEFFu, m & 0x07070707u);
    const uint32_t up = __builtin_amdgcn_perm(0u, 0x0000FF00u, (m >> 3) & 0x01010101u);
    hi = v & up & keep;
    lo = v & ~up & keep;
}

// Sums over the 16 lanes of a block, of value e in lane e: at each step a lane hands half
// of its values to another lane and takes that one's other half.
__device__ __forceinline__ uint32_t sum16(const uint32_t (&v)[16], int lane) {
    uint32_t a[8], b[4], c[2];
    const bool b3 = lane & 8, b2 = lane & 4, b1 = lane & 2, b0 = lane & 1;
#pragma unroll
    for (int i = 0; i < 8; ++i)         // lane ^ 8
        a[i] = (b3 ? v[8 + i] : v[i]) +
               (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(b3 ? v[i] : v[8 + i]), 0x128, 0xF, 0xF, true);
#pragma unroll
    for (int i = 0; i < 4; ++i)         // lane ^ 7
        b[i] = (b2 ? a[4 + i] : a[i]) +
               (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(b2 ? a[i] : a[4 + i]), 0x141, 0xF, 0xF, true);
#pragma unroll
    for (int i = 0; i < 2; ++i)         // lane ^ 2
        c[i] = (b1 ? b[2 + i] : b[i]) +
               (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(b1 ? b[i] : b[2 + i]), 0x4E, 0xF, 0xF, true);
    return (b0 ? c[1] : c[0]) +         // lane ^ 1
           (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(b0 ? c[0] : c[1]), 0xB1, 0xF, 0xF, true);
}

// Maxima of the rows over all parts, a wavefront a row.
__device__ __forceinline__ void parts_max(const Shape& sh, int64_t row_at, int rows, int lane, int wave,
                                          int waves, int* row_max) {
    for (int r = wave; r < rows; r += waves) {
        int m = INT_MIN;
        for (int i = lane; i < sh.splits; i += 64) m = max(m, sh.part_max[(row_at + r) * sh.splits + i]);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) m = max(m, __shfl_xor(m, o));
        if (lane == 0) row_max[r] = m;
    }
}

template <int RS_, int RG_, int KG_, int KS_, int NV_>
struct Config {
    static constexpr int RS = RS_;          // sets of 16 rows of a wavefront
    static constexpr int RG = RG_, KG = KG_;    // row groups, key groups: RG KG wavefronts
    static constexpr int KS = KS_, NV = NV_;    // 64-byte steps and 16-channel tiles of a head
    static constexpr int threads = 64 * RG * KG, rows = 16 * RS * RG;
    // bytes of LDS: results of the key groups but the first, and 16 rows that a wavefront turns
    static constexpr int held = (KG - 1) * RG * RS * NV * 1024, turned = 64 * (16 * NV + 4);
};

// A sum over the lanes of a wavefront: rotations within 16 lanes, then lane swaps.
template <int CTRL>
__device__ __forceinline__ uint64_t rotated(uint64_t v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, 0xF, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, 0xF, 0xF, true);
    return ((uint64_t)hi << 32) | lo;
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {
    v += rotated<0x128>(v);
    v += rotated<0x124>(v);
    v += rotated<0x122>(v);
    v += rotated<0x121>(v);
    return lis::row4_sum(v);
}

// The I-Exp values of four stored logits of a row of maximum mx, those at `end` and behind left out.
template <bool FAST>
__device__ __forceinline__ uint64_t sum4(i32x4 v, int key0, int end, int mx, const PagedArgs& a) {
    uint64_t sum = 0;
    if (FAST) {
        const int c = lis::screen_c(mx, a.k);
        double s = __longlong_as_double((int64_t)(1023 + 52 - a.k.n) << 52);    // as in RowAdder
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t e = key0 + i < end ? lis::screen_iexp(v[i], c, a.k) : 0u;
            s += (double)__uint_as_float(e);
        }
        sum = (uint64_t)__double_as_longlong(s) & ((1ull << 52) - 1);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t z;
            const uint32_t qL = lis::iexp_qL(v[i], mx, a.k, z);
            sum += key0 + i < end ? (uint64_t)qL << (a.k.n - (int)z) : 0;
        }
    }
    return sum;
}

// Sums of stored logits: a wavefront takes runs of 256 keys of [from, to) of one row after
// another, every lane four keys of each; rows fewer than the wavefronts are shared by
// them.  done(row, sum): of what the wavefront took.  logits(row): the row's.
template <bool FAST, typename L, typename F>
__device__ __forceinline__ void sum_rows(const PagedArgs& a, int len, int past, int rows, int from, int to,
                                         int lane, int wave, int waves, const int* row_max, L&& logits, F&& done) {
    const int share = rows < waves ? waves / rows : 1;          // wavefronts a row
    const int first = share > 1 ? wave % rows : wave, part = share > 1 ? wave / rows : 0;
    if (part >= share) return;
    for (int row = first; row < rows; row += waves) {
        const int end = min(to, limit_of(a, len, past, row)), mx = row_max[row];
        const auto* p = logits(row);
        uint64_t sum = 0;
        for (int key = from + 256 * part + 4 * lane; key < end; key += 256 * share)
            sum += sum4<FAST>(*reinterpret_cast<const i32x4*>(p + key), key, end, mx, a);
        sum = wave_sum(sum);
        if (lane == 0) done(row, sum);
    }
}

// Logits between the passes: taken again, in the workspace, or in LDS.
enum Keep { kNot, kWorkspace, kLds };

template <class C, Pass PASS, Keep KEEP, Mode MODE, bool WEIGHT>
__global__ __launch_bounds__(C::threads, 2) void lis_paged_kernel(PagedArgs a, Shape sh) {
    constexpr int RS = C::RS, RG = C::RG, KG = C::KG, KS = C::KS, NV = C::NV;
    constexpr int kBlock = C::threads, tile_rows = C::rows, kRows = 16 * RS;
    constexpr bool FAST = MODE != kGeneral;
    constexpr bool VALUES = PASS == kAll || PASS == kOut;
    // passes that take the logits from the keys, and the last one's way
    constexpr bool STORED = KEEP != kNot, KEYS = !(STORED && PASS == kOut);
    typedef std::integral_constant<bool, true> Yes;
    typedef std::integral_constant<bool, false> No;
    typedef Stage<RG, KG, KS, NV> St;
    // two stages; with the logits in LDS a pass needs keys or values, not both
    constexpr int kK = KG * St::kKeyBytes, kV = KG * St::kValueBytes;
    constexpr int kStageK = !KEYS ? 16 : (KEEP == kLds ? (kK > kV ? kK : kV) : kK);
    constexpr int kStageV = !VALUES || KEEP == kLds ? 16 : kV;
    __shared__ __attribute__((aligned(16))) int8_t stage_k[2][kStageK], stage_v_[2][kStageV];
    const auto stage_v = [&](int i) { return KEEP == kLds ? stage_k[i] : stage_v_[i]; };
    extern __shared__ __attribute__((aligned(16))) uint32_t dyn[];     // buckets and logits, then the workgroup's out
    __shared__ int row_max[tile_rows];
    __shared__ unsigned long long row_sum[tile_rows];
    __shared__ int U[VALUES && FAST ? tile_rows : 1][kMaxTop];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rg = wave % RG, kg = wave / RG;
    const Place at = place_of<KEEP != kNot>(a, sh, lane);
    const int split = at.split, tile = at.tile, b = at.b, h = at.h;
    const int64_t unit = at.unit;
    const int len = keys_of(a.c, b);
    const int fresh = a.n_new ? min(max(a.n_new[b], 0), a.L) : a.L;
    const int rows = fresh * a.group, past = first_new(a.c, b, fresh);
    const int first = tile * tile_rows;             // the workgroup's first row
    if (first >= rows) return;
    const int row0 = first + rg * kRows;            // the wavefront's
    const bool idle = row0 >= rows;

    int limit[RS];
#pragma unroll
    for (int s = 0; s < RS; ++s) limit[s] = limit_of(a, len, past, min(row0 + 16 * s + (lane & 15), rows - 1));
    // keys that every row of the wavefront sees, and that some row of the workgroup does
    const int full = limit_of(a, len, past, min(row0, rows - 1));
    const int all = limit_of(a, len, past, min(first + tile_rows, rows) - 1);
    const int per = ((all + kTile - 1) / kTile + sh.splits - 1) / sh.splits * kTile;
    const int from = min(split * per, all), until = min(from + per, all);
    const int to = idle ? 0 : min(until, limit_of(a, len, past, min(row0 + kRows, rows) - 1));
    const int whole = min(full, to);                // tiles that end here or before are seen whole
    const int stages = (until - from + KG * kTile - 1) / (KG * kTile);

    Queries<RS, KS> q;
    const int64_t head_bytes = (int64_t)a.c.d << a.c.log2_page;
    St st{a, b, h, len, from, lane, wave, a.c.log2_page >= 6, h * head_bytes, (uint32_t)(a.c.Hkv * head_bytes)};
    if (stages > 0) st.first = st.ids(0);
    if (KEYS) q.load(a, b, h, min(row0, rows - 1), rows, lane);
    // the lane's row of the logits that are kept
    int32_t* const lds_logits = reinterpret_cast<int32_t*>(dyn + (FAST ? tile_rows * 4 * sh.buckets : 0));
    const int64_t lg_at = (int64_t)min(lane & 15, sh.rows - 1) * sh.keys + 16 * (lane >> 4);
    int32_t* lg = nullptr;
    if (KEEP == kWorkspace) lg = sh.logits + unit * sh.rows * sh.keys + lg_at;

    // body(key0, logits + add, values, edge) for each of the wavefront's tiles.  edge: a row
    // may not see all of it; the logits that it does not see are the lowest value.  What
    // a branch on this holds is kept to a few registers, so that the passes' sums stay
    // where they are.
    constexpr int step = KG * kTile;
    typename St::Loads r[2];
    // How many stages are on their way beside the two in LDS: values of wide heads, which a
    // wavefront of few rows loads alone, leave registers for one.
    const auto sets = [](auto values) { return decltype(values)::value && NV == 8 && RG == 1 ? 1 : 2; };
    // the first stages on their way
    const auto prime = [&](auto with_keys, auto with_values) {
        constexpr bool K = decltype(with_keys)::value, V = decltype(with_values)::value;
        if (stages == 0) return;
        st.begin();
        st.template load<K, V>(st.blocks(0), r[0]);
        if (sets(with_values) == 2) st.template load<K, V>(st.blocks(1), r[1]);
    };
    const auto walk = [&](const i32x4 (&add)[RS], auto with_keys, auto with_values, auto&& body) {
        constexpr bool K = decltype(with_keys)::value, V = decltype(with_values)::value;
        constexpr int kSets = V && NV == 8 && RG == 1 ? 1 : 2;
        if (stages == 0) return;
        const int own = from + kg * kTile;
        st.template store<K, V>(r[0], stage_k[0], stage_v(0));
        st.template load<K, V>(st.blocks(kSets), r[0]);
        meet();
        const auto stored = [&](int key0, i32x4 (&acc)[RS][4]) {
            const int k = min(key0, (int)sh.keys - kTile);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                acc[0][t] = KEEP == kLds ? *reinterpret_cast<const i32x4*>(lds_logits + lg_at + k + 4 * t)
                                         : *reinterpret_cast<const i32x4*>(lg + k + 4 * t);
        };
        i32x4 ahead[RS][4];
        if (!K && KEEP == kWorkspace) stored(own, ahead);
        const auto visit = [&](int key0, i32x4 (&acc)[RS][4], const int8_t* values) {
            const bool edge = key0 + kTile > whole;
            if (edge) {
#pragma unroll
                for (int s = 0; s < RS; ++s) {
                    const int n_seen = seen(key0, min(limit[s], to), lane);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int x = 0; x < 4; ++x) acc[s][t][x] = 4 * t + x < n_seen ? acc[s][t][x] : INT_MIN;
                }
            }
            body(key0, acc, values, edge);
        };
        // Passes over keys alone that keep nothing take the logits a stage ahead of their use,
        // and the keys come into LDS two stages ahead: reads and products hide behind
        // the vector instructions (8 chunks of 16 heads over up to 4096 keys 145 us, 143 so;
        // 154 and 149 from memory).  The last pass has no registers for it.
        constexpr bool AHEAD = K && !V && KEEP == kNot;
        i32x4 two[2][RS][4];
        Operand<KS> k[4];
        if (AHEAD) {
            st.template store<K, V>(r[1], stage_k[1], stage_v(1));
            st.template load<K, V>(st.blocks(3), r[1]);
            st.read_k(stage_k[0], k);
            q.template logits<FAST>(k, add, two[0]);
            meet();
        }
        // stage n, of parity i: the next one goes into LDS, the next that is not on its way is
        // sent for
        const auto stage = [&](int n, auto i_, auto works) {
            constexpr int i = decltype(i_)::value, into = AHEAD ? i : i ^ 1, o = kSets == 2 ? into : 0;
            const int key0 = own + n * step;
            st.template store<K, V>(r[o], stage_k[into], stage_v(into));
            i32x4 acc[RS][4];
            if (!K) {
                if (KEEP == kLds) {
                    stored(key0, acc);
                } else {
#pragma unroll
                    for (int t = 0; t < 4; ++t) acc[0][t] = ahead[0][t];
                    stored(key0 + step, ahead);
                }
            }
            st.template load<K, V>(st.blocks(n + kSets + (AHEAD ? 2 : 1)), r[o]);
            if (decltype(works)::value) {
                if constexpr (AHEAD) {
                    st.read_k(stage_k[i ^ 1], k);
                    visit(key0, two[i], stage_v(i));
                    q.template logits<FAST>(k, add, two[i ^ 1]);
                } else {
                    if (K) {
                        st.read_k(stage_k[i], k);
                        q.template logits<FAST>(k, add, acc);
                    } else {
#pragma unroll
                        for (int t = 0; t < 4; ++t) acc[0][t] += add[0];
                    }
                    visit(key0, acc, stage_v(i));
                }
            }
            meet();
        };
        const auto turns = [&](auto works) {
            int n = 0;
            for (; n + 2 <= stages; n += 2) {
                stage(n, std::integral_constant<int, 0>{}, works);
                stage(n + 1, std::integral_constant<int, 1>{}, works);
            }
            if (n < stages) stage(n, std::integral_constant<int, 0>{}, works);
        };
        if (idle) turns(std::false_type{});     // no rows of its own: it loads for the others
        else turns(std::true_type{});
    };

    // the workgroup's rows in the workspace
    const int64_t row_at = (unit * sh.tiles + tile) * tile_rows;
    i32x4 add[RS];
    prime(std::integral_constant<bool, KEYS>{}, std::integral_constant<bool, PASS == kOut>{});

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
        walk(add, Yes{}, No{}, [&](int key0, const i32x4 (&acc)[RS][4], const int8_t*, bool) {
#pragma unroll
            for (int s = 0; s < RS; ++s)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    mx[s] = max(max(max(mx[s], acc[s][t][0]), acc[s][t][1]), max(acc[s][t][2], acc[s][t][3]));
                    if (STORED && (lane & 15) < sh.rows && key0 < to)
                        *reinterpret_cast<i32x4*>((KEEP == kLds ? lds_logits + lg_at : lg) + key0 + 4 * t) = acc[s][t];
                }
        });
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            const int m = lis::row4_max(mx[s]);
            if (lane < 16) atomicMax(&row_max[rg * kRows + 16 * s + lane], m);
        }
        __syncthreads();
        if (PASS == kMax) {
            for (int i = threadIdx.x; i < tile_rows; i += kBlock) {
                sh.part_max[(row_at + i) * sh.splits + split] = row_max[i];
                if (split == 0) sh.row_sum[row_at + i] = 0;     // the parts of the next pass add to it
            }
            if (split == 0 && kg == 0)      // and those of the last one to out
#pragma unroll
                for (int s = 0; s < RS; ++s) {
                    const int rho = row0 + 16 * s + (lane & 15);
                    if (rho >= rows) continue;
                    int32_t* out = a.out + query_of(a, b, h, rho) * a.c.d;
                    for (int ch = 4 * (lane >> 4); ch < a.c.d; ch += 16)
                        *reinterpret_cast<i32x4*>(out + ch) = splat(0);
                }
            return;
        }
    } else if (PASS == kSum) {
        // a lane a row, the wavefronts share the parts (a wavefront a row took 6 us more)
        static_assert(PASS != kSum || tile_rows == 64, "a lane is a row");
        int m = INT_MIN;
        for (int i = wave; i < sh.splits; i += C::threads / 64) m = max(m, sh.part_max[(row_at + lane) * sh.splits + i]);
        atomicMax(&row_max[lane], m);
        __syncthreads();
        if (split == 0)
            for (int i = threadIdx.x; i < tile_rows; i += kBlock) sh.row_max[row_at + i] = row_max[i];
    } else {
        for (int i = threadIdx.x; i < tile_rows; i += kBlock) {
            row_max[i] = sh.row_max[row_at + i];
            row_sum[i] = sh.row_sum[row_at + i];
        }
        __syncthreads();
    }

    // --- sum
    int mx[RS];
#pragma unroll
    for (int s = 0; s < RS; ++s) mx[s] = row_max[rg * kRows + 16 * s + (lane & 15)];
    if (PASS == kAll || PASS == kSum) {
        if (KEEP == kLds) {
            prime(No{}, Yes{});
            sum_rows<FAST>(a, len, past, rows, from, until, lane, wave, KG * RG, row_max,
                           [&](int row) { return lds_logits + row * (int)sh.keys; },
                           [&](int row, uint64_t v) { atomicAdd(&row_sum[row], (unsigned long long)v); });
        } else {
            if (PASS == kAll) prime(Yes{}, No{});
            RowAdder<MODE> sum[RS];
#pragma unroll
            for (int s = 0; s < RS; ++s) add[s] = splat(FAST ? -lis::screen_c(mx[s], a.k) : 0);
            walk(add, Yes{}, No{}, [&](int key0, const i32x4 (&acc)[RS][4], const int8_t*, bool edge) {
#pragma unroll
                for (int s = 0; s < RS; ++s) sum[s].add(acc[s], mx[s], a);
                if (edge)
#pragma unroll
                    for (int s = 0; s < RS; ++s) sum[s].take_off(16 - seen(key0, min(limit[s], to), lane), a);
            });
#pragma unroll
            for (int s = 0; s < RS; ++s) {
                const uint64_t v = lis::row4_sum(sum[s].sum);
                if (lane < 16) atomicAdd(&row_sum[rg * kRows + 16 * s + lane], (unsigned long long)v);
            }
        }
        __syncthreads();
        if (PASS == kSum) {
            for (int i = threadIdx.x; i < tile_rows; i += kBlock)
                atomicAdd(reinterpret_cast<unsigned long long*>(sh.row_sum) + row_at + i, row_sum[i]);
            return;
        }
    }

    // --- thresholds
    if (PASS == kAll && KEEP == kNot) prime(Yes{}, Yes{});
    lis::RowSum rs[RS];
    if (FAST) {
        for (int at = threadIdx.x; at < tile_rows * a.k.top; at += kBlock) {
            const int r = at % tile_rows, k = at / tile_rows;
            U[r][k] = threshold(2 * row_sum[r], k + 1, a.k);
        }
        __syncthreads();
        for (int at = threadIdx.x; at < tile_rows * (a.k.top + 1); at += kBlock) {
            const int r = at % tile_rows, k = at / tile_rows;
            fill_buckets(U[r], k, a.k.top, sh.shift, sh.buckets, dyn + (r >> 4) * (64 * sh.buckets) + (r & 15));
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
    const int cap = min(a.k.n, a.k.top) * (int)a.k.d_ln2 + 1;
    const auto product = [&](int key0, const i32x4 (&acc)[RS][4], const int8_t* values, bool edge) {
        i32x4 v[NV];
        st.read_v(values, v);
        uint32_t got[16] = {};          // weights of the lane's keys over the sets
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            uint32_t m[4];
            const uint32_t* end = dyn + (rg * RS + s) * (64 * sh.buckets) + 64 * (sh.buckets - 1) + lane;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                uint32_t x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (FAST) {
                        const int u = median(acc[s][t][i], -cap, 0);    // U_1 - 1 - u
                        x[i] = end[(u >> sh.shift) * 64] + (uint32_t)u;
                    } else {
                        uint32_t z;
                        const uint32_t qL = lis::iexp_qL(acc[s][t][i], mx[s], a.k, z);
                        x[i] = (uint32_t)(a.k.top - lis::lis_code(qL, z, rs[s], a.k)) << 24;
                    }
                }
                m[t] = top_bytes(x[0], x[1], x[2], x[3]);
            }
            i32x4 keep = splat(-1);
            if (edge) {
                const int n_seen = seen(key0, min(limit[s], to), lane);
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (4 * t + i >= n_seen) keep[t] &= ~(0xFF << (8 * i));
            }
            i32x4 wh, wl;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                uint32_t dh, dl;
                digits(m[t], (uint32_t)keep[t], dh, dl);
                wh[t] = (int)dh;
                wl[t] = (int)dl;
            }
#pragma unroll
            for (int ct = 0; ct < NV; ++ct) {
                hi[s][ct] = mfma(v[ct], wh, hi[s][ct]);
                lo[s][ct] = mfma(v[ct], wl, lo[s][ct]);
            }
            // sums of the weights, for zp_v: cheaper than a branch on it
            ph[s] = mfma(ones, wh, ph[s]);
            pl[s] = mfma(ones, wl, pl[s]);
            if (WEIGHT && row0 + 16 * s + (lane & 15) < rows)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    got[e] += (1u << ((m[e >> 2] >> (8 * (e & 3))) & 31u)) & ((uint32_t)keep[e >> 2] >> (8 * (e & 3)) & 1u ? ~0u : 0u);
        }
        if (WEIGHT) {
            const uint32_t sum = sum16(got, lane);          // of key lane % 16 of the lane's block
            const int at = min(key0 + 16 * (lane >> 4), (len - 1) & ~15);
            const int id = a.c.table[(int64_t)b * a.c.max_pages + (at >> a.c.log2_page)];
            // an id that is no page is not written through
            const int64_t slot = (((int64_t)id * a.c.Hkv + h) << a.c.log2_page) + (at & ((1 << a.c.log2_page) - 1));
            if (sum && (uint32_t)id < (uint32_t)a.c.pages)
                atomicAdd(reinterpret_cast<unsigned long long*>(a.c.weight) + slot + (lane & 15), (unsigned long long)sum);
        }
    };
#pragma unroll
    for (int s = 0; s < RS; ++s) add[s] = splat(FAST ? U[rg * kRows + 16 * s + (lane & 15)][0] - 1 - mx[s] : 0);
    walk(add, std::integral_constant<bool, !STORED>{}, Yes{}, product);

    // --- out: what the wavefronts of the other key groups hold comes to the first one's
#pragma unroll
    for (int s = 0; s < RS; ++s)
#pragma unroll
        for (int ct = 0; ct < NV; ++ct)
            lo[s][ct] = a.zp_v * (ph[s] * 256 + pl[s]) - (hi[s][ct] * 256 + lo[s][ct]);
    if (KG > 1) {
        i32x4* held = reinterpret_cast<i32x4*>(dyn);        // the buckets are read
        if (kg > 0)
#pragma unroll
            for (int s = 0; s < RS; ++s)
#pragma unroll
                for (int ct = 0; ct < NV; ++ct)
                    held[(((kg - 1) * RG + rg) * RS * NV + s * NV + ct) * 64 + lane] = lo[s][ct];
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int s = 0; s < RS; ++s)
#pragma unroll
            for (int ct = 0; ct < NV; ++ct)
                for (int g = 0; g + 1 < KG; ++g) lo[s][ct] += held[((g * RG + rg) * RS * NV + s * NV + ct) * 64 + lane];
    }
    if (PASS == kOut) {
        // Parts add theirs, whole rows at a time: 16 x 4 places 16 bytes apart, as the lanes hold
        // them, took 3 us more (77 tokens of 3 x 6 heads of 80 in 8 parts).
        if (stages == 0) return;        // a part without keys
        int32_t* turn = reinterpret_cast<int32_t*>(dyn) + C::held / 4 + rg * (C::turned / 4);
        constexpr int ld = 16 * NV + 4;
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            const int row = row0 + 16 * s, n = min(rows - row, 16);
            const int64_t at = query_of(a, b, h, min(row + (lane & 15), rows - 1)) * a.c.d;
#pragma unroll
            for (int ct = 0; ct < NV; ++ct)
                *reinterpret_cast<i32x4*>(turn + (lane & 15) * ld + 16 * ct + 4 * (lane >> 4)) = lo[s][ct];
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the wavefront's own
            for (int i = 0; i < n; ++i) {
                const uint32_t a0 = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)at, i);
                const uint32_t a1 = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(at >> 32), i);
                int32_t* out = a.out + (int64_t)(((uint64_t)a1 << 32) | a0);
                for (int ch = lane; ch < a.c.d; ch += 64) atomicAdd(out + ch, turn[i * ld + ch]);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
        return;
    }
#pragma unroll
    for (int s = 0; s < RS; ++s) {
        const int rho = row0 + 16 * s + (lane & 15);
        if (rho >= rows) continue;
        int32_t* out = a.out + query_of(a, b, h, rho) * a.c.d;
#pragma unroll
        for (int ct = 0; ct < NV; ++ct) {
            const int ch = 16 * ct + 4 * (lane >> 4);
            if (ch < a.c.d) *reinterpret_cast<i32x4*>(out + ch) = lo[s][ct];
        }
    }
}

// Sums of a part of the stored logits: a wavefront takes 256 keys of a row at a time,
// every lane four of them.
template <bool FAST>
__global__ __launch_bounds__(kBlock) void lis_paged_sum_kernel(PagedArgs a, Shape sh) {
    __shared__ int row_max[16];
    __shared__ unsigned long long row_sum[16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place place = place_of<true>(a, sh, lane);
    const int split = place.split, b = place.b;
    const int64_t unit = place.unit;
    const int len = keys_of(a.c, b);
    const int fresh = a.n_new ? min(max(a.n_new[b], 0), a.L) : a.L;
    const int rows = fresh * a.group, past = first_new(a.c, b, fresh);
    if (rows == 0) return;
    const int all = limit_of(a, len, past, rows - 1);
    const int per = ((all + kTile - 1) / kTile + sh.splits - 1) / sh.splits * kTile;
    const int from = min(split * per, all), to = min(from + per, all);
    const int64_t row_at = unit * 16;
    if (threadIdx.x < 16) row_sum[threadIdx.x] = 0;
    parts_max(sh, row_at, rows, lane, wave, kBlock / 64, row_max);
    __syncthreads();
    if (split == 0 && threadIdx.x < rows) sh.row_max[row_at + threadIdx.x] = row_max[threadIdx.x];
    const int32_t* lg = sh.logits + unit * sh.rows * sh.keys;
    sum_rows<FAST>(a, len, past, rows, from, to, lane, wave, kBlock / 64, row_max,
                   [&](int row) { return lg + row * sh.keys; },
                   [&](int row, uint64_t v) { atomicAdd(&row_sum[row], (unsigned long long)v); });
    __syncthreads();
    if (threadIdx.x < rows)
        atomicAdd(reinterpret_cast<unsigned long long*>(sh.row_sum) + row_at + threadIdx.x, row_sum[threadIdx.x]);
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------

// Whether the thresholds and the binary32 I-Exp hold for these constants: q_L below
// 2^24 (which keeps d below 2^11), e(u) not increasing over an octave's end, the sums of
// a tile below 2^52, and -zp_q a byte.
Mode mode_of(const PagedArgs& a) {
    const LisConsts& k = a.k;
    const uint64_t first = (uint64_t)k.qb * k.qb + k.qc;
    const uint64_t w = k.qb - k.d_ln2 + 1, last = w * w + k.qc;
    if (first >= (1u << 24) || 2 * last < first || k.n > 23 || a.zp_q == -128) return kGeneral;
    return k.s_pre ? kShifted : kPlain;
}

template <class C, Pass PASS, Keep KEEP>
void enqueue(const PagedArgs& a, const Shape& sh, const Plan& p, hipStream_t stream) {
    constexpr bool last = PASS == kAll || PASS == kOut;
    const Mode mode = mode_of(a);
    // the buckets, and after them what the key groups hold
    const size_t buckets = mode != kGeneral ? (size_t)C::rows * sh.buckets * 16 : 0;
    const size_t held = C::held + (PASS == kOut ? C::RG * C::turned : 0);
    const size_t logits = KEEP == kLds ? (size_t)(p.rows * p.keys) * 4 : 0;
    const size_t lds = last ? std::max(buckets + logits, held) : 0;
    const bool weight = last && a.c.weight;
    const auto kernel =
        mode == kPlain ? (weight ? lis_paged_kernel<C, PASS, KEEP, kPlain, last>
                                 : lis_paged_kernel<C, PASS, KEEP, kPlain, false>)
        : mode == kShifted ? (weight ? lis_paged_kernel<C, PASS, KEEP, kShifted, last>
                                     : lis_paged_kernel<C, PASS, KEEP, kShifted, false>)
                           : (weight ? lis_paged_kernel<C, PASS, KEEP, kGeneral, last>
                                     : lis_paged_kernel<C, PASS, KEEP, kGeneral, false>);
    launch_kernel(kernel, dim3((uint32_t)(p.units * p.tiles * p.splits)), dim3(C::threads), lds, stream, a, sh);
}

// CHUNK: more than 16 rows, 64 a workgroup (of 128, three workgroups no longer share a
// compute unit: 158 us for 147); heads of 32 channels, whose values are two loads, have two wavefronts
// over the rows and two over the keys.  FEW: up to 16 rows, eight tiles of keys at a time (wide
// heads four: registers), to have as many bytes on their way.
template <class CHUNK, class FEW>
void launch(const PagedArgs& a, const Shape& sh, const Plan& p, hipStream_t stream) {
    if (p.way == paged::kOneFew) return enqueue<FEW, kAll, kLds>(a, sh, p, stream);
    if (p.way == paged::kOne) return enqueue<CHUNK, kAll, kNot>(a, sh, p, stream);
    const bool few = p.way == paged::kPartsFew;
    const LaunchEvents ev = launch_events();
    set_launch_events(ev.start, nullptr);
    if (few) enqueue<FEW, kMax, kWorkspace>(a, sh, p, stream);
    else enqueue<CHUNK, kMax, kNot>(a, sh, p, stream);
    set_launch_events(nullptr, nullptr);
    if (few)
        launch_kernel(mode_of(a) != kGeneral ? lis_paged_sum_kernel<true> : lis_paged_sum_kernel<false>,
                      dim3((uint32_t)(p.units * p.splits)), dim3(kBlock), 0, stream, a, sh);
    else enqueue<CHUNK, kSum, kNot>(a, sh, p, stream);
    set_launch_events(nullptr, ev.stop);
    if (few) enqueue<FEW, kOut, kWorkspace>(a, sh, p, stream);
    else enqueue<CHUNK, kOut, kNot>(a, sh, p, stream);
}

}  // namespace

#if defined(FQ_PAGED_32)
void launch_lis_paged_32(const PagedArgs& a, const paged::Shape& sh, const paged::Plan& p, hipStream_t s) { launch<Config<2, 2, 2, 1, 2>, Config<1, 1, 8, 1, 2>>(a, sh, p, s); }
#elif defined(FQ_PAGED_64)
void launch_lis_paged_64(const PagedArgs& a, const paged::Shape& sh, const paged::Plan& p, hipStream_t s) { launch<Config<1, 4, 1, 1, 4>, Config<1, 1, 8, 1, 4>>(a, sh, p, s); }
#elif defined(FQ_PAGED_128)
void launch_lis_paged_128(const PagedArgs& a, const paged::Shape& sh, const paged::Plan& p, hipStream_t s) { launch<Config<1, 4, 1, 2, 8>, Config<1, 1, 4, 2, 8>>(a, sh, p, s); }
#else
void launch_lis_paged_32(const PagedArgs& a, const paged::Shape& sh, const paged::Plan& p, hipStream_t s);
void launch_lis_paged_64(const PagedArgs& a, const paged::Shape& sh, const paged::Plan& p, hipStream_t s);
void launch_lis_paged_128(const PagedArgs& a, const paged::Shape& sh, const paged::Plan& p, hipStream_t s);

size_t lis_paged_workspace(int32_t B, int32_t Hq, int32_t Hkv, int32_t L, int32_t,
                           int64_t max_keys) {
    return paged::plan(B, Hq, Hkv, L, max_keys).bytes();
}

hipError_t launch_lis_paged(const PagedArgs& a, hipStream_t stream) {
    const Plan p = paged::plan(a.c.B, a.Hq, a.c.Hkv, a.L, (int64_t)a.c.max_pages << a.c.log2_page);
    Shape sh = paged::shape(p, a.workspace);
    while ((2u << sh.shift) <= a.k.d_ln2) ++sh.shift;       // 2^shift <= q_ln2
    const int cap = (a.k.n < a.k.top ? a.k.n : a.k.top) * (int)a.k.d_ln2 + 1;
    sh.buckets = ((cap - 1) >> sh.shift) + 2;
    if (a.c.d <= 32) launch_lis_paged_32(a, sh, p, stream);
    else if (a.c.d <= 64) launch_lis_paged_64(a, sh, p, stream);
    else launch_lis_paged_128(a, sh, p, stream);
    return hipGetLastError();
}
#endif

}  // namespace fqvit
