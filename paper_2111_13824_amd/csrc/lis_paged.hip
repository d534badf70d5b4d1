// Attention of new tokens over a paged cache, integer-only, for gfx950: the int8
// product Q K^T, Log-Int-Softmax and the BitShift product with V (Sec. 3.1, 3.3;
// Supplement A.2), with logits and codes kept on chip.
//
// Layout.  The product is taken transposed: D = K Q^T of the 16x16x64 int8 matrix
// instruction gives a lane (r, g) = (lane % 16, lane / 16) four keys of query r.  Row
// m of the K operand of instruction t (0..3) is key 16 (m / 4) + 4 t + m % 4 of a tile
// of 64, so that lane (r, g) holds the 16 neighbouring keys 16 g .. 16 g + 15 of query
// r: a row's maximum, sum and thresholds live in one register of its lane, its codes
// need no exchange, and the 16 weights P of a lane are, as bytes, its operand of the
// second product D = V^T P^T.  The V^T operand is 16 neighbouring keys of a channel:
// the cache holds values with their channels in rows.  No operand goes through LDS.
//
// A weight P = 2^m, m = (2^b - 1) - code in [0, 15], is not an int8: it is taken as
// -256 hi - lo with hi, lo in {0, -1, -2, .. -128}, two products with the same V
// operand, exact in int32.
//
// The row's maximum is needed before the first I-Exp, its exact sum before the first
// code: three passes over the keys, each of which takes the logits again.
#include "cache_device.h"
#include "fqvit_launch.h"
#include "lis_device.h"

namespace fqvit {
namespace {

using cache::head_base;
using cache::keys_of;
using cache::page_at;

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kTile = 64;           // keys a wavefront takes at a time

template <int KS>
struct Operand {
    i32x4 w[KS];
};

// Row rho of a sequence and head is query (token rho / group, head rho % group).
__device__ __forceinline__ int64_t query_of(const PagedArgs& a, int b, int h, int rho) {
    const int i = rho / a.group, g = rho - i * a.group;
    return ((int64_t)b * a.Hq + h * a.group + g) * a.L + i;
}

__device__ __forceinline__ int limit_of(const PagedArgs& a, int len, int fresh, int rho) {
    return a.causal ? min(max(len - fresh + rho / a.group + 1, 0), len) : len;
}

template <int KS>
struct Tiles {
    const PagedArgs& a;
    int b, h, len, lane;

    // first byte of the 16 keys that hold place `at` (a multiple of 16), in k or v
    __device__ __forceinline__ int64_t base(int at, int& off) const {
        const int last = (len - 1) & ~15;       // behind the last key: its block again
        at = min(at, last);
        off = at & ((1 << a.c.log2_page) - 1);
        return head_base(a.c, page_at(a.c.table, a.c.max_pages, a.c.pages, b, at >> a.c.log2_page), h);
    }

    __device__ __forceinline__ void load_k(int key0, Operand<KS> (&k)[4]) const {
        const int m = lane & 15, g = lane >> 4;
        int off;
        const int8_t* p = a.c.k + base(key0 + 16 * (m >> 2), off) + (int64_t)(off + (m & 3)) * a.c.d;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int at = 64 * s + 16 * g;
                k[t].w[s] = at < a.c.d ? *reinterpret_cast<const i32x4*>(p + 4 * t * a.c.d + at)
                                       : i32x4{0, 0, 0, 0};
            }
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

template <int RS, int KS>
struct Queries {
    Operand<KS> q[RS];
    i32x4 zp[2];            // bytes of -zp_q, in two terms
    int zps;                // how many of them are not zero

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
        const int z0 = min(-a.zp_q, 127), z1 = -a.zp_q - z0;       // 128 = 127 + 1
        const int b0 = (z0 & 0xFF) * 0x01010101, b1 = (z1 & 0xFF) * 0x01010101;
        zp[0] = i32x4{b0, b0, b0, b0};
        zp[1] = i32x4{b1, b1, b1, b1};
        zps = z1 ? 2 : (z0 ? 1 : 0);
    }

    // logits of 64 keys: acc[s][t][i] is key 16 (lane / 16) + 4 t + i of row lane % 16
    __device__ __forceinline__ void logits(const Operand<KS> (&k)[4], i32x4 (&acc)[RS][4]) const {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            i32x4 c = {0, 0, 0, 0};
            for (int z = 0; z < zps; ++z)
#pragma unroll
                for (int x = 0; x < KS; ++x) c = mfma(k[t].w[x], zp[z], c);
#pragma unroll
            for (int s = 0; s < RS; ++s) {
                acc[s][t] = c;
#pragma unroll
                for (int x = 0; x < KS; ++x) acc[s][t] = mfma(k[t].w[x], q[s].w[x], acc[s][t]);
            }
        }
    }
};

// Every key of the tile at `key0` for every row of the wavefront.
__device__ __forceinline__ bool seen(int key0, int t, int i, int limit, int lane) {
    return key0 + 16 * (lane >> 4) + 4 * t + i < limit;
}

template <int RS, int KS, int NV>
__global__ __launch_bounds__(kWaves * 64) void lis_paged_kernel(PagedArgs a, int tiles) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t unit = blockIdx.x / tiles;
    const int tile = blockIdx.x - (int)unit * tiles;
    const int b = (int)(unit / a.c.Hkv), h = (int)(unit % a.c.Hkv);
    const int len = keys_of(a.c, b);
    const int fresh = a.n_new ? min(max(a.n_new[b], 0), a.L) : a.L;
    const int rows = fresh * a.group;
    const int row0 = (tile * kWaves + wave) * 16 * RS;
    if (row0 >= rows) return;

    int limit[RS], mx[RS];
    lis::RowSum rs[RS];
#pragma unroll
    for (int s = 0; s < RS; ++s) limit[s] = limit_of(a, len, fresh, min(row0 + 16 * s + (lane & 15), rows - 1));
    const int reach = limit_of(a, len, fresh, min(row0 + 16 * RS, rows) - 1);
    const int full = limit_of(a, len, fresh, row0);

    Queries<RS, KS> q;
    q.load(a, b, h, row0, rows, lane);
    const Tiles<KS> tl{a, b, h, len, lane};

#pragma unroll
    for (int s = 0; s < RS; ++s) mx[s] = INT_MIN;
    for (int key0 = 0; key0 < reach; key0 += kTile) {
        Operand<KS> k[4];
        i32x4 acc[RS][4];
        tl.load_k(key0, k);
        q.logits(k, acc);
#pragma unroll
        for (int s = 0; s < RS; ++s)
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    mx[s] = max(mx[s], key0 + kTile <= full || seen(key0, t, i, limit[s], lane) ? acc[s][t][i] : INT_MIN);
    }
#pragma unroll
    for (int s = 0; s < RS; ++s) mx[s] = lis::row4_max(mx[s]);

    uint64_t sum[RS] = {};
    for (int key0 = 0; key0 < reach; key0 += kTile) {
        Operand<KS> k[4];
        i32x4 acc[RS][4];
        tl.load_k(key0, k);
        q.logits(k, acc);
#pragma unroll
        for (int s = 0; s < RS; ++s)
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t z;
                    const uint32_t qL = lis::iexp_qL(acc[s][t][i], mx[s], a.k, z);
                    const uint64_t e = (uint64_t)qL << (a.k.n - (int)z);
                    sum[s] += key0 + kTile <= full || seen(key0, t, i, limit[s], lane) ? e : 0;
                }
    }
#pragma unroll
    for (int s = 0; s < RS; ++s) rs[s] = lis::row_sum(sum[s], a.k);

    i32x4 hi[RS][NV] = {}, lo[RS][NV] = {}, ph[RS] = {}, pl[RS] = {};
    const i32x4 ones = {0x01010101, 0x01010101, 0x01010101, 0x01010101};
    for (int key0 = 0; key0 < reach; key0 += kTile) {
        Operand<KS> k[4];
        i32x4 acc[RS][4], v[NV];
        tl.load_k(key0, k);
        tl.load_v(key0, v);
        q.logits(k, acc);
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            i32x4 wh, wl;
            uint32_t got[16];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                uint32_t dh = 0, dl = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t z;
                    const uint32_t qL = lis::iexp_qL(acc[s][t][i], mx[s], a.k, z);
                    const int m = a.k.top - lis::lis_code(qL, z, rs[s], a.k);
                    const bool in = key0 + kTile <= full || seen(key0, t, i, limit[s], lane);
                    const uint32_t P = in ? 1u << m : 0u;
                    got[4 * t + i] = P;
                    dl |= ((0u - (P & 0xFFu)) & 0xFFu) << (8 * i);
                    dh |= ((0u - (P >> 8)) & 0xFFu) << (8 * i);
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
            if (a.c.weight) {
                const bool mine = row0 + 16 * s + (lane & 15) < rows;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    uint32_t p = mine ? got[e] : 0u;
#pragma unroll
                    for (int o = 1; o < 16; o <<= 1) p += __shfl_xor(p, o);
                    const int key = key0 + 16 * (lane >> 4) + e;
                    if ((lane & 15) == e && key < len) {
                        const int id = page_at(a.c.table, a.c.max_pages, a.c.pages, b, key >> a.c.log2_page);
                        atomicAdd(reinterpret_cast<unsigned long long*>(a.c.weight) +
                                      (((int64_t)id * a.c.Hkv + h) << a.c.log2_page) +
                                      (key & ((1 << a.c.log2_page) - 1)),
                                  (unsigned long long)p);
                    }
                }
            }
        }
    }
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
            *reinterpret_cast<i32x4*>(out + ch) = o;
        }
    }
}

template <int KS, int NV>
void launch(const PagedArgs& a, hipStream_t stream) {
    const int rows = a.L * a.group;
    const int tiles = (rows + kWaves * 16 - 1) / (kWaves * 16);
    launch_kernel(lis_paged_kernel<1, KS, NV>, dim3((uint32_t)((int64_t)a.c.B * a.c.Hkv * tiles)),
                  dim3(kWaves * 64), 0, stream, a, tiles);
}

}  // namespace

size_t lis_paged_workspace(int32_t, int32_t, int32_t, int32_t, int32_t, int64_t) { return 0; }

hipError_t launch_lis_paged(const PagedArgs& a, hipStream_t stream) {
    if (a.c.d <= 32) launch<1, 2>(a, stream);
    else if (a.c.d <= 64) launch<1, 4>(a, stream);
    else launch<2, 8>(a, stream);
    return hipGetLastError();
}

}  // namespace fqvit
