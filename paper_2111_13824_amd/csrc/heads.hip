// Rotary positions on the query-key-value layer's rows, and the attention's
// heads back to rows, for gfx950.  Both move each byte once and are bound by
// memory: what counts is that rows are read and written in whole lines with many
// loads under way.  On ViT-L/16 at batch 16 (9232 rows of 48 heads of 64, 57 MB) the
// rotation takes 13.4 us by itself (median of a trace; 11.6 at least), 12.6 among
// others of its kind, 4.5 TB/s; on ViT-B/16 at batch 64 the way back to rows (48 MB)
// 11.2 (9.8) and 10.6, 4.6 TB/s; a large copy reaches 5.1.
#include <algorithm>

#include "bytes_device.h"
#include "fqvit.h"
#include "fqvit_launch.h"
#include "layers_internal.h"
#include "requant_device.h"

namespace fqvit {
namespace {

constexpr int kBlock = 256;
constexpr float kMagic = 12582912.0f;   // 1.5 * 2^23: v + kMagic has rint(v) in its low bits

// ---------------------------------------------------------------------------
// The table: a token and pair of a thread at a time
// ---------------------------------------------------------------------------

__global__ __launch_bounds__(kBlock) void rope_table_kernel(RopeTableArgs p) {
    const int64_t step = (int64_t)gridDim.x * kBlock;
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < p.T * p.P; i += step) {
        const int64_t tok = i / p.P;
        const int pair = (int)(i - tok * p.P);
        const int ax = min((int)p.axis[pair], p.axes - 1);
        const double t = (double)p.positions[ax * p.T + tok] * p.freq[pair];
        double s, c;
        sincos(t, &s, &c);
        const uint32_t lo = (uint32_t)(int)rint(16384.0 * c) & 0xFFFFu;
        const uint32_t hi = (uint32_t)(int)rint(16384.0 * s) << 16;
        reinterpret_cast<uint32_t*>(p.table)[i] = lo | hi;
    }
}

// ---------------------------------------------------------------------------
// Rotation
// ---------------------------------------------------------------------------

// A lane holds V bytes of a head's row; 64 / (d / V) rows of consecutive tokens
// make a wavefront, which walks over a group of heads: its stores are runs of
// consecutive tokens of one head, and its loads of four heads one after another
// are whole lines of the tokens' rows.  The turn of the lane's V values is the
// same for every head and stays in registers: with f, g the value and its
// partner + 128 and z = 128 + zp_x,
//   turned = f c + g s + k,  k = -z (c + s),
// where s has the sign of the value's side of its pair, and a value that does
// not turn has c = 2^14, s = 0.  All terms are integers below 2^24: exact.
template <int V>
struct Bytes {
    uint32_t w[V / 4];
};

// V bytes to an address of their alignment, past L2: the next kernel reads rows of
// many megabytes from elsewhere by then (9232 rows of 48 heads of 64: 13.3 -> 11.9 us).
template <int V>
__device__ __forceinline__ void store_bytes(int8_t* at, const Bytes<V>& b) {
    typedef uint32_t words __attribute__((ext_vector_type(V / 4)));
    if constexpr (V == 4)
        __builtin_nontemporal_store(b.w[0], reinterpret_cast<uint32_t*>(at));
    else
        __builtin_nontemporal_store(__builtin_bit_cast(words, b), reinterpret_cast<words*>(at));
}

// V bytes at any address.
template <int V>
__device__ __forceinline__ Bytes<V> load_bytes(const int8_t* at) {
    Bytes<V> b;
    __builtin_memcpy(&b, at, V);
    return b;
}

// The same moved up by n <= V bytes, zeros below.
template <int V>
__device__ __forceinline__ Bytes<V> move_up(Bytes<V> b, int n) {
    Bytes16 u = {};
    __builtin_memcpy(&u, &b, V);
    u = bytes_up(u, n);
    __builtin_memcpy(&b, &u, V);
    return b;
}

template <int V>
__device__ __forceinline__ float ubyte(const Bytes<V>& b, int j) {
    return (float)((b.w[j >> 2] >> (8 * (j & 3))) & 0xFFu);
}

// How a lane finds its values' partners.
enum Partner {
    kInside,    // pairs lie together (V is even): in the lane's own bytes
    kLane,      // P is a multiple of V: one other lane has them all
    kMemory,    // any P: two loads of the row, from P bytes on and from P before
};

template <int V, Partner HOW>
__global__ __launch_bounds__(kBlock) void rope_qkv_kernel(RopeArgs p, int64_t tiles, int groups,
                                                          int per_group) {
    typedef Bytes<V> B;
    const int lane = threadIdx.x & 63;
    const int64_t job = (int64_t)blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6);
    const int64_t tile = job / groups;
    if (tile >= tiles) return;
    const int heads = p.Hq + 2 * p.Hkv;
    const int h0 = (int)(job - tile * groups) * per_group, h1 = min(h0 + per_group, heads);
    const int lanes = p.d / V, rows = 64 / lanes;     // of a head's row; of a wavefront
    const int slot = lane / lanes, j0 = (lane - slot * lanes) * V;
    const int64_t tok = tile * rows + slot;
    const bool live = slot < rows && tok < p.B * p.L;
    const int64_t t = live ? tok : 0;
    const int64_t b = t / p.L;
    const int l = (int)(t - b * p.L);

    const float z = (float)(128 + p.zp_x);
    float c[V], s[V], k[V];
    {
        constexpr int E = HOW == kInside ? V / 2 : V;     // table entries a lane needs
        uint32_t e[E];
        const uint32_t* row =
            reinterpret_cast<const uint32_t*>(p.table) + (p.per_image ? t : (int64_t)l) * p.P;
        if (HOW != kMemory && (HOW == kInside ? j0 + V <= 2 * p.P : j0 < 2 * p.P)) {
            // one after another
            __builtin_memcpy(e, row + (HOW == kInside ? j0 / 2 : (j0 >= p.P ? j0 - p.P : j0)), sizeof(e));
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const int at = HOW == kInside ? j0 + 2 * i : j0 + i;
                const int pair = HOW == kInside ? at >> 1 : (at >= p.P ? at - p.P : at);
                e[i] = at < 2 * p.P ? row[pair] : 16384u;
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const bool second = HOW == kInside ? (j & 1) : j0 + j >= p.P;
            const uint32_t x = e[HOW == kInside ? j / 2 : j];
            c[j] = (float)(int16_t)x;
            s[j] = (float)((int)x >> 16);
            s[j] = second ? s[j] : -s[j];
            k[j] = -z * (c[j] + s[j]);
        }
    }
    // kLane: the lane with this lane's partners
    const int apart = p.P / V;
    const int with = j0 >= 2 * p.P ? lane : (j0 >= p.P ? lane - apart : lane + apart);
    // kMemory: the partners of the values before P lie P on (that many bytes are
    // there: a value head follows every head that turns), those from P on P before
    const int on = j0 < p.P ? p.P : 0, before = j0 >= p.P ? p.P : j0, up = j0 < p.P ? min(p.P - j0, V) : 0;
    Bytes<V> from_before;
    if (HOW == kMemory) {
        for (int i = 0; i < V / 4; ++i) from_before.w[i] = 0xFFFFFFFFu;
        from_before = move_up(from_before, up);
    }
    const int half = 1 << (p.bits - 1);
    const float lo = kMagic - (float)half, hi = kMagic + (float)(half - 1);
    const int64_t step = (int64_t)p.L * p.d;          // from a head to the next
    const int8_t* in = p.qkv + t * heads * p.d + j0;
    int8_t* q = p.q + (b * p.Hq * p.L + l) * p.d + j0;
    int8_t* kk = p.k + (b * p.Hkv * p.L + l) * p.d + j0;
    int8_t* v = p.v + (b * p.Hkv * p.L + l) * p.d + j0;

    auto one = [&](B x, int h) __attribute__((always_inline)) {
        if (h >= p.Hq + p.Hkv) {
            if (live) store_bytes<V>(v + (h - p.Hq - p.Hkv) * step, x);
            return;
        }
        const bool is_q = h < p.Hq;
        const float m = is_q ? p.m_q : p.m_k, zp = kMagic + (float)(is_q ? p.zp_q : p.zp_k);
        B y, out;
        if constexpr (HOW == kMemory) {
            const int8_t* own = in + h * p.d;
            const B far = load_bytes<V>(own + on), near = move_up(load_bytes<V>(own - before), up);
#pragma unroll
            for (int i = 0; i < V / 4; ++i)
                y.w[i] = ((near.w[i] & from_before.w[i]) | (far.w[i] & ~from_before.w[i])) ^ 0x80808080u;
        }
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            x.w[i] ^= 0x80808080u;
            if constexpr (HOW == kLane) y.w[i] = (uint32_t)__shfl((int)x.w[i], with, 64);
        }
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            uint32_t r[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = 4 * i + e;
                const float f = ubyte(x, j), g = HOW == kInside ? ubyte(x, j ^ 1) : ubyte(y, j);
                const float a = __builtin_fmaf(f, c[j], __builtin_fmaf(g, s[j], k[j]));
                r[e] = __builtin_bit_cast(
                    uint32_t, __builtin_amdgcn_fmed3f(__builtin_fmaf(a, m, zp), lo, hi));
            }
            out.w[i] = __builtin_amdgcn_perm(r[1], r[0], 0x0c0c0400u) |
                       __builtin_amdgcn_perm(r[3], r[2], 0x04000c0cu);
        }
        if (live) store_bytes<V>(is_q ? q + h * step : kk + (h - p.Hq) * step, out);
    };

    constexpr int kAhead = 4;
    int h = h0;
    for (; h + kAhead <= h1; h += kAhead) {
        B x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) x[i] = *reinterpret_cast<const B*>(in + (h + i) * p.d);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) one(x[i], h + i);
    }
    for (; h < h1; ++h) one(*reinterpret_cast<const B*>(in + h * p.d), h);
}

// Heads of any size on any base: one value of a thread at a time.
__global__ __launch_bounds__(kBlock) void rope_qkv_bytes_kernel(RopeArgs p) {
    const int heads = p.Hq + 2 * p.Hkv;
    const int64_t row = (int64_t)heads * p.d, n = p.B * p.L * row;
    const int half = 1 << (p.bits - 1);
    const int64_t step = (int64_t)gridDim.x * kBlock;
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += step) {
        const int64_t tok = i / row;
        const int at = (int)(i - tok * row);
        const int h = at / p.d, j = at - h * p.d;
        const int64_t b = tok / p.L;
        const int l = (int)(tok - b * p.L);
        if (h >= p.Hq + p.Hkv) {
            p.v[((b * p.Hkv + h - p.Hq - p.Hkv) * p.L + l) * p.d + j] = p.qkv[i];
            continue;
        }
        const int x = p.qkv[i] - p.zp_x;
        float a = (float)(x * 16384);
        if (j < 2 * p.P) {
            const int pair = p.interleaved ? j >> 1 : (j < p.P ? j : j - p.P);
            const bool second = p.interleaved ? (j & 1) : j >= p.P;
            const int off = p.interleaved ? 1 : p.P;
            const int16_t* cs = p.table + 2 * ((p.per_image ? tok : (int64_t)l) * p.P + pair);
            const int o = p.qkv[second ? i - off : i + off] - p.zp_x;
            a = (float)(second ? o * cs[1] + x * cs[0] : x * cs[0] - o * cs[1]);
        }
        const bool is_q = h < p.Hq;
        float v = __builtin_fmaf(a, is_q ? p.m_q : p.m_k, kMagic + (float)(is_q ? p.zp_q : p.zp_k));
        v = __builtin_amdgcn_fmed3f(v, kMagic - (float)half, kMagic + (float)(half - 1));
        int8_t* out = is_q ? p.q + ((b * p.Hq + h) * p.L + l) * p.d
                           : p.k + ((b * p.Hkv + h - p.Hq) * p.L + l) * p.d;
        out[j] = (int8_t)__builtin_bit_cast(uint32_t, v);
    }
}

// ---------------------------------------------------------------------------
// Heads back to rows
// ---------------------------------------------------------------------------

// A lane holds four values of a row of a head (16 bytes read, 4 written, neither
// aligned where d is odd; the last lane of a row may hold fewer); 64 / ceil(d / 4)
// rows of consecutive tokens make a wavefront, which walks over a group of heads
// with four heads' loads under way.
template <bool HI>
__global__ __launch_bounds__(kBlock) void requant_heads_kernel(RequantHeadsArgs p, int64_t tiles,
                                                               int groups, int per_group) {
    typedef int vi4 __attribute__((ext_vector_type(4)));
    typedef int vi4u __attribute__((ext_vector_type(4), aligned(4)));
    const int lane = threadIdx.x & 63;
    const int64_t job = (int64_t)blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6);
    const int64_t tile = job / groups;
    if (tile >= tiles) return;
    const int h0 = (int)(job - tile * groups) * per_group, h1 = min(h0 + per_group, p.H);
    const int lanes = (p.d + 3) / 4, rows = 64 / lanes;
    const int slot = lane / lanes, j0 = (lane - slot * lanes) * 4;
    const int64_t tok = tile * rows + slot;
    if (slot >= rows || tok >= p.B * p.L) return;
    const int64_t b = tok / p.L;
    const int l = (int)(tok - b * p.L);
    const int64_t step = (int64_t)p.L * p.d;
    const int32_t* in = p.r.q + (b * p.H * p.L + l) * p.d + j0;
    int8_t* out = p.r.y + tok * p.H * p.d + j0;
    const int half = 1 << (p.r.bits - 1);
    auto one = [&](int32_t x) __attribute__((always_inline)) {
        if constexpr (HI)
            return requant_hi(x, (int32_t)p.r.N2, (uint64_t)1 << (p.r.N1 - 1), p.r.N1 - 32, p.r.zp, -half,
                              half - 1);
        else
            return requant_one(x, p.r.N2, p.r.N1, p.r.zp + half, 2 * half - 1, half);
    };
    if (j0 + 4 > p.d) {                                // a row's end
        for (int h = h0; h < h1; ++h)
            for (int j = 0; j < p.d - j0; ++j) out[h * p.d + j] = (int8_t)one(in[h * step + j]);
        return;
    }
    auto four = [&](vi4 x, int h) __attribute__((always_inline)) {
        const uint32_t lo = __builtin_amdgcn_perm((uint32_t)one(x[1]), (uint32_t)one(x[0]), 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm((uint32_t)one(x[3]), (uint32_t)one(x[2]), 0x04000c0cu);
        const uint32_t w = lo | hi;
        __builtin_memcpy(out + h * p.d, &w, 4);
    };
    auto load = [&](int h) __attribute__((always_inline)) {
        return __builtin_nontemporal_load(reinterpret_cast<const vi4u*>(in + h * step));
    };
    constexpr int kAhead = 4;
    int h = h0;
    for (; h + kAhead <= h1; h += kAhead) {
        vi4 x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) x[i] = load(h + i);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) four(x[i], h + i);
    }
    for (; h < h1; ++h) four(load(h), h);
}

// Workgroups of a kernel that takes one value of a thread at a time.
unsigned blocks(int64_t n) { return (unsigned)std::min<int64_t>((n + kBlock - 1) / kBlock, 1 << 20); }

// Tiles of `rows` tokens times groups of heads, a wavefront each: groups of four
// heads where that many wavefronts are needed to fill the chip (16 a CU), longer
// ones, which load the turn once for more heads, where there are enough.  With 8
// and 32 a CU instead, 64 x 197 rows of 36 heads of 64 take 14.2 and 13.4 us (12.9
// with 16), and 64 x 12 x 197 x 64 values brought back to rows 9.8 and 8.4 (8.6).
struct Jobs {
    int64_t tiles;
    int groups, per_group;
    unsigned blocks;
};

Jobs jobs(int64_t tokens, int rows, int heads) {
    Jobs j;
    j.tiles = (tokens + rows - 1) / rows;
    const int64_t want = (4096 + j.tiles - 1) / j.tiles;              // groups wanted
    const int most = (heads + 3) / 4;
    const int groups = (int)std::min<int64_t>(want, most);
    j.per_group = ((heads + groups - 1) / groups + 3) / 4 * 4;
    j.groups = (heads + j.per_group - 1) / j.per_group;
    j.blocks = (unsigned)((j.tiles * j.groups + kBlock / 64 - 1) / (kBlock / 64));
    return j;
}

bool aligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

template <int V>
bool rope_fits(const RopeArgs& a) {
    return a.d % V == 0 && aligned(a.qkv, V) && aligned(a.q, V) &&
           aligned(a.k, V) && aligned(a.v, V);
}

template <int V>
void launch_rope(const RopeArgs& a, hipStream_t stream) {
    const Jobs j = jobs(a.B * a.L, 64 / (a.d / V), a.Hq + 2 * a.Hkv);
    auto go = [&](auto kernel) {
        launch_kernel(kernel, dim3(j.blocks), dim3(kBlock), 0, stream, a, j.tiles, j.groups, j.per_group);
    };
    if (a.interleaved || a.P == 0)
        go(rope_qkv_kernel<V, kInside>);
    else if (a.P % V == 0)
        go(rope_qkv_kernel<V, kLane>);
    else
        go(rope_qkv_kernel<V, kMemory>);
}

}  // namespace

hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t stream) {
    launch_kernel(rope_table_kernel, dim3(blocks(a.T * a.P)), dim3(kBlock), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_rope_qkv(const RopeArgs& a, hipStream_t stream) {
    // 8 bytes a lane where that lets a lane find its partners in another lane and
    // 16 do not: 16 x 577 rows of 48 heads of 80, P = 40: 17.5 us, 23.1 with 16
    const bool lane8 = !a.interleaved && a.P % 16 != 0 && a.P % 8 == 0;
    if (rope_fits<16>(a) && !lane8)
        launch_rope<16>(a, stream);
    else if (rope_fits<8>(a))
        launch_rope<8>(a, stream);
    else if (rope_fits<4>(a))
        launch_rope<4>(a, stream);
    else
        launch_kernel(rope_qkv_bytes_kernel, dim3(blocks(a.B * a.L * (a.Hq + 2 * a.Hkv) * (int64_t)a.d)),
                      dim3(kBlock), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_requant_heads(const RequantHeadsArgs& a, hipStream_t stream) {
    const Jobs j = jobs(a.B * a.L, 64 / ((a.d + 3) / 4), a.H);
    if (a.r.N1 >= 32)
        launch_kernel(requant_heads_kernel<true>, dim3(j.blocks), dim3(kBlock), 0, stream, a, j.tiles,
                      j.groups, j.per_group);
    else
        launch_kernel(requant_heads_kernel<false>, dim3(j.blocks), dim3(kBlock), 0, stream, a, j.tiles,
                      j.groups, j.per_group);
    return hipGetLastError();
}

}  // namespace fqvit
