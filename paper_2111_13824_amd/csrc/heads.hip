// Rotary positions on the query-key-value layer's rows, and the attention's
// heads back to rows, for gfx950.
#include <algorithm>

#include "fqvit.h"
#include "fqvit_launch.h"

namespace fqvit {
namespace {

constexpr int kBlock = 256;

__global__ __launch_bounds__(kBlock) void rope_table_kernel(RopeTableArgs p) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i >= p.T * p.P) return;
    const int64_t tok = i / p.P;
    const int pair = (int)(i - tok * p.P);
    const int ax = min((int)p.axis[pair], p.axes - 1);
    const double t = (double)p.positions[ax * p.T + tok] * p.freq[pair];
    double s, c;
    sincos(t, &s, &c);
    p.table[2 * i] = (int16_t)rint(16384.0 * c);
    p.table[2 * i + 1] = (int16_t)rint(16384.0 * s);
}

constexpr float kMagic = 12582912.0f;   // v + kMagic: rint(v) in the low bits

// One value of one head a thread.
__global__ __launch_bounds__(kBlock) void rope_qkv_kernel(RopeArgs p) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    const int heads = p.Hq + 2 * p.Hkv;
    const int64_t row = (int64_t)heads * p.d;
    if (i >= p.B * p.L * row) return;
    const int64_t tok = i / row;
    const int at = (int)(i - tok * row);
    const int h = at / p.d, j = at - h * p.d;
    const int64_t b = tok / p.L;
    const int l = (int)(tok - b * p.L);
    if (h >= p.Hq + p.Hkv) {
        p.v[((b * p.Hkv + h - p.Hq - p.Hkv) * p.L + l) * p.d + j] = p.qkv[i];
        return;
    }
    float a = (float)((p.qkv[i] - p.zp_x) * 16384);
    if (j < 2 * p.P) {
        const int pair = p.interleaved ? j >> 1 : (j < p.P ? j : j - p.P);
        const bool second = p.interleaved ? (j & 1) : j >= p.P;
        const int off = p.interleaved ? 1 : p.P;
        const int16_t* cs = p.table + 2 * ((p.per_image ? tok : (int64_t)l) * p.P + pair);
        const int x = p.qkv[i] - p.zp_x, o = p.qkv[second ? i - off : i + off] - p.zp_x;
        a = (float)(second ? o * cs[1] + x * cs[0] : x * cs[0] - o * cs[1]);
    }
    const bool is_q = h < p.Hq;
    const int half = 1 << (p.bits - 1);
    float v = __builtin_fmaf(a, is_q ? p.m_q : p.m_k, kMagic + (float)(is_q ? p.zp_q : p.zp_k));
    v = __builtin_amdgcn_fmed3f(v, kMagic - (float)half, kMagic + (float)(half - 1));
    int8_t* out = is_q ? p.q + ((b * p.Hq + h) * p.L + l) * p.d
                       : p.k + ((b * p.Hkv + h - p.Hq) * p.L + l) * p.d;
    out[j] = (int8_t)__builtin_bit_cast(uint32_t, v);
}

__global__ __launch_bounds__(kBlock) void requant_heads_kernel(RequantHeadsArgs p) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    const int64_t row = (int64_t)p.H * p.d;
    if (i >= p.B * p.L * row) return;
    const int64_t tok = i / row;
    const int at = (int)(i - tok * row);
    const int h = at / p.d, j = at - h * p.d;
    const int64_t b = tok / p.L;
    const int l = (int)(tok - b * p.L);
    const int64_t q = p.r.q[((b * p.H + h) * p.L + l) * p.d + j];
    const int half = 1 << (p.r.bits - 1);
    const int64_t prod = p.r.N2 * q;
    const int64_t w =
        (p.r.N1 > 0 ? (prod + ((int64_t)1 << (p.r.N1 - 1))) >> p.r.N1 : prod) + p.r.zp;
    p.r.y[i] = (int8_t)(w < -half ? -half : (w > half - 1 ? half - 1 : w));
}

unsigned blocks(int64_t n) { return (unsigned)((n + kBlock - 1) / kBlock); }

}  // namespace

hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t stream) {
    launch_kernel(rope_table_kernel, dim3(blocks(a.T * a.P)), dim3(kBlock), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_rope_qkv(const RopeArgs& a, hipStream_t stream) {
    launch_kernel(rope_qkv_kernel, dim3(blocks(a.B * a.L * (a.Hq + 2 * a.Hkv) * (int64_t)a.d)),
                  dim3(kBlock), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_requant_heads(const RequantHeadsArgs& a, hipStream_t stream) {
    launch_kernel(requant_heads_kernel, dim3(blocks(a.B * a.L * (int64_t)a.H * a.d)), dim3(kBlock), 0,
                  stream, a);
    return hipGetLastError();
}

}  // namespace fqvit
