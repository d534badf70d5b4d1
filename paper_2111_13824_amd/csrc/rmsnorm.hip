// Root-mean-square norm of an int16 stream with an int8 branch added to it, for
// gfx950.  Memory-bound: 6 bytes a value (branch 1, stream 2 read and 2 written,
// output 1), all of them once: a row's values stay in the registers of a group of lanes, a
// wavefront up to 1024 channels and a workgroup above.  9232 x 1024: 12.1 us, 4.7 TB/s (a
// copy reaches 5.2); with the factors loaded one by one 25.5.  One row: 2.8 us of a call
// of 9.5.
//
//   h = clip16(r + rint((x - zp_x) 2^min(alpha, K) m_x)),  M2 = sum h^2
//   rho = 1 / sqrt(M2 / C + eps)  (binary64, each operation rounded once)
//   one scale:   y = clip(rint(h f + zp)), f = RN(gamma RN(rho / s_out))
//   row scales:  a = RN(gamma h), A = max |a|, t = 2^(b-1) - 1,
//                y = rint(a RN(t / A)), scale = RN(RN(A RN(rho)) / t)
//
// M2 is exact in 64 bits (h^2 <= 2^30).  A product with a binary32 factor is rounded
// to the grid by one fma with 1.5 2^23 added, whose sum has the integer in its low
// bits: the exact product is rounded once, ties to even, as rint does (|product|
// stays below 2^22, or far outside the clip).
#include "fqvit_launch.h"
#include "stream_internal.h"

namespace fqvit {
namespace {

constexpr int kBlock = 256;
constexpr float kMagic = 12582912.0f;   // 1.5 * 2^23

// A row's values: V of them a lane in NV groups of 8.  VEC: a group is 8 neighbours
// (16-byte loads); else the lanes take single values in turn.
template <int LANES, bool VEC>
__device__ __forceinline__ int place(int lane, int j, int e) {
    return VEC ? 8 * (lane + LANES * j) + e : lane + LANES * (8 * j + e);
}

template <int LANES>
__device__ __forceinline__ uint64_t row_sum(uint64_t v, uint64_t* lds) {
#pragma unroll
    for (int o = 1; o < (LANES < 64 ? LANES : 64); o <<= 1) v += __shfl_xor(v, o);
    if (LANES > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0;
        for (int i = 0; i < LANES / 64; ++i) v += lds[i];
    }
    return v;
}

template <int LANES>
__device__ __forceinline__ float row_max(float v, float* lds) {
#pragma unroll
    for (int o = 1; o < (LANES < 64 ? LANES : 64); o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
    if (LANES > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
        for (int i = 0; i < LANES / 64; ++i) v = fmaxf(v, lds[i]);
    }
    return v;
}

typedef int16_t i16x8 __attribute__((ext_vector_type(8)));
typedef int8_t i8x8 __attribute__((ext_vector_type(8)));
typedef uint8_t u8x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// The factors of a group's channels (0 beyond C).
template <int LANES, bool VEC>
__device__ __forceinline__ void load_gamma(const float* p, int lane, int j, int C, float (&out)[8]) {
    if (VEC) {
        const int c = place<LANES, true>(lane, j, 0);
        f32x4 g0 = {0.0f, 0.0f, 0.0f, 0.0f}, g1 = g0;
        if (c < C) {
            g0 = *reinterpret_cast<const f32x4*>(p + c);
            g1 = *reinterpret_cast<const f32x4*>(p + c + 4);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            out[e] = g0[e];
            out[4 + e] = g1[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = place<LANES, false>(lane, j, e);
            out[e] = c < C ? p[c] : 0.0f;
        }
    }
}

// Values at and beyond C are skipped.
template <int LANES, bool VEC, typename T, typename V8>
__device__ __forceinline__ void load8(const T* p, int lane, int j, int C, T (&out)[8]) {
    if (VEC) {
        const int c = place<LANES, true>(lane, j, 0);
        if (c < C) {
            const V8 v = *reinterpret_cast<const V8*>(p + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = v[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = place<LANES, false>(lane, j, e);
            if (c < C) out[e] = p[c];
        }
    }
}

template <int LANES, bool VEC, typename T, typename V8>
__device__ __forceinline__ void store8(T* p, int lane, int j, int C, const T (&in)[8]) {
    if (VEC) {
        const int c = place<LANES, true>(lane, j, 0);
        if (c < C) {
            V8 v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = in[e];
            *reinterpret_cast<V8*>(p + c) = v;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = place<LANES, false>(lane, j, e);
            if (c < C) p[c] = in[e];
        }
    }
}

template <int LANES, int NV, bool VEC, bool ROWS>
__global__ __launch_bounds__(kBlock) void rmsnorm_kernel(RmsArgs a) {
    __shared__ uint64_t sums[4];
    __shared__ float tops[4];
    constexpr int kRows = kBlock / LANES;
    const int lane = threadIdx.x % LANES;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
    // a row behind the last works on the last one's values and stores nothing
    const bool live = row < a.T;
    const int64_t base = (live ? row : a.T - 1) * a.C;
    const int C = a.C;

    int h[NV][8];
    float gamma[NV][8];
    uint64_t m2 = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) load_gamma<LANES, VEC>(a.gamma, lane, j, C, gamma[j]);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        int16_t r[8] = {};
        load8<LANES, VEC, int16_t, i16x8>(a.r + base, lane, j, C, r);
        if (a.x) {
            int8_t x[8];
            uint8_t al[8] = {};
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (int8_t)a.zp_x;      // nothing behind C
            load8<LANES, VEC, int8_t, i8x8>(a.x + base, lane, j, C, x);
            if (a.alpha) load8<LANES, VEC, uint8_t, u8x8>(a.alpha, lane, j, C, al);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int lifted = (x[e] - a.zp_x) << min((int)al[e], a.K);
                const float t = __builtin_fmaf((float)lifted, a.m_x, kMagic);
                h[j][e] = min(max(r[e] + (__float_as_int(t) - __float_as_int(kMagic)), -32768), 32767);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) h[j][e] = r[e];
        }
#pragma unroll
        for (int e = 0; e < 8; e += 2)      // two squares stay within 2^31
            m2 += (uint32_t)(h[j][e] * h[j][e]) + (uint32_t)(h[j][e + 1] * h[j][e + 1]);
        if (live) {
            int16_t o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (int16_t)h[j][e];
            store8<LANES, VEC, int16_t, i16x8>(a.h + base, lane, j, C, o);
        }
    }
    m2 = row_sum<LANES>(m2, sums);
    const double mean = (double)m2 / (double)C + (double)a.eps;
    const double rho = mean > 0.0 ? 1.0 / sqrt(mean) : 0.0;

    const int half = 1 << (a.bits - 1);
    const float lo = (float)-half, hi = (float)(half - 1);
    float add = kMagic, factor = 0.0f;
    if (ROWS) {
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                gamma[j][e] *= (float)h[j][e];          // a
                top = fmaxf(top, fabsf(gamma[j][e]));
            }
        top = row_max<LANES>(top, tops);
        factor = top > 0.0f ? (float)((double)hi / (double)top) : 0.0f;
        if (live && lane == 0) a.scales[row] = (float)((double)(top * (float)rho) / (double)hi);
    } else {
        factor = (float)(rho / (double)a.s_out);
        add += (float)a.zp_out;
    }
    if (!live) return;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        int8_t o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float t;
            if (ROWS) t = __builtin_fmaf(gamma[j][e], factor, add);
            else t = __builtin_fmaf((float)h[j][e], gamma[j][e] * factor, add);
            o[e] = (int8_t)(int)fminf(fmaxf(t - kMagic, lo), hi);
        }
        store8<LANES, VEC, int8_t, i8x8>(a.y + base, lane, j, C, o);
    }
}

template <int LANES, int NV>
void launch(const RmsArgs& a, bool vec, hipStream_t stream) {
    constexpr int kRows = kBlock / LANES;
    const dim3 grid((uint32_t)((a.T + kRows - 1) / kRows)), block(kBlock);
    if (a.scales)
        launch_kernel(vec ? rmsnorm_kernel<LANES, NV, true, true> : rmsnorm_kernel<LANES, NV, false, true>,
                      grid, block, 0, stream, a);
    else
        launch_kernel(vec ? rmsnorm_kernel<LANES, NV, true, false> : rmsnorm_kernel<LANES, NV, false, false>,
                      grid, block, 0, stream, a);
}

}  // namespace

hipError_t launch_rmsnorm(const RmsArgs& a, hipStream_t stream) {
    const auto aligned = [](const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
    const bool vec = a.C % 8 == 0 && aligned(a.r, 16) && aligned(a.h, 16) && aligned(a.x, 8) &&
                     aligned(a.alpha, 8) && aligned(a.y, 8) && aligned(a.gamma, 16);
    if (a.C <= 32) launch<4, 1>(a, vec, stream);
    else if (a.C <= 128) launch<16, 1>(a, vec, stream);
    else if (a.C <= 512) launch<64, 1>(a, vec, stream);
    else if (a.C <= 1024) launch<64, 2>(a, vec, stream);
    else if (a.C <= 2048) launch<256, 1>(a, vec, stream);
    else if (a.C <= 4096) launch<256, 2>(a, vec, stream);
    else launch<256, 4>(a, vec, stream);
    return hipGetLastError();
}

}  // namespace fqvit
