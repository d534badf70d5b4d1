// Linear layers (int8 x int8 -> int32, with bias, activation, residual and
// requantization in the epilogue) for gfx950.
#include <algorithm>

#include "fqvit.h"
#include "fqvit_launch.h"

namespace fqvit {
namespace {

typedef int vi4 __attribute__((ext_vector_type(4)));
typedef int vi16 __attribute__((ext_vector_type(16)));

constexpr int kBlock = 256;

// ---------------------------------------------------------------------------
// Epilogue
// ---------------------------------------------------------------------------

// Rounding to the nearest integer by adding kMagic: sums in [2^23, 2^24) have a
// step of 1, so v + kMagic is kMagic + rint(v) for |v| < 2^22, the integer in the
// low bits of the binary32 pattern.  Values beyond that range leave it on their
// own side (rounding is monotone), where the clamp that follows takes them.
constexpr float kMagic = 12582912.0f;   // 1.5 * 2^23
constexpr uint32_t kMagicBits = 0x4B400000u;

__device__ __forceinline__ float clamp3(float v, float lo, float hi) {
    return __builtin_amdgcn_fmed3f(v, lo, hi);
}

// One output value as a binary32 pattern whose low byte is the int8 container.
// `r` is the residual's byte with its top bit flipped (its value + 128).
template <int ACT, bool RES>
__device__ __forceinline__ uint32_t requant(int acc, float mul, uint32_t r, const LinearArgs& p,
                                            const float* table, float lo, float hi) {
    const float a = (float)acc;
    const float zp = kMagic + (float)p.zp_y;
    float v;
    if constexpr (ACT == FQ_ACT_TABLE) {
        const float u = clamp3(__builtin_fmaf(a, mul, kMagic + (float)p.zp_t), kMagic,
                               kMagic + (float)((1 << p.table_bits) - 1));
        v = table[__builtin_bit_cast(uint32_t, u) - kMagicBits];
    }
    if constexpr (RES) {
        const float z = __builtin_fmaf((float)r, p.mul_r, p.add_r);
        if constexpr (ACT == FQ_ACT_TABLE)
            v = v + z;
        else if constexpr (ACT == FQ_ACT_RELU)
            v = fmaxf(a * mul, 0.0f) + z;
        else
            v = __builtin_fmaf(a, mul, z);
        v = v + kMagic;
    } else if constexpr (ACT == FQ_ACT_TABLE) {
        v = v + zp;
    } else {
        v = __builtin_fmaf(a, mul, zp);
        // max(., 0) commutes with the rounding: the lower end of the clamp
        if constexpr (ACT == FQ_ACT_RELU) lo = fmaxf(lo, zp);
    }
    return __builtin_bit_cast(uint32_t, clamp3(v, lo, hi));
}

// ---------------------------------------------------------------------------
// Tile kernel: 64 channels x 64 rows a workgroup, 64 inputs a step
// ---------------------------------------------------------------------------

constexpr int kTile = 64;
constexpr int kStep = 64;
constexpr int kPitch = kStep + 16;

// 16 bytes of row `row` from input k on; what lies beyond the matrix is 0.
__device__ __forceinline__ vi4 load_unit(const int8_t* m, int64_t rows, int64_t row, int K, int k) {
    vi4 v = {0, 0, 0, 0};
    if (row < rows) {
        const int8_t* p = m + row * K + k;
        if (k + 16 <= K) {
            __builtin_memcpy(&v, p, 16);
        } else {
            uint32_t w[4] = {0, 0, 0, 0};
            for (int b = 0; b < 16 && k + b < K; ++b) w[b >> 2] |= (uint32_t)(uint8_t)p[b] << ((b & 3) * 8);
            v = vi4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
        }
    }
    return v;
}

template <int ACT, bool RES, bool ACC>
__global__ __launch_bounds__(kBlock) void linear_tile_kernel(LinearArgs p, int tiles_n) {
    __shared__ __align__(16) int8_t ws[kTile * kPitch], xs[kTile * kPitch];
    __shared__ float table[ACT == FQ_ACT_TABLE ? 4096 : 1];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t t0 = (int64_t)(blockIdx.x / tiles_n) * kTile;
    const int n0 = (int)(blockIdx.x % tiles_n) * kTile;
    if constexpr (ACT == FQ_ACT_TABLE)
        for (int i = t; i < (1 << p.table_bits); i += kBlock) table[i] = p.table[i];
    const int row = t >> 2, unit = (t & 3) * 16;
    const int wn = (wave & 1) * 32, wt = (wave >> 1) * 32;
    vi16 acc = {0};
    for (int k0 = 0; k0 < p.K; k0 += kStep) {
        const vi4 a = load_unit(p.w, p.N, n0 + row, p.K, k0 + unit);
        const vi4 b = load_unit(p.x, p.T, t0 + row, p.K, k0 + unit);
        __syncthreads();
        *reinterpret_cast<vi4*>(ws + row * kPitch + unit) = a;
        *reinterpret_cast<vi4*>(xs + row * kPitch + unit) = b;
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kStep; s += 32) {
            const int at = (lane & 31) * kPitch + s + (lane >> 5) * 16;
            acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(
                *reinterpret_cast<const vi4*>(ws + wn * kPitch + at),
                *reinterpret_cast<const vi4*>(xs + wt * kPitch + at), acc, 0, 0, 0);
        }
    }
    const int64_t tok = t0 + wt + (lane & 31);
    if (tok >= p.T) return;
    const int half = 1 << (p.bits - 1);
    const float lo = kMagic - (float)half, hi = kMagic + (float)(half - 1);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int n = n0 + wn + (lane >> 5) * 4 + (i & 3) + 8 * (i >> 2);
        if (n >= p.N) continue;
        const int64_t o = tok * p.N + n;
        const int s = acc[i] + (p.fold ? p.fold[n] : 0);
        if constexpr (ACC) {
            p.acc[o] = s;
        } else {
            const uint32_t r = RES ? (uint32_t)(uint8_t)(p.residual[o] ^ 0x80) : 0;
            p.y[o] = (int8_t)requant<ACT, RES>(s, p.mul[n], r, p, table, lo, hi);
        }
    }
}

// ---------------------------------------------------------------------------
// Folded bias and multipliers: a wavefront a channel
// ---------------------------------------------------------------------------

__global__ __launch_bounds__(kBlock) void linear_fold_kernel(LinearFoldArgs p) {
    const int n = blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6);
    if (n >= p.N) return;
    const int lane = threadIdx.x & 63;
    const int8_t* row = p.w + (int64_t)n * p.K;
    int sum = 0;
    for (int k = lane; k < p.K; k += 64) sum += row[k];
    for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (lane != 0) return;
    const double s_w = (double)p.s_w[n];
    const bool live = s_w > 0.0 && isfinite(s_w);
    const double s_n = (double)p.s_x * s_w;
    double b = live && p.bias ? (double)p.bias[n] / s_n : 0.0;
    b = b == b ? fmin(fmax(rint(b), -1073741824.0), 1073741824.0) : 0.0;
    p.fold[n] = (int)b - p.zp_x * sum;
    if (p.mul) p.mul[n] = live ? (float)fmin(s_n / (double)p.s_y, 3.4028234663852886e38) : 0.0f;
}

template <int ACT, bool RES, bool ACC>
void launch_tile(const LinearArgs& a, hipStream_t stream) {
    const int tiles_n = (a.N + kTile - 1) / kTile;
    const int64_t tiles = (a.T + kTile - 1) / kTile * tiles_n;
    launch_kernel(linear_tile_kernel<ACT, RES, ACC>, dim3((unsigned)tiles), dim3(kBlock), 0, stream,
                  a, tiles_n);
}

}  // namespace

hipError_t launch_linear_fold(const LinearFoldArgs& a, hipStream_t stream) {
    launch_kernel(linear_fold_kernel, dim3((unsigned)((a.N + 3) / 4)), dim3(kBlock), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_linear(const LinearArgs& a, hipStream_t stream) {
    const bool res = a.residual != nullptr;
    if (a.acc)
        launch_tile<FQ_ACT_NONE, false, true>(a, stream);
    else if (a.act == FQ_ACT_TABLE)
        res ? launch_tile<FQ_ACT_TABLE, true, false>(a, stream)
            : launch_tile<FQ_ACT_TABLE, false, false>(a, stream);
    else if (a.act == FQ_ACT_RELU)
        res ? launch_tile<FQ_ACT_RELU, true, false>(a, stream)
            : launch_tile<FQ_ACT_RELU, false, false>(a, stream);
    else
        res ? launch_tile<FQ_ACT_NONE, true, false>(a, stream)
            : launch_tile<FQ_ACT_NONE, false, false>(a, stream);
    return hipGetLastError();
}

}  // namespace fqvit
