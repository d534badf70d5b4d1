// Linear layers of a few rows of x (one token, a small image) for gfx950: what
// counts is that every CU's loads are under way at once.
//
// A workgroup of eight wavefronts takes 16 channels; the wavefronts share the
// inputs, 64 of each row at a time, and load the weights from global memory
// straight into the matrix instruction's operands (no other wavefront needs
// them).  Their sums meet in LDS, where one thread adds the eight of each output.
#include "linear_tile.h"

namespace fqvit {
namespace linear {
namespace {

constexpr int kWaves = 8;
constexpr int kAhead = 4;       // steps of 64 inputs whose loads are under way

// 16 * FT rows of x: FT blocks of 16 channels x 16 rows a wavefront.
template <int FT, int ACT, bool RES, bool ACC>
__global__ __launch_bounds__(64 * kWaves) void linear_rows_kernel(LinearArgs p) {
    __shared__ int sums[kWaves][FT][256];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int n0 = blockIdx.x * 16;
    const int64_t t0 = (int64_t)blockIdx.y * (16 * FT);
    const int K = p.K, unit = (lane >> 4) * 16;
    const int8_t* w = p.w + (int64_t)min(n0 + (lane & 15), p.N - 1) * K;
    const int8_t* x[FT];
#pragma unroll
    for (int g = 0; g < FT; ++g) x[g] = p.x + min(t0 + 16 * g + (lane & 15), p.T - 1) * K;

    vi4 acc[FT] = {};
    const int full = K / 64;
    int s = wave;
    for (; s + (kAhead - 1) * kWaves < full; s += kAhead * kWaves) {
        vi4 a[kAhead], b[kAhead][FT];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int k = (s + i * kWaves) * 64 + unit;
            __builtin_memcpy(&a[i], w + k, 16);
#pragma unroll
            for (int g = 0; g < FT; ++g) __builtin_memcpy(&b[i][g], x[g] + k, 16);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int g = 0; g < FT; ++g)
                acc[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], b[i][g], acc[g], 0, 0, 0);
    }
    for (; s * 64 < K; s += kWaves) {
        const int k = s * 64 + unit;
        const bool whole = s < full;
        vi4 a, b[FT];
        if (whole) {
            __builtin_memcpy(&a, w + k, 16);
#pragma unroll
            for (int g = 0; g < FT; ++g) __builtin_memcpy(&b[g], x[g] + k, 16);
        } else {
            a = load_tail(w, K, k);
#pragma unroll
            for (int g = 0; g < FT; ++g) b[g] = load_tail(x[g], K, k);
        }
#pragma unroll
        for (int g = 0; g < FT; ++g)
            acc[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b[g], acc[g], 0, 0, 0);
    }
    // lane (row, q) holds channels 4 q + 0 .. 3 of its row: outputs in rows of 16
#pragma unroll
    for (int g = 0; g < FT; ++g)
        *reinterpret_cast<vi4*>(&sums[wave][g][(lane & 15) * 16 + (lane >> 4) * 4]) = acc[g];
    __syncthreads();
    const Epilogue e = epilogue(p);
#pragma unroll
    for (int o = t; o < 256 * FT; o += 64 * kWaves) {
        const int64_t row = t0 + (o >> 4);
        const int n = n0 + (o & 15);
        if (row >= p.T || n >= p.N) continue;
        int sum = p.fold ? p.fold[n] : 0;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) sum += sums[v][o >> 8][o & 255];
        const int64_t at = row * p.N + n;
        if constexpr (ACC) {
            p.acc[at] = sum;
        } else {
            const float r = RES ? (float)(p.residual[at] + 128) : 0.0f;
            p.y[at] = (int8_t)requant<ACT, RES>(sum, p.mul[n], r, e, p.table);
        }
    }
}

template <int FT, int ACT, bool RES, bool ACC>
void go(const LinearArgs& a, hipStream_t stream) {
    launch_kernel(linear_rows_kernel<FT, ACT, RES, ACC>,
                  dim3((unsigned)((a.N + 15) / 16), (unsigned)((a.T + 16 * FT - 1) / (16 * FT))),
                  dim3(64 * kWaves), 0, stream, a);
}

}  // namespace

template <int FT>
void launch_rows(const LinearArgs& a, hipStream_t stream) {
    const bool res = a.residual != nullptr;
    if (a.acc)
        go<FT, FQ_ACT_NONE, false, true>(a, stream);
    else if (a.act == FQ_ACT_TABLE)
        res ? go<FT, FQ_ACT_TABLE, true, false>(a, stream) : go<FT, FQ_ACT_TABLE, false, false>(a, stream);
    else if (a.act == FQ_ACT_RELU)
        res ? go<FT, FQ_ACT_RELU, true, false>(a, stream) : go<FT, FQ_ACT_RELU, false, false>(a, stream);
    else
        res ? go<FT, FQ_ACT_NONE, true, false>(a, stream) : go<FT, FQ_ACT_NONE, false, false>(a, stream);
}

template void launch_rows<1>(const LinearArgs&, hipStream_t);
template void launch_rows<2>(const LinearArgs&, hipStream_t);

}  // namespace linear
}  // namespace fqvit
