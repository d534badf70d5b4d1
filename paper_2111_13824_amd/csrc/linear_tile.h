// Tile kernel of the linear layers (int8 x int8 -> int32 on the matrix cores,
// with bias, activation, residual and requantization in the epilogue).
#pragma once

#include "bytes_device.h"
#include "fqvit.h"
#include "fqvit_launch.h"
#include "layers_internal.h"

namespace fqvit {
namespace linear {

typedef int vi4 __attribute__((ext_vector_type(4)));
typedef int vi16 __attribute__((ext_vector_type(16)));
typedef float vf4 __attribute__((ext_vector_type(4)));
typedef int vi4u __attribute__((ext_vector_type(4), aligned(1)));     // at any address

constexpr int kBlock = 256;

// ---------------------------------------------------------------------------
// Epilogue
// ---------------------------------------------------------------------------

// Rounding to the nearest integer by adding kMagic: sums in [2^23, 2^24) have a
// step of 1, so v + kMagic is kMagic + rint(v) for |v| < 2^22, the integer in the
// low bits of the binary32 pattern.  Values beyond that range leave it on their
// own side (rounding is monotone), where the clamp that follows takes them.
// The conversion, the multiply-add and the clamp are three instructions a value;
// the 31-bit dyadic form of requant_dyadic_int8 takes a quarter-rate 64-bit
// multiply-add and a shift instead of the first two.
constexpr float kMagic = 12582912.0f;   // 1.5 * 2^23
constexpr uint32_t kMagicBits = 0x4B400000u;

__device__ __forceinline__ float clamp3(float v, float lo, float hi) {
    return __builtin_amdgcn_fmed3f(v, lo, hi);
}

// The epilogue's constants, as the kernels use them.
struct Epilogue {
    float zp, lo, hi;       // kMagic + the output's zero point and ends
    float zp_t, hi_t;       // kMagic + the table's zero point and last index
    float mul_r, add_r;
};

__device__ __forceinline__ Epilogue epilogue(const LinearArgs& p) {
    const int half = 1 << (p.bits - 1);
    return Epilogue{kMagic + (float)p.zp_y,
                    kMagic - (float)half,
                    kMagic + (float)(half - 1),
                    kMagic + (float)p.zp_t,
                    kMagic + (float)((1 << p.table_bits) - 1),
                    p.mul_r,
                    p.add_r};
}

// One output value as a binary32 pattern whose low byte is the int8 container.
// `r` is the residual + 128.
template <int ACT, bool RES>
__device__ __forceinline__ uint32_t requant(int acc, float mul, float r, const Epilogue& e,
                                            const float* table) {
    const float a = (float)acc;
    float v, lo = e.lo;
    if constexpr (ACT == FQ_ACT_TABLE) {
        const float u = clamp3(__builtin_fmaf(a, mul, e.zp_t), kMagic, e.hi_t);
        v = table[__builtin_bit_cast(uint32_t, u) - kMagicBits];
    }
    if constexpr (RES) {
        const float z = __builtin_fmaf(r, e.mul_r, e.add_r);
        if constexpr (ACT == FQ_ACT_TABLE)
            v = v + z;
        else if constexpr (ACT == FQ_ACT_RELU)
            v = fmaxf(a * mul, 0.0f) + z;
        else
            v = __builtin_fmaf(a, mul, z);
        v = v + kMagic;
    } else if constexpr (ACT == FQ_ACT_TABLE) {
        v = v + e.zp;
    } else {
        v = __builtin_fmaf(a, mul, e.zp);
        // max(., 0) commutes with the rounding: the lower end of the clamp
        if constexpr (ACT == FQ_ACT_RELU) lo = e.zp;
    }
    return __builtin_bit_cast(uint32_t, clamp3(v, lo, e.hi));
}

// Four patterns' low bytes in one dword, the first lowest.
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
    return lo | hi;
}

// Byte b of a dword of residuals, each with its top bit flipped, as a float.
__device__ __forceinline__ float byte_of(uint32_t w, int b) {
    return (float)((w >> (8 * b)) & 0xFFu);
}

// ---------------------------------------------------------------------------
// Tiles
// ---------------------------------------------------------------------------

// WN x WT wavefronts; each holds FN x FT blocks of 32 channels x 32 rows.  The
// channels are the matrix instruction's rows, so a lane holds channels that lie
// together of one row of x.
//
// Inputs are taken STEP bytes of a row at a time, NBUF stages of them in LDS.  A
// stage's rows are STEP bytes, in units of 16; the unit of inputs c lies at place
// c ^ (a slice of the row's number): the sixteen lanes that LDS serves at once
// read one unit of sixteen rows and find it in sixteen different columns of a
// 256-byte line, without a bank conflict, while the stage stays linear in the
// order in which loads fill it.
template <int WN_, int WT_, int FN_, int FT_, int STEP_, int NBUF_, bool DMA_, int PER>
struct Shape {
    static constexpr int WN = WN_, WT = WT_, FN = FN_, FT = FT_, STEP = STEP_, NBUF = NBUF_;
    static constexpr bool DMA = DMA_;
    static constexpr int threads = 64 * WN * WT;
    static constexpr int waves = PER * WN * WT / 4;       // a SIMD: PER workgroups a CU
    static constexpr int BN = 32 * WN * FN, BT = 32 * WT * FT;
    static constexpr int units = STEP / 16;                               // of a row
    // loads of a thread a stage
    static constexpr int UN = BN * units / threads, UT = BT * units / threads;
    static_assert(BN * units % threads == 0 && BT * units % threads == 0, "whole loads");
    static constexpr int bytes = (BN + BT) * STEP;
    static constexpr int slice = STEP == 128 ? 1 : 2;
    static constexpr int ahead = FN * FT == 1 ? STEP / 32 : 1;            // parts read ahead

    // The place in a stage of a row's unit.
    static __device__ __forceinline__ int place(int row, int unit) {
        return row * STEP + ((unit ^ (row >> slice)) & (units - 1)) * 16;
    }
    // Row and unit that thread t fills with its i-th load.
    static __device__ __forceinline__ int fill_row(int t, int i) { return (i * threads + t) / units; }
    static __device__ __forceinline__ int fill_unit(int t, int i) {
        return (t ^ (fill_row(t, i) >> slice)) & (units - 1);
    }
};

// The operands of 32 inputs and their products.  `wa` and `xa` are the places of a
// lane's first unit in the first blocks of its wavefront's channels and rows: those
// of the next 32 inputs differ in bits 5 and 6 alone, and the other blocks lie
// whole multiples of 32 rows on.
template <class S>
struct Part {
    vi4 a[S::FN], b[S::FT];

    __device__ __forceinline__ void read(const int8_t* s, int q, int wa, int xa) {
        // worked out anew each time: kept, the places of all parts and stages are
        // two dozen registers, which the widest tile does not have
        asm volatile("" : "+v"(wa), "+v"(xa));
        wa ^= 32 * q;
        xa ^= 32 * q;
#pragma unroll
        for (int f = 0; f < S::FN; ++f)
            a[f] = *reinterpret_cast<const vi4*>(s + wa + 32 * f * S::STEP);
#pragma unroll
        for (int g = 0; g < S::FT; ++g)
            b[g] = *reinterpret_cast<const vi4*>(s + S::BN * S::STEP + xa + 32 * g * S::STEP);
    }
    __device__ __forceinline__ void multiply(vi16 (&acc)[S::FN][S::FT]) const {
#pragma unroll
        for (int f = 0; f < S::FN; ++f)
#pragma unroll
            for (int g = 0; g < S::FT; ++g)
                acc[f][g] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[f], b[g], acc[f][g], 0, 0, 0);
    }
};

// Asks for LDS reads between the products, while there are any.
template <class S>
__device__ __forceinline__ void interleave() {
    constexpr int n = S::FN * S::FT;
#pragma unroll
    for (int i = 0; i < n; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, (S::FN + S::FT + n - 1) / n, 0);
    }
}

// Waits until at most N of this wavefront's loads are still on their way and its
// LDS reads have arrived, then for the workgroup.  Nothing moves across it.
template <int N>
__device__ __forceinline__ void arrive() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// What lanes of this wavefront wrote to LDS before, its other lanes read after, and
// what they read before is not yet overwritten.  LDS serves a wavefront's accesses
// in their order; this holds the compiler to it and is no instruction.
__device__ __forceinline__ void exchange() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// A matrix's rows from `row0` on as a buffer of at most kNone bytes (a tile's are
// 10 MiB at most): reads beyond its end give nothing.
constexpr unsigned kNone = 0x70000000u;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const int8_t* m, int64_t rows, int64_t row0,
                                                          int K) {
    const int64_t bytes = (rows - row0) * K;
    return __builtin_amdgcn_make_buffer_rsrc((void*)(m + row0 * K), (short)0,
                                             (int)(bytes < kNone ? bytes : kNone), 0x00020000);
}

// One load of 16 bytes a lane from a buffer straight into LDS: the wavefront's
// lanes one after another from `s` on.
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t m, int8_t* s, unsigned off) {
    typedef __attribute__((address_space(3))) void* lds_ptr;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(m, (lds_ptr)s, 16, off, 0, 0, 0);
}

// 16 bytes of a row of any alignment from input k on; beyond K they are 0.
__device__ __forceinline__ vi4 load_tail(const int8_t* row, int K, int k) {
    vi4 v = {0, 0, 0, 0};
    if (k + 16 <= K) {
        __builtin_memcpy(&v, row + k, 16);
    } else if (k < K && K >= 16) {
        // the row's last 16 bytes, moved down by the part that lies before k
        Bytes16 u;
        __builtin_memcpy(&u, row + K - 16, 16);
        v = __builtin_bit_cast(vi4, bytes_down(u, k + 16 - K));
    } else if (k < K) {
        unsigned __int128 u = 0;
#pragma unroll 1
        for (int j = K - 1; j >= k; --j) u = u << 8 | (uint8_t)row[j];
        v = __builtin_bit_cast(vi4, u);
    }
    return v;
}

// Up to `count` bytes or dwords of a lane's 16, in a loop that stays small: the
// rest of a row whose channels end inside a unit.  (Unrolled at each place that
// stores, these ends were most of the kernel's code, and fetching it was most of
// the time of a short product: 197 x 192 x 192 10.4 us.)
template <typename T>
__device__ __forceinline__ void store_end(T* y, vi4 v, int count) {
    unsigned __int128 u = __builtin_bit_cast(unsigned __int128, v);
#pragma unroll 1
    for (int j = 0; j < count; ++j) {
        y[j] = (T)u;
        u >>= 8 * sizeof(T);
    }
}

// 16 residuals of a row from channel n on; beyond N they are 0.
__device__ __forceinline__ vi4 load_end(const int8_t* row, int N, int n) {
    if (n >= N) return vi4{0, 0, 0, 0};
    if (N >= 16) {
        Bytes16 u;
        __builtin_memcpy(&u, row + N - 16, 16);
        return __builtin_bit_cast(vi4, bytes_down(u, n + 16 - N));
    }
    unsigned __int128 u = 0;
#pragma unroll 1
    for (int j = N - 1; j >= n; --j) u = u << 8 | (uint8_t)row[j];
    return __builtin_bit_cast(vi4, u);
}

// DMA: rows of whole 16-byte units on 16-byte aligned bases go straight into
// LDS; else through registers.
template <class S, int ACT, bool RES, bool ACC>
__global__ __launch_bounds__(S::threads, S::waves) void linear_tile_kernel(LinearArgs p, int tiles_n,
                                                                    unsigned tiles) {
    constexpr int FN = S::FN, FT = S::FT, STEP = S::STEP, Q = S::STEP / 32;
    // separate arrays: the compiler then waits for the loads into the one that
    // it reads, not for all of them
    __shared__ __align__(16) int8_t s0[S::bytes], s1[S::bytes], s2[S::NBUF == 3 ? S::bytes : 16];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    // Workgroups go to the eight dies in turn; each die takes a run of tiles that
    // lie together, channels first, so that its L2 keeps their rows of x.
    const unsigned die = blockIdx.x & 7, q8 = tiles >> 3, r8 = tiles & 7;
    const unsigned tile = die * q8 + min(die, r8) + (blockIdx.x >> 3);
    const int64_t t0 = (int64_t)(tile / tiles_n) * S::BT;
    const int n0 = (int)(tile % tiles_n) * S::BN;
    const int wn = (wave % S::WN) * 32 * FN, wt = (wave / S::WN) * 32 * FT;
    const int h = lane >> 5, K = p.K;
    const int wa = S::place(wn + (lane & 31), h), xa = S::place(wt + (lane & 31), h);
    const int nk = (K + STEP - 1) / STEP;

    // The accumulators start as the folded bias.
    vi16 acc[FN][FT];
    auto start = [&]() __attribute__((always_inline)) {
        const __amdgpu_buffer_rsrc_t fr = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(p.fold ? p.fold : (const int32_t*)p.x), (short)0, p.fold ? p.N * 4 : 0, 0x00020000);
#pragma unroll
        for (int f = 0; f < FN; ++f)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const vi4 v = __builtin_bit_cast(
                    vi4, __builtin_amdgcn_raw_buffer_load_b128(fr, 4 * (n0 + wn + 32 * f + 8 * q + 4 * h),
                                                               0, 0));
#pragma unroll
                for (int g = 0; g < FT; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[f][g][4 * q + i] = v[i];
            }
    };

    if constexpr (S::DMA) {
        const __amdgpu_buffer_rsrc_t wr = rows_of(p.w, p.N, n0, K), xr = rows_of(p.x, p.T, t0, K);
        constexpr int U = S::UN > S::UT ? S::UN : S::UT;
        unsigned off[U];
#pragma unroll
        for (int i = 0; i < U; ++i) off[i] = S::fill_row(t, i) * K + S::fill_unit(t, i) * 16;
        auto fill = [&](int8_t* s, int k) __attribute__((always_inline)) {
            // past the last stage: outside the buffers, nothing is read, and the loads
            // that arrive() counts stay the same
            const unsigned k0 = k < nk ? k * STEP : kNone;
#pragma unroll
            for (int i = 0; i < S::UN; ++i)
                load_to_lds(wr, s + 16 * (S::threads * i + 64 * wave), off[i] + k0);
#pragma unroll
            for (int i = 0; i < S::UT; ++i)
                load_to_lds(xr, s + S::BN * STEP + 16 * (S::threads * i + 64 * wave), off[i] + k0);
        };
        // The last stage of a K that is no multiple of STEP holds other bytes
        // behind the row: the units of the weights there count 0.
        auto last = [&](int8_t* s) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < S::UN; ++i)
                if ((nk - 1) * STEP + S::fill_unit(t, i) * 16 >= K)
                    *reinterpret_cast<vi4*>(s + 16 * (S::threads * i + t)) = vi4{0, 0, 0, 0};
            arrive<0>();
        };
        constexpr int kLoads = S::UN + S::UT;
        const bool ragged = K % STEP != 0;
        // After a stage's last LDS reads: the next one has arrived, and the stage's own
        // LDS is filled again.
        auto turn = [&](int8_t* cur, int8_t* next, int k) __attribute__((always_inline)) {
            arrive<(S::NBUF - 2) * kLoads>();
            if (ragged && k + 2 == nk) last(next);
            fill(cur, k + S::NBUF);
        };

        // the first stage and the folded bias on their way together, and the other
        // stages behind them
        fill(s0, 0);
        start();
        fill(s1, 1);
        if constexpr (S::NBUF == 3) fill(s2, 2);
        arrive<(S::NBUF - 1) * kLoads>();
        if (ragged && nk == 1) last(s0);

        // The stages left over come after the loops: a way round them inside would have
        // the compiler wait for the youngest load at the loop's head.
        int k = 0;
        if constexpr (S::ahead > 1) {
            // A part is a single product, too short to read under: all of the next
            // stage's parts are read under all products of this one, which lie in half
            // `b` of `part` (197 x 1024 x 1024 4.8 -> 4.4 us, 788 x 768 x 768 4.6 -> 4.3).
            Part<S> part[2][S::ahead];
            auto stage = [&](int8_t* cur, int8_t* next, int k, int b) __attribute__((always_inline)) {
                turn(cur, next, k);
#pragma unroll
                for (int q = 0; q < Q; ++q) part[b ^ 1][q].read(next, q, wa, xa);
#pragma unroll
                for (int q = 0; q < Q; ++q) part[b][q].multiply(acc);
            };
#pragma unroll
            for (int q = 0; q < Q; ++q) part[0][q].read(s0, q, wa, xa);
            int8_t* const stages[3] = {s0, s1, s2};
            constexpr int kTurn = S::NBUF % 2 ? 2 * S::NBUF : S::NBUF;
            for (; k + kTurn <= nk; k += kTurn)
#pragma unroll
                for (int i = 0; i < kTurn; ++i)
                    stage(stages[i % S::NBUF], stages[(i + 1) % S::NBUF], k + i, i & 1);
#pragma unroll
            for (int i = 0; i + 1 < kTurn; ++i)
                if (k + i < nk) stage(stages[i % S::NBUF], stages[(i + 1) % S::NBUF], k + i, i & 1);
        } else {
            // One stage, its first operands read before: each part's operands are read
            // under the products of the part before, those of the next stage's first
            // part under the last.  (Written with the loop above, the widest tile spills.)
            Part<S> part[2];
            auto stage = [&](int8_t* cur, int8_t* next, int k) __attribute__((always_inline)) {
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    if (q + 1 < Q) {
                        part[(q + 1) & 1].read(cur, q + 1, wa, xa);
                    } else {
                        turn(cur, next, k);
                        part[0].read(next, 0, wa, xa);
                    }
                    part[q & 1].multiply(acc);
                    interleave<S>();
                }
            };
            part[0].read(s0, 0, wa, xa);
            if constexpr (S::NBUF == 3) {
                int8_t* const stages[3] = {s0, s1, s2};
                for (; k + 3 <= nk; k += 3)
#pragma unroll
                    for (int i = 0; i < 3; ++i) stage(stages[i], stages[(i + 1) % 3], k + i);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (k + i < nk) stage(stages[i], stages[i + 1], k + i);
            } else {
                for (; k + 2 <= nk; k += 2) {
                    stage(s0, s1, k);
                    stage(s1, s0, k + 1);
                }
                if (k < nk) stage(s0, s1, k);
            }
        }
    } else {
        vi4 a[S::UN], b[S::UT];
        const int8_t *wrow[S::UN], *xrow[S::UT];
        const int unit = (t % S::units) * 16;
#pragma unroll
        for (int i = 0; i < S::UN; ++i)
            wrow[i] = p.w + (int64_t)min(n0 + S::fill_row(t, i), p.N - 1) * K;
#pragma unroll
        for (int i = 0; i < S::UT; ++i)
            xrow[i] = p.x + min(t0 + S::fill_row(t, i), p.T - 1) * K;
        auto load = [&](int k) __attribute__((always_inline)) {
            const int k0 = k * STEP + unit;
            if (k * STEP + STEP <= K) {
#pragma unroll
                for (int i = 0; i < S::UN; ++i) __builtin_memcpy(&a[i], wrow[i] + k0, 16);
#pragma unroll
                for (int i = 0; i < S::UT; ++i) __builtin_memcpy(&b[i], xrow[i] + k0, 16);
            } else {
#pragma unroll
                for (int i = 0; i < S::UN; ++i) a[i] = load_tail(wrow[i], K, k0);
#pragma unroll
                for (int i = 0; i < S::UT; ++i) b[i] = load_tail(xrow[i], K, k0);
            }
        };
        auto store = [&](int8_t* s) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < S::UN; ++i)
                *reinterpret_cast<vi4*>(s + S::place(S::fill_row(t, i), t % S::units)) = a[i];
#pragma unroll
            for (int i = 0; i < S::UT; ++i)
                *reinterpret_cast<vi4*>(s + S::BN * STEP + S::place(S::fill_row(t, i), t % S::units)) = b[i];
        };
        auto all = [&](const int8_t* s) __attribute__((always_inline)) {
            Part<S> part[2];
            part[0].read(s, 0, wa, xa);
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                if (q + 1 < Q) part[(q + 1) & 1].read(s, q + 1, wa, xa);
                part[q & 1].multiply(acc);
            }
        };
        load(0);
        start();
        store(s0);
        for (int k = 0; k < nk; k += 2) {
            if (k + 1 < nk) load(k + 1);
            __syncthreads();
            all(s0);
            if (k + 1 < nk) store(s1);
            if (k + 2 < nk) load(k + 2);
            __syncthreads();
            if (k + 1 < nk) all(s1);
            if (k + 2 < nk) store(s0);
        }
    }

    // Epilogue.  Lane (row, h) of a block holds channels 8 q + 4 h + 0 .. 3 of its
    // row, q = 0 .. 3.  A wavefront brings 32 rows at a time through LDS of its
    // own, so that its stores (and the residual's loads) are runs of the rows of 32
    // FN bytes in whole 16-byte units: 64 where FN = 2, half a line.
    vf4 mul[FN][4];
    if constexpr (!ACC) {
        const __amdgpu_buffer_rsrc_t mr =
            __builtin_amdgcn_make_buffer_rsrc((void*)p.mul, (short)0, p.N * 4, 0x00020000);
#pragma unroll
        for (int f = 0; f < FN; ++f)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                mul[f][q] = __builtin_bit_cast(
                    vf4, __builtin_amdgcn_raw_buffer_load_b128(mr, 4 * (n0 + wn + 32 * f + 8 * q + 4 * h),
                                                               0, 0));
    }
    arrive<0>();                        // the stages are free, no load under way
    constexpr int kUnits = ACC ? 4 : 2 * FN;          // of 16 bytes a row
    constexpr int kPitch = 16 * kUnits + 16;
    static_assert(32 * kPitch * S::WN * S::WT <= S::bytes && S::bytes >= 16384, "");
    int8_t* own = s0 + 32 * kPitch * wave;
    int8_t* mine = own + (lane & 31) * kPitch + 16 * h;
    // this lane's part of pass i over the rows in memory order
    constexpr int kRows = 64 / kUnits, kPasses = (32 + kRows - 1) / kRows;
    const int prow = lane / kUnits, punit = lane % kUnits;
    auto has = [&](int i) __attribute__((always_inline)) {       // a row of the block's 32
        return 64 % kUnits == 0 || (prow < kRows && prow + i * kRows < 32);
    };
    const int8_t* part_of = own + prow * kPitch + 16 * punit;
    const int64_t row0 = t0 + wt + prow;
    if constexpr (ACC) {
#pragma unroll
        for (int g = 0; g < FT; ++g)
#pragma unroll
            for (int j = 0; j < 8 * FN / kUnits; ++j) {
                const int f = j * kUnits / 8, q0 = j * kUnits / 2 % 4;
#pragma unroll
                for (int q = 0; q < kUnits / 2; ++q) {
                    const vi16& c = acc[f][g];
                    const int at = 4 * (q0 + q);
                    *reinterpret_cast<vi4*>(mine + 32 * q) = vi4{c[at], c[at + 1], c[at + 2], c[at + 3]};
                }
                exchange();
                const int n = n0 + wn + 32 * f + 8 * q0 + 4 * punit;
#pragma unroll
                for (int i = 0; i < kPasses; ++i) {
                    const vi4 v = *reinterpret_cast<const vi4*>(part_of + i * kRows * kPitch);
                    const int64_t row = row0 + 32 * g + i * kRows;
                    if (!has(i) || row >= p.T) continue;
                    int32_t* o = p.acc + row * p.N + n;
                    if (n + 4 <= p.N)
                        __builtin_memcpy(o, &v, 16);
                    else
                        store_end(o, v, p.N - n);
                }
                exchange();
            }
    } else {
        const Epilogue e = epilogue(p);
        float* table = reinterpret_cast<float*>(s1);
        if constexpr (ACT == FQ_ACT_TABLE) {
            for (int i = t; i < (1 << p.table_bits); i += S::threads) table[i] = p.table[i];
            __syncthreads();
        }
        const int first = n0 + wn + 16 * punit;
        const bool whole = first + 16 <= p.N;
#pragma unroll
        for (int g = 0; g < FT; ++g) {
            if constexpr (RES) {
                vi4 r[kPasses];
#pragma unroll
                for (int i = 0; i < kPasses; ++i) {
                    const int64_t row = row0 + 32 * g + i * kRows;
                    const int8_t* res = p.residual + row * p.N;
                    r[i] = vi4{0, 0, 0, 0};
                    if (!has(i) || row >= p.T) continue;
                    if (whole)
                        __builtin_memcpy(&r[i], res + first, 16);
                    else
                        r[i] = load_end(res, p.N, first);
                }
#pragma unroll
                for (int i = 0; i < kPasses; ++i)
                    if (has(i))
                        *reinterpret_cast<vi4*>(const_cast<int8_t*>(part_of) + i * kRows * kPitch) = r[i];
                exchange();
            }
#pragma unroll
            for (int f = 0; f < FN; ++f) {
                // In memory's order a block's first 16 channels belong to the low
                // half of the wavefront, the others to the high half: two swaps
                // between the halves each way.
                uint32_t d[4], r[4] = {0, 0, 0, 0};
                if constexpr (RES) {
                    const vi4 v = *reinterpret_cast<const vi4*>(mine + 32 * f);
                    const auto x = __builtin_amdgcn_permlane32_swap((uint32_t)v[0], (uint32_t)v[1], false, false);
                    const auto z = __builtin_amdgcn_permlane32_swap((uint32_t)v[2], (uint32_t)v[3], false, false);
                    r[0] = x[0] ^ 0x80808080u;
                    r[1] = z[0] ^ 0x80808080u;
                    r[2] = x[1] ^ 0x80808080u;
                    r[3] = z[1] ^ 0x80808080u;
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[i] = requant<ACT, RES>(acc[f][g][4 * q + i], mul[f][q][i], byte_of(r[q], i), e, table);
                    d[q] = pack4(v[0], v[1], v[2], v[3]);
                }
                const auto x = __builtin_amdgcn_permlane32_swap(d[0], d[2], false, false);
                const auto z = __builtin_amdgcn_permlane32_swap(d[1], d[3], false, false);
                *reinterpret_cast<vi4*>(mine + 32 * f) = vi4{(int)x[0], (int)x[1], (int)z[0], (int)z[1]};
            }
            exchange();
            // with a residual, the place in a row worked out here: kept from the residual's
            // loads on as an offset of 64 bits and a count, it was spilled in tiles of 256 x 128
            int n = first;
            if constexpr (RES) asm volatile("" : "+v"(n));
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                const vi4 v = *reinterpret_cast<const vi4*>(part_of + i * kRows * kPitch);
                const int64_t row = row0 + 32 * g + i * kRows;
                if (!has(i) || row >= p.T) continue;
                int8_t* y = p.y + row * p.N + n;
                // large results pass through L2 without staying: 12608 x 768 x 2304
                // 32.1 -> 29.8 us, 12608 x 768 x 768 16.1 -> 14.7
                if (whole && S::BN * S::BT > 64 * 64)
                    __builtin_nontemporal_store(v, reinterpret_cast<vi4u*>(y));
                else if (whole)
                    __builtin_memcpy(y, &v, 16);
                else
                    store_end(y, v, p.N - n);
            }
            exchange();
        }
    }
}

// ---------------------------------------------------------------------------
// Launches (tiles: instantiated in linear_tile.hip)
// ---------------------------------------------------------------------------

// 256 channels x 64 FT rows.  Two stages of 128 inputs, whole 128-byte lines of the
// rows, or three of 64, half lines: 12608 x 768 x 2304 takes 30.2 us with the first and
// 32.4 with the second (inputs that were not read just before), the longer
// products 9232 x 4096 x 1024 and 9232 x 1024 x 4096 the same with both.  The smallest
// has room for two workgroups on a CU with the second.
template <int FT>
using TileW = Shape<4, 2, 2, FT, (FT > 2 ? 128 : 64), (FT > 2 ? 2 : 3), true, (FT > 2 ? 1 : 2)>;
// Smaller tiles: whole 128-byte lines of the rows at a time, which halves the
// requests to L2 (64 inputs: 1560 TOPS in tiles of 128 x 128 instead of 1870).
typedef Shape<2, 2, 2, 2, 128, 2, true, 2> Tile128;
typedef Shape<2, 2, 1, 1, 128, 3, true, 3> Tile64;
// Rows of any length on bases of any alignment.
typedef Shape<2, 2, 2, 2, 128, 2, false, 2> Tile128R;
typedef Shape<2, 2, 1, 1, 128, 2, false, 3> Tile64R;
typedef Shape<4, 2, 2, 4, 64, 2, false, 1> Tile256R;

template <class S>
void launch_tiles(const LinearArgs& a, hipStream_t stream);

// 16 FT rows of x a workgroup (linear_rows.hip).
template <int FT>
void launch_rows(const LinearArgs& a, hipStream_t stream);

}  // namespace linear
}  // namespace fqvit
