// Arguments and launchers of the layers around the attention: linear layers,
// rotary positions, heads back to rows.  Weak: a host-only build of the C ABI
// (argument checks without kernels) may leave these launchers out; a call that
// reaches a missing one returns FQ_ERR_HIP.
#pragma once

#include "fqvit_internal.h"

namespace fqvit {

struct LinearFoldArgs {
    const int8_t* w;        // [N, K]
    int32_t N, K;
    const float* s_w;       // [N]
    const float* bias;      // nullable [N]
    int32_t zp_x;
    float s_x, s_y;
    int32_t* fold;          // [N] out
    float* mul;             // nullable [N] out
};

__attribute__((weak)) hipError_t launch_linear_fold(const LinearFoldArgs& a, hipStream_t stream);

struct LinearArgs {
    const int8_t* x;        // [T, K]
    const int8_t* w;        // [N, K]
    const int32_t* fold;    // nullable [N]
    const float* mul;       // [N] (int8 output)
    int64_t T;
    int32_t N, K;
    int32_t act;            // FQ_ACT_*
    const float* table;     // 2^table_bits values
    int32_t table_bits, zp_t;
    const int8_t* residual; // nullable [T, N]
    float mul_r, add_r;     // z = fma(r + 128, mul_r, add_r)
    int32_t zp_y, bits;
    int8_t* y;              // [T, N] int8 output, or
    int32_t* acc;           // [T, N] int32 output
};

__attribute__((weak)) hipError_t launch_linear(const LinearArgs& a, hipStream_t stream);

struct RopeTableArgs {
    const int32_t* positions;   // [axes, T]
    int32_t axes;
    int64_t T;
    const double* freq;         // [P]
    const uint8_t* axis;        // [P]
    int32_t P;
    int16_t* table;             // [T, P, 2]
};

__attribute__((weak)) hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t stream);

struct RopeArgs {
    const int8_t* qkv;          // [B, L, (Hq + 2 Hkv) d]
    int64_t B;
    int32_t L, Hq, Hkv, d;
    int32_t zp_x;
    const int16_t* table;       // [L or B L, P, 2]
    int32_t per_image;          // the table has a row for each (b, l)
    int32_t P;
    int32_t interleaved;
    float m_q, m_k;             // multipliers of queries and keys
    int32_t zp_q, zp_k, bits;
    int8_t *q, *k, *v;
};

__attribute__((weak)) hipError_t launch_rope_qkv(const RopeArgs& a, hipStream_t stream);

struct RequantHeadsArgs {
    RequantArgs r;              // q, y and the multiplier; n is unused
    int64_t B;
    int32_t H, L, d;
};

__attribute__((weak)) hipError_t launch_requant_heads(const RequantHeadsArgs& a, hipStream_t stream);

}  // namespace fqvit
