// Test-only stand-ins for the launchers of the linear layers, the rotary
// positions and the heads' way back to rows: each keeps what the C ABI's host
// code passed it and launches nothing (tests/test_layers_abi.py).
#include "layers_internal.h"
#include "linear_plan.h"

namespace fqvit {

static int g_calls = 0;
static LinearArgs g_linear;
static RopeArgs g_rope;
static RequantHeadsArgs g_heads;

hipError_t launch_linear_fold(const LinearFoldArgs&, hipStream_t) { ++g_calls; return hipSuccess; }
hipError_t launch_linear(const LinearArgs& a, hipStream_t) {
    ++g_calls;
    g_linear = a;
    return hipSuccess;
}
hipError_t launch_rope_table(const RopeTableArgs&, hipStream_t) { ++g_calls; return hipSuccess; }
hipError_t launch_rope_qkv(const RopeArgs& a, hipStream_t) {
    ++g_calls;
    g_rope = a;
    return hipSuccess;
}
hipError_t launch_requant_heads(const RequantHeadsArgs& a, hipStream_t) {
    ++g_calls;
    g_heads = a;
    return hipSuccess;
}

}  // namespace fqvit

extern "C" {
int fq_test_layer_calls(void) { return fqvit::g_calls; }
// add_r of the last product; m_q, m_k of the last rotation
void fq_test_multipliers(float* out) {
    out[0] = fqvit::g_linear.add_r;
    out[1] = fqvit::g_rope.m_q;
    out[2] = fqvit::g_rope.m_k;
}
// The kernel that the last product would take (linear::Kernel).
int fq_test_linear_kernel(void) { return (int)fqvit::linear::plan(fqvit::g_linear); }
// N2, N1 of the last requantization; whether the last table had a row per image
void fq_test_integers(long long* out) {
    out[0] = fqvit::g_heads.r.N2;
    out[1] = fqvit::g_heads.r.N1;
    out[2] = fqvit::g_rope.per_image;
}
}
