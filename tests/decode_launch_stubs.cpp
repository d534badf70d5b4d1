// Test-only stand-ins for the launchers of the step over a stream of tokens: each
// counts its calls and keeps what the C ABI's host code passed it
// (tests/test_decode_abi.py).
#include "stream_internal.h"

namespace fqvit {

static int g_calls = 0;
static PagedArgs g_paged;
static RmsArgs g_rms;

hipError_t launch_rmsnorm(const RmsArgs& a, hipStream_t) {
    ++g_calls;
    g_rms = a;
    return hipSuccess;
}
hipError_t launch_kv_append(const AppendArgs&, hipStream_t) { ++g_calls; return hipSuccess; }
size_t lis_paged_workspace(int32_t, int32_t, int32_t, int32_t L, int32_t, int64_t) { return L == 7 ? 96 : 0; }
hipError_t launch_lis_paged(const PagedArgs& a, hipStream_t) {
    ++g_calls;
    g_paged = a;
    return hipSuccess;
}
hipError_t launch_kv_evict(const EvictArgs&, hipStream_t) { ++g_calls; return hipSuccess; }

}  // namespace fqvit

extern "C" {
int fq_test_layer_calls(void) { return fqvit::g_calls; }
// group, log2 of the page, whether the last norm had factors
void fq_test_integers(long long* out) {
    out[0] = fqvit::g_paged.group;
    out[1] = fqvit::g_paged.c.log2_page;
    out[2] = fqvit::g_rms.alpha != nullptr;
}
// the bound of the last norm's factors
int fq_test_norm_bound(void) { return fqvit::g_rms.K; }
}
