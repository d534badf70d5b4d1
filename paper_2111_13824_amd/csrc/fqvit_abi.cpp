// C ABI of libfqvit (declared in include/fqvit.h): argument validation, the
// host-side integer constants of I-Exp, and the kernel launches.  Nothing here
// allocates or synchronises; the only state is the per-thread pair of timing
// events of fq_time_next_call, consumed by the next entry-point call.
#include "fqvit.h"

#include <cmath>
#include <cstdint>

#include "fqvit_internal.h"
#include "layers_internal.h"
#include "stream_internal.h"

namespace {

constexpr int32_t kMaxC = 8192;
constexpr int32_t kMaxLk = 4096;
constexpr int32_t kMaxD = 256;
// The alpha search's grid has one y index per block of 64 rows: at most
// 65535 of them.
constexpr int64_t kMaxCalibT = (int64_t)65535 * 64;

fq_status from_hip(hipError_t e) { return e == hipSuccess ? FQ_OK : FQ_ERR_HIP; }

thread_local fqvit::LaunchEvents t_events;

// Clears the timing events when an entry point returns, whatever the path.
struct ConsumeEvents {
    ~ConsumeEvents() { t_events = fqvit::LaunchEvents{}; }
};

// Integer constants of Algorithm 1 (Supplement A.2) for input scale s, plus the
// bounds that let the kernels use 32-bit and 24-bit arithmetic.
fq_status lis_constants(float s_logit, int32_t bits, int32_t n, int32_t Lk,
                        fqvit::LisConsts* k) {
    if (!(s_logit >= 1e-4f && s_logit <= 0.5f)) return FQ_ERR_PARAM;
    if (bits < 1 || bits > 8 || n < 1 || n > 30) return FQ_ERR_PARAM;
    const double s = (double)s_logit;
    const double q_ln2 = std::floor(-0.69314718055994530942 / s);   // floor(-ln2 / s)
    const double q_b = std::floor(1.353 / s);                       // floor(b / s)
    const double q_c = std::floor(0.344 / ((0.3585 * s) * s));      // floor(c / (a s^2))
    const uint64_t d = (uint64_t)(-q_ln2);
    const uint64_t qb = (uint64_t)q_b;
    const uint64_t qc = (uint64_t)q_c;
    // q_p + q_b lies in [q_b - d + 1, q_b]: positive and below 2^16; 3 q_L < 2^32.
    if (d < 1 || qb < d || qb >= 65536 || 3 * (qb * qb + qc) >= (1ull << 32)) return FQ_ERR_PARAM;
    int pre = 0;
    while ((d << pre) <= 256) ++pre;
    const uint64_t dp = d << pre;
    if ((uint64_t)n * dp * dp >= (1ull << 32) || (uint64_t)n * dp >= (1ull << 24)) return FQ_ERR_PARAM;
    // The row sum (and 2 sum + e) must stay below 2^63.
    const unsigned __int128 emax = (unsigned __int128)(qb * qb + qc) << n;
    if ((unsigned __int128)(2 * (uint64_t)Lk + 1) * emax >= ((unsigned __int128)1 << 63))
        return FQ_ERR_HEADROOM;
    k->d_ln2 = (uint32_t)d;
    k->qb = (uint32_t)qb;
    k->qc = (uint32_t)qc;
    k->u_max = (uint32_t)(n * d);
    k->magic = (uint32_t)((1ull << 32) / dp + 1);
    k->pre = pre;
    k->n = n;
    k->top = (1 << bits) - 1;
    // The float path: every e = qL 2^(n - z) is exact in binary32 (qL < 2^24)
    // and 2S + e stays below 2^52 (exact in binary64).
    const uint64_t qlmax = qb * qb + qc;
    k->fp_ok = qlmax < (1ull << 24) &&
               (unsigned __int128)(2 * (uint64_t)Lk + 1) * ((unsigned __int128)qlmax << n) <
                   ((unsigned __int128)1 << 52);
    // The screened float path divides by d through a signed 24-bit
    // multiply-high: floor(a / d) for a in [-n d, d) scaled by 2^s_pre.  With
    // ds = d << s_pre in (512, 1024] (or d itself when larger; fp_ok keeps it
    // below 2^11) and n <= 30, n ds < 2^23 and n ds^2 < 2^32, so it is exact.
    k->s_pre = 0;
    while ((d << k->s_pre) <= 512) ++k->s_pre;
    k->s_magic = (int32_t)((1ull << 32) / (d << k->s_pre));
    k->s_add = (float)((double)qb - (double)d + 1.0 - 8388608.0);
    k->s_qc = (float)qc;
    return FQ_OK;
}

bool grid_fits(int64_t G, int32_t Lq, int32_t rows_per_block) {
    const int64_t tiles = (Lq + rows_per_block - 1) / rows_per_block;
    return G <= (int64_t)0x7FFFFFFF / (tiles > 0 ? tiles : 1);
}

// N2 / 2^N1: the 31-bit dyadic form of M = s_in / s_out.
void dyadic(float s_in, float s_out, int64_t* n2, int32_t* n1) {
    const double M = (double)s_in / (double)s_out;
    int e = 0;
    (void)std::frexp(M, &e);
    int64_t N1 = 31 - (int64_t)e;
    N1 = N1 < 0 ? 0 : (N1 > 62 ? 62 : N1);
    double m = std::floor(std::ldexp(M, (int)N1));
    if (m > 2147483647.0) m = 2147483647.0;
    *n2 = (int64_t)m;
    *n1 = (int32_t)N1;
}

constexpr int32_t kMaxN = 1 << 20;      // output channels of a linear layer
// Products of (x - zp) w, |.| <= 255 * 128, of this many inputs stay below 2^30,
// as the folded bias does: every accumulator fits int32.
constexpr int32_t kMaxK = 32768;

constexpr int32_t kMaxHeads = 1024;

// num / den as a binary32 multiplier (at most the largest finite one).
float multiplier(double num, double den) {
    return (float)std::fmin(num / den, 3.4028234663852886e38);
}

bool positive(float s) { return s > 0.0f && std::isfinite(s); }
bool int8_zp(int32_t zp) { return zp >= -128 && zp <= 127; }

// Sizes of a linear product.  A launch has fewer than 2^32 threads: the smallest
// tiles, 64 x 64, have 256 each.
bool linear_sizes(int64_t T, int32_t N, int32_t K) {
    if (T < 0 || T > ((int64_t)1 << 40) || N < 1 || N > kMaxN || K < 1 || K > kMaxK) return false;
    return (T + 63) / 64 * ((N + 63) / 64) < ((int64_t)1 << 24);
}

// Tokens of the rotation and of the heads' way back: a wavefront holds one or more.
constexpr int64_t kMaxTokens = (int64_t)1 << 25;
bool token_count(int64_t B, int32_t L) {
    return B >= 0 && L >= 0 && (L == 0 || B <= kMaxTokens / L);
}

// The launch, where this build has its kernels.
template <typename A>
fq_status launched(hipError_t (*launch)(const A&, hipStream_t), const A& a, void* stream) {
    return launch ? from_hip(launch(a, (hipStream_t)stream)) : FQ_ERR_HIP;
}

}  // namespace

// Workspace of the calibration: the min/max partials, the per-block error sums
// of every candidate alpha and channel, and the per-channel totals.
size_t fqvit::ptf_calibrate_workspace_bytes(int64_t T, int32_t C, int32_t K) {
    const int64_t nb = (T + kPtfErrBlock - 1) / kPtfErrBlock;
    return (size_t)kMinmaxParts * 2 * sizeof(float) + (size_t)(K + 1) * nb * C * sizeof(double) +
           (size_t)(K + 1) * C * sizeof(double);
}

const fqvit::LaunchEvents& fqvit::launch_events() { return t_events; }
void fqvit::set_launch_events(hipEvent_t start, hipEvent_t stop) {
    t_events.start = start;
    t_events.stop = stop;
}

extern "C" {

const char* fq_status_str(int status) {
    switch (status) {
        case FQ_OK: return "FQ_OK";
        case FQ_ERR_NULL: return "FQ_ERR_NULL: a required pointer is NULL";
        case FQ_ERR_SHAPE: return "FQ_ERR_SHAPE: a size is out of the supported range";
        case FQ_ERR_PARAM: return "FQ_ERR_PARAM: a scalar parameter is out of range";
        case FQ_ERR_HEADROOM: return "FQ_ERR_HEADROOM: the i-exp row sum could overflow 64 bits";
        case FQ_ERR_HIP: return "FQ_ERR_HIP: the HIP runtime rejected a launch";
        case FQ_ERR_SCRATCH:
            return "FQ_ERR_SCRATCH: the call needs more than the library's fixed device scratch holds";
        default: return "unknown fq_status";
    }
}

int32_t fq_version(void) { return 100; }

fq_status fq_time_next_call(void* start_event, void* stop_event) {
    t_events.start = (hipEvent_t)start_event;
    t_events.stop = (hipEvent_t)stop_event;
    return FQ_OK;
}

fq_status ptf_layernorm_int8(const int8_t* x_q, int64_t T, int32_t C, int32_t zp_in,
                             const uint8_t* alpha, int32_t K, const float* gamma,
                             const float* beta, float s_out, int32_t zp_out, int32_t bits,
                             int8_t* y_q, void* stream) {
    ConsumeEvents consume;
    if (T < 0 || C < 1 || C > kMaxC) return FQ_ERR_SHAPE;
    if (bits < 2 || bits > 8 || K < 0 || K > 7) return FQ_ERR_PARAM;
    if (!(s_out > 0.0f) || !std::isfinite(s_out)) return FQ_ERR_PARAM;
    const int32_t half = 1 << (bits - 1);
    if (zp_in < -half || zp_in >= half || zp_out < -half || zp_out >= half) return FQ_ERR_PARAM;
    if (T == 0) return FQ_OK;
    if (!x_q || !alpha || !gamma || !beta || !y_q) return FQ_ERR_NULL;
    fqvit::LnArgs a{x_q, y_q, alpha, gamma, beta, T, C, zp_in, K, s_out, zp_out, bits};
    return from_hip(fqvit::launch_ptf_layernorm(a, (hipStream_t)stream));
}

fq_status lis_softmax_log4(const int32_t* logits, int64_t G, int32_t Lq, int32_t Lk,
                           const int32_t* bias, int32_t Hb, float s_logit, int32_t bits,
                           int32_t exp_n, uint8_t* codes, int32_t ld_codes, void* stream) {
    ConsumeEvents consume;
    // codes of up to 4 bits two per byte, wider codes one per byte
    const int32_t row_bytes = (bits >= 5 && bits <= 8) ? Lk : (Lk + 1) / 2;
    if (G < 0 || Lq < 0 || Lk < 1 || Lk > kMaxLk || ld_codes < row_bytes || (bias && Hb < 1) ||
        !grid_fits(G, Lq, 64))
        return FQ_ERR_SHAPE;
    fqvit::LisConsts k;
    const fq_status st = lis_constants(s_logit, bits, exp_n, Lk, &k);
    if (st != FQ_OK) return st;
    if (G == 0 || Lq == 0) return FQ_OK;
    if (!logits || !codes) return FQ_ERR_NULL;
    fqvit::LisArgs a{};
    a.logits = logits;
    a.bias = bias;
    a.Hb = bias ? Hb : 1;
    a.G = G;
    a.Lq = Lq;
    a.Lk = Lk;
    a.k = k;
    a.codes = codes;
    a.ld_codes = ld_codes;
    return from_hip(fqvit::launch_lis(a, (hipStream_t)stream));
}

fq_status lis_attn_v_shift(const uint8_t* codes, int32_t ld_codes, const int8_t* v,
                           int32_t zp_v, int64_t G, int32_t Lq, int32_t Lk, int32_t d,
                           int32_t bits, int32_t* out, void* stream) {
    ConsumeEvents consume;
    if (G < 0 || Lq < 0 || Lk < 1 || Lk > kMaxLk || d < 1 || d > kMaxD ||
        ld_codes < (Lk + 1) / 2 || !grid_fits(G, Lq, 16))
        return FQ_ERR_SHAPE;
    if (bits < 1 || bits > 4 || zp_v < -128 || zp_v > 127) return FQ_ERR_PARAM;
    if (G == 0 || Lq == 0) return FQ_OK;
    if (!codes || !v || !out) return FQ_ERR_NULL;
    fqvit::AvArgs a{codes, ld_codes, v, zp_v, G, Lq, Lk, d, (1 << bits) - 1, out};
    return from_hip(fqvit::launch_attn_v_shift(a, (hipStream_t)stream));
}

fq_status lis_attn_v_shift_wide(const uint8_t* codes, int32_t ld_codes, const int8_t* v,
                                int32_t zp_v, int64_t G, int32_t Lq, int32_t Lk, int32_t d,
                                int32_t bits, int64_t* out, void* stream) {
    ConsumeEvents consume;
    const int32_t row_bytes = (bits >= 5 && bits <= 8) ? Lk : (Lk + 1) / 2;
    if (G < 0 || Lq < 0 || Lk < 1 || Lk > kMaxLk || d < 1 || d > kMaxD || ld_codes < row_bytes ||
        !grid_fits(G, Lq, 16))
        return FQ_ERR_SHAPE;
    if (bits < 1 || bits > 8 || zp_v < -128 || zp_v > 127) return FQ_ERR_PARAM;
    if (G == 0 || Lq == 0) return FQ_OK;
    if (!codes || !v || !out) return FQ_ERR_NULL;
    const int32_t N = (1 << bits) - 1;
    fqvit::AvWideArgs a{codes, ld_codes, v, zp_v, G, Lq, Lk, d, bits, N < 44 ? N : 44, out};
    return from_hip(fqvit::launch_attn_v_shift_wide(a, (hipStream_t)stream));
}

fq_status lis_attention_head(const int32_t* logits, const int32_t* bias, int32_t Hb,
                             int64_t G, int32_t Lq, int32_t Lk, float s_logit, int32_t bits,
                             int32_t exp_n, const int8_t* v, int32_t zp_v, int32_t d,
                             int32_t* out, uint8_t* codes_out, int32_t ld_codes, void* stream) {
    ConsumeEvents consume;
    if (G < 0 || Lq < 0 || Lk < 1 || Lk > kMaxLk || d < 1 || d > kMaxD || (bias && Hb < 1) ||
        (codes_out && ld_codes < (Lk + 1) / 2) || !grid_fits(G, Lq, 64))
        return FQ_ERR_SHAPE;
    if (zp_v < -128 || zp_v > 127) return FQ_ERR_PARAM;
    if (bits > 4) return FQ_ERR_PARAM;   // the BitShift product shifts by at most 15
    fqvit::LisConsts k;
    const fq_status st = lis_constants(s_logit, bits, exp_n, Lk, &k);
    if (st != FQ_OK) return st;
    if (G == 0 || Lq == 0) return FQ_OK;
    if (!logits || !v || !out) return FQ_ERR_NULL;
    fqvit::LisArgs a{};
    a.logits = logits;
    a.bias = bias;
    a.Hb = bias ? Hb : 1;
    a.G = G;
    a.Lq = Lq;
    a.Lk = Lk;
    a.k = k;
    a.v = v;
    a.zp_v = zp_v;
    a.d = d;
    a.out = out;
    a.codes = codes_out;
    a.ld_codes = codes_out ? ld_codes : 0;
    return from_hip(fqvit::launch_lis(a, (hipStream_t)stream));
}

fq_status lis_attention_qk(const int8_t* q, const int8_t* k, int32_t zp_q, int32_t zp_k,
                           int32_t dk, const int32_t* bias, int32_t Hb, int64_t G, int32_t Lq,
                           int32_t Lk, float s_logit, int32_t bits, int32_t exp_n,
                           const int8_t* v, int32_t zp_v, int32_t d, int32_t* out, void* stream) {
    ConsumeEvents consume;
    if (G < 0 || G > 0x7FFFFFFF || Lq < 0 || Lk < 1 || Lk > fqvit::kQkMaxLk || d < 1 || d > 64 ||
        (dk != 32 && dk != 64) || (bias && Hb < 1))
        return FQ_ERR_SHAPE;
    if (zp_q < -128 || zp_q > 127 || zp_k < -128 || zp_k > 127 || zp_v < -128 || zp_v > 127)
        return FQ_ERR_PARAM;
    if (bits > 4) return FQ_ERR_PARAM;   // the BitShift product shifts by at most 15
    fqvit::LisConsts kc;
    const fq_status st = lis_constants(s_logit, bits, exp_n, Lk, &kc);
    if (st != FQ_OK) return st;
    if (G == 0 || Lq == 0) return FQ_OK;
    if (!q || !k || !v || !out) return FQ_ERR_NULL;
    if (((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k)) & 15) != 0)
        return FQ_ERR_PARAM;
    fqvit::LisArgs a{};
    a.bias = bias;
    a.Hb = bias ? Hb : 1;
    a.G = G;
    a.Lq = Lq;
    a.Lk = Lk;
    a.k = kc;
    a.v = v;
    a.zp_v = zp_v;
    a.d = d;
    a.out = out;
    const fqvit::QkInput in{q, k, zp_q, zp_k, dk};
    return from_hip(fqvit::launch_lis_qk(a, in, (hipStream_t)stream));
}

size_t fq_ptf_calibrate_workspace_bytes(int64_t T, int32_t C, int32_t K) {
    if (T < 1 || T > kMaxCalibT || C < 1 || C > kMaxC || K < 0 || K > 7) return 0;
    return fqvit::ptf_calibrate_workspace_bytes(T, C, K);
}

fq_status ptf_calibrate(const float* x, int64_t T, int32_t C, int32_t bits, int32_t K, double* s,
                        int32_t* zp, uint8_t* alpha, void* workspace, size_t workspace_bytes,
                        void* stream) {
    ConsumeEvents consume;
    if (T < 0 || T > kMaxCalibT || C < 1 || C > kMaxC) return FQ_ERR_SHAPE;
    if (bits < 2 || bits > 8 || K < 0 || K > 7) return FQ_ERR_PARAM;
    if (T == 0) return FQ_OK;
    if (!x || !s || !zp || !alpha || !workspace) return FQ_ERR_NULL;
    if (workspace_bytes < fqvit::ptf_calibrate_workspace_bytes(T, C, K)) return FQ_ERR_PARAM;
    fqvit::PtfCalibArgs a{x, T, C, bits, K, s, zp, alpha, workspace};
    return from_hip(fqvit::launch_ptf_calibrate(a, (hipStream_t)stream));
}

fq_status ptf_calibrate_noalloc(const float* x, int64_t T, int32_t C, int32_t bits, int32_t K,
                                double* s, int32_t* zp, uint8_t* alpha, void* stream) {
    ConsumeEvents consume;
    if (T < 0 || T > kMaxCalibT || C < 1 || C > kMaxC) return FQ_ERR_SHAPE;
    if (bits < 2 || bits > 8 || K < 0 || K > 7) return FQ_ERR_PARAM;
    if (T == 0) return FQ_OK;
    if (!x || !s || !zp || !alpha) return FQ_ERR_NULL;
    if (fqvit::ptf_calibrate_workspace_bytes(T, C, K) > FQ_NOALLOC_SCRATCH_BYTES)
        return FQ_ERR_SCRATCH;
    fqvit::PtfCalibArgs a{x, T, C, bits, K, s, zp, alpha, nullptr};
    return from_hip(fqvit::launch_ptf_calibrate_noalloc(a, (hipStream_t)stream));
}

fq_status ptf_quantize_int8(const float* x, int64_t T, int32_t C, const double* s,
                            const int32_t* zp, const uint8_t* alpha, int32_t bits, int8_t* x_q,
                            void* stream) {
    ConsumeEvents consume;
    if (T < 0 || C < 1 || C > kMaxC) return FQ_ERR_SHAPE;
    if (bits < 2 || bits > 8) return FQ_ERR_PARAM;
    if (T == 0) return FQ_OK;
    if (!x || !s || !zp || !alpha || !x_q) return FQ_ERR_NULL;
    fqvit::PtfQuantArgs a{x, T, C, s, zp, alpha, bits, x_q};
    return from_hip(fqvit::launch_ptf_quantize(a, (hipStream_t)stream));
}

fq_status requant_dyadic_int8(const int32_t* q, int64_t n, float s_in, float s_out,
                              int32_t zp_out, int32_t bits, int8_t* y, void* stream) {
    ConsumeEvents consume;
    if (n < 0) return FQ_ERR_SHAPE;
    if (bits < 2 || bits > 8) return FQ_ERR_PARAM;
    if (!(s_in > 0.0f) || !std::isfinite(s_in) || !(s_out > 0.0f) || !std::isfinite(s_out))
        return FQ_ERR_PARAM;
    const int32_t half = 1 << (bits - 1);
    if (zp_out < -half || zp_out >= half) return FQ_ERR_PARAM;
    if (n == 0) return FQ_OK;
    if (!q || !y) return FQ_ERR_NULL;
    int64_t n2;
    int32_t n1;
    dyadic(s_in, s_out, &n2, &n1);
    fqvit::RequantArgs a{q, n, n2, n1, zp_out, bits, y};
    return from_hip(fqvit::launch_requant(a, (hipStream_t)stream));
}

fq_status linear_fold_int8(const int8_t* w, int32_t N, int32_t K, const float* s_w,
                           const float* bias, int32_t zp_x, float s_x, float s_y, int32_t* fold,
                           float* mul, void* stream) {
    ConsumeEvents consume;
    if (!linear_sizes(1, N, K)) return FQ_ERR_SHAPE;
    if (!int8_zp(zp_x) || !positive(s_x) || (mul && !positive(s_y))) return FQ_ERR_PARAM;
    if (!w || !s_w || !fold) return FQ_ERR_NULL;
    const fqvit::LinearFoldArgs a{w, N, K, s_w, bias, zp_x, s_x, s_y, fold, mul};
    return launched(fqvit::launch_linear_fold, a, stream);
}

fq_status linear_int8(const int8_t* x, int64_t T, const int8_t* w, int32_t N, int32_t K,
                      const int32_t* fold, const float* mul, int32_t act, const float* table,
                      int32_t table_bits, int32_t zp_t, const int8_t* residual, int32_t zp_r,
                      float mul_r, int32_t zp_y, int32_t bits, int8_t* y, void* stream) {
    ConsumeEvents consume;
    if (!linear_sizes(T, N, K)) return FQ_ERR_SHAPE;
    if (act != FQ_ACT_NONE && act != FQ_ACT_RELU && act != FQ_ACT_TABLE) return FQ_ERR_PARAM;
    if (act == FQ_ACT_TABLE &&
        (table_bits < 4 || table_bits > 12 || zp_t < 0 || zp_t >= (1 << table_bits)))
        return FQ_ERR_PARAM;
    if (residual && (!int8_zp(zp_r) || !(mul_r >= 0x1p-20f && mul_r <= 0x1p20f)))
        return FQ_ERR_PARAM;
    if (bits < 2 || bits > 8) return FQ_ERR_PARAM;
    const int32_t half = 1 << (bits - 1);
    if (zp_y < -half || zp_y >= half) return FQ_ERR_PARAM;
    if (T == 0) return FQ_OK;
    if (!x || !w || !mul || !y || (act == FQ_ACT_TABLE && !table)) return FQ_ERR_NULL;
    fqvit::LinearArgs a{};
    a.x = x;
    a.w = w;
    a.fold = fold;
    a.mul = mul;
    a.T = T;
    a.N = N;
    a.K = K;
    a.act = act;
    if (act == FQ_ACT_TABLE) {
        a.table = table;
        a.table_bits = table_bits;
        a.zp_t = zp_t;
    }
    if (residual) {
        a.residual = residual;
        a.mul_r = mul_r;
        // 8 + 24 bits: the product and the difference are exact in binary64
        a.add_r = (float)((double)zp_y - (double)(128 + zp_r) * (double)mul_r);
    }
    a.zp_y = zp_y;
    a.bits = bits;
    a.y = y;
    return launched(fqvit::launch_linear, a, stream);
}

fq_status linear_int32(const int8_t* x, int64_t T, const int8_t* w, int32_t N, int32_t K,
                       const int32_t* fold, int32_t* out, void* stream) {
    ConsumeEvents consume;
    if (!linear_sizes(T, N, K)) return FQ_ERR_SHAPE;
    if (T == 0) return FQ_OK;
    if (!x || !w || !out) return FQ_ERR_NULL;
    fqvit::LinearArgs a{};
    a.x = x;
    a.w = w;
    a.fold = fold;
    a.T = T;
    a.N = N;
    a.K = K;
    a.acc = out;
    return launched(fqvit::launch_linear, a, stream);
}

fq_status fq_activation_table(int32_t kind, float s_t, int32_t zp_t, int32_t table_bits, float s_y,
                              float* table) {
    if (kind < FQ_FN_GELU || kind > FQ_FN_SILU || table_bits < 4 || table_bits > 12 || zp_t < 0 ||
        zp_t >= (1 << table_bits) || !positive(s_t) || !positive(s_y))
        return FQ_ERR_PARAM;
    if (!table) return FQ_ERR_NULL;
    auto value = [=](int u) {
        const double t = (double)s_t * (u - zp_t);
        double f;
        if (kind == FQ_FN_GELU)
            f = 0.5 * t * (1.0 + std::erf(t * 0.70710678118654752440));
        else if (kind == FQ_FN_GELU_TANH)
            f = 0.5 * t *
                (1.0 + std::tanh(0.79788456080286535588 * (t + 0.044715 * t * t * t)));
        else
            f = t < -700.0 ? 0.0 : t / (1.0 + std::exp(-t));   // exp's range ends at 709
        return f / (double)s_y;
    };
    // GELU and SiLU have an extremum inside: every value is checked, and none is
    // written unless all can be
    const int last = (1 << table_bits) - 1;
    for (int u = 0; u <= last; ++u)
        if (!(std::fabs(value(u)) <= 3.4028234663852886e38)) return FQ_ERR_PARAM;
    for (int u = 0; u <= last; ++u) table[u] = (float)value(u);
    return FQ_OK;
}

fq_status rope_table_int16(const int32_t* positions, int32_t axes, int64_t T, const double* freq,
                           const uint8_t* axis, int32_t P, int16_t* table, void* stream) {
    ConsumeEvents consume;
    if (T < 0 || T > kMaxTokens || axes < 1 || axes > 8 || P < 1 || P > kMaxD / 2)
        return FQ_ERR_SHAPE;
    if (T == 0) return FQ_OK;
    if (!positions || !freq || !axis || !table) return FQ_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(table) & 3) != 0) return FQ_ERR_PARAM;
    const fqvit::RopeTableArgs a{positions, axes, T, freq, axis, P, table};
    return launched(fqvit::launch_rope_table, a, stream);
}

fq_status rope_qkv_int8(const int8_t* qkv, int64_t B, int32_t L, int32_t Hq, int32_t Hkv, int32_t d,
                        float s_x, int32_t zp_x, const int16_t* table, int64_t table_rows, int32_t P,
                        int32_t interleaved, float s_q, int32_t zp_q, float s_k, int32_t zp_k,
                        int32_t bits, int8_t* q, int8_t* k, int8_t* v, void* stream) {
    ConsumeEvents consume;
    if (!token_count(B, L) || Hq < 1 || Hq > kMaxHeads || Hkv < 1 || Hkv > kMaxHeads || d < 1 ||
        d > kMaxD || P < 0 || P > d / 2)
        return FQ_ERR_SHAPE;
    if (P > 0 && table_rows != L && table_rows != B * L) return FQ_ERR_SHAPE;
    if (bits < 2 || bits > 8 || (interleaved != 0 && interleaved != 1)) return FQ_ERR_PARAM;
    const int32_t half = 1 << (bits - 1);
    if (!int8_zp(zp_x) || zp_q < -half || zp_q >= half || zp_k < -half || zp_k >= half)
        return FQ_ERR_PARAM;
    if (!positive(s_x) || !positive(s_q) || !positive(s_k)) return FQ_ERR_PARAM;
    if (B == 0 || L == 0) return FQ_OK;
    if (!qkv || !q || !k || !v || (P > 0 && !table)) return FQ_ERR_NULL;
    if (P > 0 && (reinterpret_cast<uintptr_t>(table) & 3) != 0) return FQ_ERR_PARAM;
    fqvit::RopeArgs a{};
    a.qkv = qkv;
    a.B = B;
    a.L = L;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.d = d;
    a.zp_x = zp_x;
    a.table = table;
    a.per_image = table_rows != L;
    a.P = P;
    a.interleaved = interleaved;
    a.m_q = multiplier((double)s_x, 16384.0 * (double)s_q);
    a.m_k = multiplier((double)s_x, 16384.0 * (double)s_k);
    a.zp_q = zp_q;
    a.zp_k = zp_k;
    a.bits = bits;
    a.q = q;
    a.k = k;
    a.v = v;
    return launched(fqvit::launch_rope_qkv, a, stream);
}

fq_status requant_heads_int8(const int32_t* q, int64_t B, int32_t H, int32_t L, int32_t d,
                             float s_in, float s_out, int32_t zp_out, int32_t bits, int8_t* y,
                             void* stream) {
    ConsumeEvents consume;
    if (!token_count(B, L) || H < 1 || H > kMaxHeads || d < 1 || d > kMaxD) return FQ_ERR_SHAPE;
    if (bits < 2 || bits > 8) return FQ_ERR_PARAM;
    if (!positive(s_in) || !positive(s_out)) return FQ_ERR_PARAM;
    const int32_t half = 1 << (bits - 1);
    if (zp_out < -half || zp_out >= half) return FQ_ERR_PARAM;
    if (B == 0 || L == 0) return FQ_OK;
    if (!q || !y) return FQ_ERR_NULL;
    fqvit::RequantHeadsArgs a{};
    a.r.q = q;
    dyadic(s_in, s_out, &a.r.N2, &a.r.N1);
    a.r.zp = zp_out;
    a.r.bits = bits;
    a.r.y = y;
    a.B = B;
    a.H = H;
    a.L = L;
    a.d = d;
    return launched(fqvit::launch_requant_heads, a, stream);
}

namespace {

fq_status rmsnorm(const int8_t* x, int32_t zp_x, const uint8_t* alpha, int32_t K, float m_x,
                  const int16_t* r, int64_t T, int32_t C, const float* gamma, float eps, float s_out,
                  int32_t zp_out, int32_t bits, int16_t* h, int8_t* y, float* scales, bool rows,
                  void* stream) {
    ConsumeEvents consume;
    if (T < 0 || T >= ((int64_t)1 << 24) || C < 1 || C > kMaxC) return FQ_ERR_SHAPE;
    if (bits < 2 || bits > 8 || !(eps >= 0.0f) || !std::isfinite(eps)) return FQ_ERR_PARAM;
    const int32_t half = 1 << (bits - 1);
    if (!rows && (!positive(s_out) || zp_out < -half || zp_out >= half)) return FQ_ERR_PARAM;
    // (x - zp_x) 2^K m_x stays below 2^21
    if (x && (!int8_zp(zp_x) || !(m_x >= 0x1p-20f && m_x <= 64.0f))) return FQ_ERR_PARAM;
    if (x && alpha && (K < 0 || K > 7)) return FQ_ERR_PARAM;
    if (T == 0) return FQ_OK;
    if (!r || !gamma || !h || !y || (rows && !scales)) return FQ_ERR_NULL;
    fqvit::RmsArgs a{};
    a.x = x;
    a.alpha = x ? alpha : nullptr;
    a.zp_x = zp_x;
    a.K = a.alpha ? K : 0;      // factors of 0 are not clamped below 0 by a K that is not looked at
    a.m_x = m_x;
    a.r = r;
    a.gamma = gamma;
    a.T = T;
    a.C = C;
    a.eps = eps;
    a.s_out = s_out;
    a.zp_out = zp_out;
    a.bits = bits;
    a.h = h;
    a.y = y;
    a.scales = scales;
    return launched(fqvit::launch_rmsnorm, a, stream);
}

constexpr int32_t kMaxCacheD = 128;
constexpr int32_t kMaxPage = 1024;
constexpr int64_t kMaxCacheKeys = (int64_t)1 << 20;
constexpr int64_t kMaxUnits = 65536;                    // sequences times key heads
constexpr int64_t kMaxGroups = (int64_t)1 << 24;        // workgroups of 256: fewer than 2^32 threads

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Sizes of a cache; its view.
bool cache_view(int8_t* k, int8_t* v, int64_t* weight, const int32_t* table, const int32_t* length,
                int32_t pages, int32_t page, int32_t max_pages, int32_t B, int32_t Hkv, int32_t d,
                fqvit::CacheView* c) {
    if (pages < 1 || pages > (1 << 30) || page < 16 || page > kMaxPage || (page & (page - 1)) != 0 ||
        max_pages < 1 || (int64_t)max_pages * page > kMaxCacheKeys || B < 0 || Hkv < 1 ||
        Hkv > kMaxHeads || (int64_t)B * Hkv > kMaxUnits || d < 16 || d > kMaxCacheD || d % 16 != 0)
        return false;
    int32_t log2_page = 0;
    while ((1 << log2_page) < page) ++log2_page;
    *c = fqvit::CacheView{k, v, weight, table, length, pages, max_pages, log2_page, B, Hkv, d};
    return true;
}

}  // namespace

fq_status rmsnorm_int8(const int8_t* x, int32_t zp_x, const uint8_t* alpha, int32_t K, float m_x,
                       const int16_t* r, int64_t T, int32_t C, const float* gamma, float eps,
                       float s_out, int32_t zp_out, int32_t bits, int16_t* h, int8_t* y,
                       void* stream) {
    return rmsnorm(x, zp_x, alpha, K, m_x, r, T, C, gamma, eps, s_out, zp_out, bits, h, y, nullptr,
                   false, stream);
}

fq_status rmsnorm_rows_int8(const int8_t* x, int32_t zp_x, const uint8_t* alpha, int32_t K,
                            float m_x, const int16_t* r, int64_t T, int32_t C, const float* gamma,
                            float eps, int32_t bits, int16_t* h, int8_t* y, float* scales,
                            void* stream) {
    return rmsnorm(x, zp_x, alpha, K, m_x, r, T, C, gamma, eps, 1.0f, 0, bits, h, y, scales, true,
                   stream);
}

fq_status kv_cache_append_int8(const int8_t* k, const int8_t* v, int32_t B, int32_t Hkv, int32_t L,
                               int32_t d, const int32_t* n_new, int8_t* k_pages, int8_t* v_pages,
                               int64_t* weight, int32_t pages, int32_t page, const int32_t* table,
                               int32_t max_pages, const int32_t* length, void* stream) {
    ConsumeEvents consume;
    fqvit::AppendArgs a{};
    if (!cache_view(k_pages, v_pages, weight, table, length, pages, page, max_pages, B, Hkv, d, &a.c) ||
        L < 0 || L > kMaxCacheKeys || (int64_t)B * Hkv * (L / 64 + 2) >= kMaxGroups)
        return FQ_ERR_SHAPE;
    if (B == 0 || L == 0) return FQ_OK;
    if (!k || !v || !k_pages || !v_pages || !table || !length) return FQ_ERR_NULL;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) ||
        !aligned(weight, 8))
        return FQ_ERR_PARAM;
    a.k = k;
    a.v = v;
    a.n_new = n_new;
    a.L = L;
    return launched(fqvit::launch_kv_append, a, stream);
}

namespace {

// Sizes of queries over a cache whose view holds.
bool query_sizes(int32_t B, int32_t Hq, int32_t Hkv, int32_t L) {
    if (Hq < 1 || Hq > kMaxHeads || Hkv < 1 || Hq % Hkv != 0 || L < 0 || L > kMaxCacheKeys) return false;
    const int64_t rows = (int64_t)L * (Hq / Hkv);
    return rows < ((int64_t)1 << 30) && (int64_t)B * Hkv * (rows / 16 + 1) < kMaxGroups;
}

}  // namespace

size_t fq_lis_attention_paged_workspace_bytes(int32_t B, int32_t Hq, int32_t Hkv, int32_t L,
                                              int32_t d, int64_t max_keys) {
    if (B < 1 || Hkv < 1 || !query_sizes(B, Hq, Hkv, L) || L < 1 || d < 1 || max_keys < 1 ||
        max_keys > kMaxCacheKeys)
        return 0;
    return fqvit::lis_paged_workspace ? fqvit::lis_paged_workspace(B, Hq, Hkv, L, d, max_keys) : 0;
}

fq_status lis_attention_paged(const int8_t* q, int32_t B, int32_t Hq, int32_t Hkv, int32_t L,
                              int32_t d, const int32_t* n_new, const int8_t* k_pages,
                              const int8_t* v_pages, int64_t* weight, int32_t pages, int32_t page,
                              const int32_t* table, int32_t max_pages, const int32_t* length,
                              int32_t zp_q, int32_t zp_k, int32_t zp_v, int32_t causal,
                              float s_logit, int32_t bits, int32_t exp_n, int32_t* out,
                              void* workspace, size_t workspace_bytes, void* stream) {
    ConsumeEvents consume;
    fqvit::PagedArgs a{};
    if (!cache_view(const_cast<int8_t*>(k_pages), const_cast<int8_t*>(v_pages), weight, table, length,
                    pages, page, max_pages, B, Hkv, d, &a.c) ||
        !query_sizes(B, Hq, Hkv, L))
        return FQ_ERR_SHAPE;
    if (!int8_zp(zp_q) || !int8_zp(zp_k) || !int8_zp(zp_v) || bits > 4 || (causal != 0 && causal != 1))
        return FQ_ERR_PARAM;
    const fq_status st = lis_constants(s_logit, bits, exp_n, max_pages * page, &a.k);
    if (st != FQ_OK) return st;
    if (B == 0 || L == 0) return FQ_OK;
    if (!q || !k_pages || !v_pages || !table || !length || !out) return FQ_ERR_NULL;
    const size_t need =
        fq_lis_attention_paged_workspace_bytes(B, Hq, Hkv, L, d, (int64_t)max_pages * page);
    if (need && !workspace) return FQ_ERR_NULL;
    if (workspace_bytes < need || !aligned(q, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) ||
        !aligned(out, 16) || !aligned(weight, 8) || (need && !aligned(workspace, 16)))
        return FQ_ERR_PARAM;
    a.q = q;
    a.n_new = n_new;
    a.Hq = Hq;
    a.L = L;
    a.group = Hq / Hkv;
    a.zp_q = zp_q;
    a.zp_v = zp_v;
    a.causal = causal;
    a.out = out;
    a.workspace = workspace;
    return launched(fqvit::launch_lis_paged, a, stream);
}

fq_status kv_cache_evict(int8_t* k_pages, int8_t* v_pages, int64_t* weight, int32_t pages,
                         int32_t Hkv, int32_t page, int32_t d, const int32_t* table,
                         int32_t max_pages, const int32_t* length, int32_t B, int32_t keep,
                         int32_t recent, const int32_t* table_out, int32_t max_out,
                         int32_t* length_out, int32_t* kept, void* stream) {
    ConsumeEvents consume;
    fqvit::EvictArgs a{};
    if (!cache_view(k_pages, v_pages, weight, table, length, pages, page, max_pages, B, Hkv, d, &a.c) ||
        keep < 1 || keep > kMaxCacheKeys || max_out < 1 || (int64_t)max_out * page > kMaxCacheKeys ||
        (int64_t)max_out * page < keep || (table_out == table && max_out != max_pages))
        return FQ_ERR_SHAPE;
    if (recent < 0 || recent > keep) return FQ_ERR_PARAM;
    if (B == 0) return FQ_OK;
    if (!k_pages || !v_pages || !weight || !table || !length || !table_out || !length_out || !kept)
        return FQ_ERR_NULL;
    if (!aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(weight, 8)) return FQ_ERR_PARAM;
    a.table_out = table_out;
    a.max_out = max_out;
    a.keep = keep;
    a.recent = recent;
    a.length_out = length_out;
    a.kept = kept;
    return launched(fqvit::launch_kv_evict, a, stream);
}

}  // extern "C"
