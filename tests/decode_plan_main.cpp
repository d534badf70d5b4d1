// Test-only: how calls of the attention over a paged cache are divided, over drawn sizes
// (tests/test_decode_plan.py).  Prints the number of calls of each way; ends with 1 and
// the sizes where a plan does not hold.
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <random>

#include "lis_paged_plan.h"

using namespace fqvit::paged;

static int32_t B, Hq, Hkv, L;
static int64_t most;

static void hold(bool ok, const char* what) {
    if (ok) return;
    printf("%s: B %d Hq %d Hkv %d L %d keys %lld\n", what, B, Hq, Hkv, L, (long long)most);
    exit(1);
}

// Every size that the entry point lets through.
static bool allowed() {
    const int64_t rows = (int64_t)L * (Hq / Hkv);
    return (int64_t)B * Hkv <= 65536 && Hq <= 1024 && L <= (1 << 20) && rows < ((int64_t)1 << 30) &&
           (int64_t)B * Hkv * (rows / 16 + 1) < ((int64_t)1 << 24);
}

int main() {
    std::mt19937_64 rng(7);
    const auto drawn = [&](int64_t lo, int64_t hi) {       // even over the logarithm
        const double x = std::uniform_real_distribution<double>(0.0, 1.0)(rng);
        double v = (double)lo;
        while (v < (double)hi && v < (double)hi * 0.5) {
            if (std::uniform_real_distribution<double>(0.0, 1.0)(rng) < 0.12) break;
            v *= 2.0;
        }
        return std::min(hi, (int64_t)(v * (1.0 + x)));
    };
    long count[4] = {};
    size_t largest = 0;
    for (int n = 0; n < 2000000; ++n) {
        B = (int32_t)drawn(1, 65536);
        Hkv = (int32_t)drawn(1, 1024);
        Hq = Hkv * (int32_t)drawn(1, std::max<int64_t>(1, 1024 / Hkv));
        L = (int32_t)drawn(1, 1 << 20);
        if (n % 2) L = 1 + n % 16;
        most = 16 * drawn(1, 1 << 16);
        if (!allowed()) continue;
        const Plan p = plan(B, Hq, Hkv, L, most);
        ++count[p.way];
        hold(p.units == (int64_t)B * Hkv && p.rows == L * (Hq / Hkv), "sizes");
        hold(p.keys >= most && p.keys % 64 == 0 && p.keys < most + 64, "keys");
        hold((p.tile_rows == 16 || p.tile_rows == 64) && (int64_t)p.tiles * p.tile_rows >= p.rows &&
             (int64_t)(p.tiles - 1) * p.tile_rows < p.rows, "tiles");
        hold(p.splits >= 1 && p.splits <= 256 && (p.splits == 1 || p.way >= kParts), "parts");
        hold(p.units * p.tiles * p.splits < ((int64_t)1 << 24), "workgroups");
        const bool kept = p.way == kOneFew || p.way == kPartsFew;
        hold(!kept || (p.rows <= 16 && p.tile_rows == 16 && p.tiles == 1), "few rows");
        hold(kept || p.tile_rows == 64, "many rows");
        hold(p.way != kOneFew || p.rows * p.keys <= kLdsLogits, "logits in LDS");
        // the arrays lie behind one another within the bytes that the caller is asked for
        char* const base = reinterpret_cast<char*>((size_t)1 << 40);
        const Shape sh = shape(p, base);
        const auto at = [&](const void* q) { return (size_t)(static_cast<const char*>(q) - base); };
        const size_t rows = p.way >= kParts ? (size_t)(p.units * p.tiles * p.tile_rows) : 0;
        hold(at(sh.row_sum) == 0 && at(sh.row_max) == 8 * rows && at(sh.part_max) == 12 * rows, "sums");
        hold(at(sh.logits) == (12 + 4 * (size_t)p.splits) * rows && at(sh.logits) % 16 == 0, "maxima");
        const size_t end = at(sh.logits) + (p.way == kPartsFew ? 4 * (size_t)(p.units * p.rows * p.keys) : 0);
        hold(end == p.bytes(), "bytes");
        hold(at(sh.logits) <= 17000000 && end - at(sh.logits) <= (size_t)1 << 30, "a workspace of more than its limit");
        largest = std::max(largest, end);
    }
    printf("%ld %ld %ld %ld %zu\n", count[kOne], count[kOneFew], count[kParts], count[kPartsFew], largest);
}
