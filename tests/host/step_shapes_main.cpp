// How many threads the launches of xattn_prefill, xattn_rope_kvcache and xbeam_logprobs have at the ends of the ranges that their headers state: a
// launch has fewer than 2^32.  Prints "all scenarios ran" and exits with 0 if every check held.
#include <cstdint>
#include <cstdio>

#include "../../paper_2510_14686_amd/csrc/xattn_prefill_plan.h"
#include "../../paper_2510_14686_amd/csrc/xattn_rope.h"
#include "../../paper_2510_14686_amd/csrc/xbeam_logprobs.h"

using namespace xattn;

static int g_failures = 0;
static void check(bool ok, const char* what, long a, long b, long c, long d) {
    if (ok) return;
    std::fprintf(stderr, "%s: %ld %ld %ld %ld\n", what, a, b, c, d);
    ++g_failures;
}

int main() {
    const int64_t limit = (int64_t)1 << 32;
    const int totals[] = {1, 2, 1023, 1024, 4096, 1 << 20, (1 << 24) - 1, 1 << 24}, heads[] = {1, 2, 3, 8, 40, 64, 128, 513, 1024};
    for (int total : totals)
        for (int hq : heads) {
            if ((int64_t)total * hq > 1 << 30) continue;
            for (int hkv : heads) {
                for (int d = 16; d <= 256; d += 16) {
                    const int rows = rope_rows_per_workgroup(total, hq, hkv, d);
                    check(rows == 1 || rows == 2 || rows == 4, "rows per workgroup", total, hq, hkv, d);
                    check((int64_t)((total + rows - 1) / rows) * kRopeThreads < limit, "rotary positions", total, hq, hkv, d);
                }
                if (hq % hkv == 0)
                    for (int batch : {1, 64, 4096}) check(prefill_grid(total, batch, hq / hkv, hkv) * 256 < limit, "prompts", total, hq, hkv, batch);
            }
        }
    // What was chosen before the last row that a launch has threads for.
    check(rope_rows_per_workgroup((1 << 24) - 1, 64, 8, 128) == 1 && rope_rows_per_workgroup(1 << 24, 64, 8, 128) == 2, "the most rows", 0, 0, 0, 0);
    for (int rows : {1, 256, 1 << 22})
        for (int vocab : {1, 8192, 8193, 100003, 1 << 24}) {
            const LogprobsCut c = logprobs_cut(rows, vocab, vocab < 512 ? vocab : 512);
            const int waves = (int64_t)rows * c.parts <= kParts ? kMostWaves : kRowWaves;
            check((int64_t)rows * c.parts * waves * 64 < limit && (int64_t)rows * kRowWaves * 64 < limit, "logits", rows, vocab, c.parts, 0);
        }
    if (g_failures) return 1;
    std::puts("all scenarios ran");
    return 0;
}
