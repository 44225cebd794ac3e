// How xattn_prefill's work is cut (csrc/xattn_prefill_plan.h) on random batches: the bounds of grid and workspace hold, and the
// parts of a tile cover its keys once.  Prints "all batches ran" and exits with 0 if every check held.
#include <cstdio>
#include <random>
#include <vector>

#include "../../paper_2510_14686_amd/csrc/xattn_prefill_plan.h"

using namespace xattn;

static int g_failures = 0;
#define CHECK(cond)                                                                      \
    do {                                                                                 \
        if (!(cond)) {                                                                   \
            if (++g_failures < 20) std::fprintf(stderr, "line %d: %s\n", __LINE__, #cond); \
        }                                                                                \
    } while (0)

static std::mt19937_64 g_rng(7);
static int draw(int lo, int hi) { return lo + (int)(g_rng() % (uint64_t)(hi - lo + 1)); }
static int draw_log(int hi) { return draw(0, hi >> draw(0, 20)); }

static void one_batch(int batch, int group, int n_kv_heads, int max_q, int max_kv) {
    std::vector<int> starts{0}, kv;
    for (int b = 0; b < batch; ++b) {
        starts.push_back(starts.back() + draw_log(max_q));
        kv.push_back(draw(0, 3) ? starts[b + 1] - starts[b] + draw_log(max_kv) : draw_log(max_kv) - 2);
    }
    const int total_q = starts.back() + draw(0, 3) + (starts.back() == 0);
    std::vector<PrefillSeq> seqs;
    float cost = 0.0f;
    for (int b = 0; b < batch; ++b) {
        seqs.push_back(prefill_seq(starts[b], starts[b + 1], kv[b], total_q, group));
        cost += prefill_cost(seqs.back());
    }
    const int share = prefill_share(cost * (float)n_kv_heads);
    long parts_in_all = 0, slots = 0, split_tiles = 0, tiles = 0;
    for (const PrefillSeq& s : seqs) {
        const int parts = prefill_parts(s.blocks, share), size = prefill_part_blocks(s.blocks, parts);
        CHECK(parts >= 1 && (s.blocks == 0 || (size >= 1 && (long)size * parts >= s.blocks && size <= share)));
        tiles += s.tiles;
        parts_in_all += (long)s.tiles * parts;
        if (parts > 1) {
            slots += (long)s.tiles * parts;
            split_tiles += s.tiles;
        }
        CHECK((long)s.tiles * kPrefillRows >= (long)s.q * group && (long)(s.tiles - 1) * kPrefillRows < (long)s.q * group);
        for (int probe = 0; probe < 4 && s.tiles > 0; ++probe) {
            const int tile = probe == 0 ? s.tiles - 1 : draw(0, s.tiles - 1);
            const int blocks = prefill_tile_blocks(s, tile, group);
            CHECK(blocks >= 0 && blocks <= s.blocks);
            long covered = 0;
            for (int p = 0; p < parts; ++p) {
                const int from = p * size, to = from + size < blocks ? from + size : blocks;
                covered += to > from ? to - from : 0;
            }
            CHECK(covered == blocks);
            // the tile's last row sees no key behind its blocks, and one in the last of them
            const long last = (long)(tile + 1) * kPrefillRows < (long)s.q * group ? (long)(tile + 1) * kPrefillRows - 1 : (long)s.q * group - 1;
            const int seen = prefill_visible(s, (int)(last / group));
            CHECK(seen <= blocks * kPrefillKeys && seen > (blocks - 1) * kPrefillKeys);
        }
    }
    CHECK(tiles <= prefill_tiles_bound(total_q, batch, group));
    CHECK(parts_in_all * n_kv_heads <= prefill_grid(total_q, batch, group, n_kv_heads));
    CHECK(slots * n_kv_heads <= kPrefillSlots);
    CHECK(split_tiles * n_kv_heads <= kPrefillShares);
    CHECK(prefill_slot_rows(total_q, group) <= kPrefillRows);
}

int main() {
    for (int i = 0; i < 4000; ++i)
        one_batch(i % 7 == 0 ? draw(500, 4096) : draw(1, 100), draw(0, 3) ? draw(1, 16) : draw(1, 1024), draw(1, 16), draw(0, 1) ? 40000 : 50,
                  draw(0, 1) ? 1000000 : 2000);
    one_batch(1, 1024, 1, 1 << 14, 1 << 24);
    one_batch(4096, 1, 1024, 200, 1 << 22);
    if (g_failures) return 1;
    std::puts("all batches ran");
    return 0;
}
