// How xattn_prefill's work is cut (paper section 4.4.3, "Layer 3"), as plain integer code for the device and the host.
//
// The query rows of a sequence and a KV head, new token x query head of the group, are cut into tiles of kPrefillRows; a
// tile's keys, in blocks of kPrefillKeys, into one or more parts, each a workgroup's work.  The host knows neither lengths
// nor which parts there are: every workgroup finds its own from q_starts and kv_lens.
//
// A part holds at most `share` blocks, 1 / kPrefillShares of the batch's sum of blocks over tiles (a causal prompt needs
// half of that sum, so one that fills the chip by itself is not split).  With cost = the sum over tiles of their sequence's blocks,
// and share > cost / kPrefillShares:
//   parts in all      <= sum (blocks / share + 1)       < tiles + kPrefillShares
//   tiles of sequences in several parts: blocks > share, so fewer than kPrefillShares
//   their parts       <= sum 2 * blocks / share         < 2 * kPrefillShares = kPrefillSlots
// which bounds the grid and the workspace whatever the lengths are.
#ifndef XATTN_PREFILL_PLAN_H_
#define XATTN_PREFILL_PLAN_H_

#include "xattn_plan.h"

namespace xattn {

constexpr int kPrefillRows = 128;
constexpr int kPrefillKeys = 64;
// Two workgroups per compute unit.  1024: one prompt of 2048 (32 / 8 heads) 59 -> 95 us, 64 sequences of 4096 and one new token 200 -> 226.
constexpr int kPrefillShares = 512;
constexpr int kPrefillSlots = 2 * kPrefillShares;
// Shorter parts cost more to put together than they save.  With 4 / 8 / 16: one prompt of 512 (32 / 8 heads) 24.6 / 19.3 / 19.5 us, of 1024
// (8 / 2) 23.9 / 25.3 / 30.4, 20 new tokens behind 30000 (8 / 1) 21.9 / 25.5 / 36.2.
constexpr int kPrefillMinBlocks = 8;

// New tokens [first, first + q) of the packed rows, clamped to those that there are.
struct PrefillSeq {
    int first, q, kv;
    int tiles, blocks;
};
XATTN_HD int prefill_clamp(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }
XATTN_HD PrefillSeq prefill_seq(int start, int end, int kv_len, int total_q, int group) {
    PrefillSeq s;
    s.first = prefill_clamp(start, 0, total_q);
    s.q = prefill_clamp(end, s.first, total_q) - s.first;
    s.kv = clamp_len(kv_len);
    s.tiles = (int)(((unsigned)s.q * (unsigned)group + (kPrefillRows - 1)) / kPrefillRows);
    s.blocks = (int)(((unsigned)s.kv + (kPrefillKeys - 1)) / kPrefillKeys);
    return s;
}
XATTN_HD float prefill_cost(const PrefillSeq& s) { return (float)s.tiles * (float)s.blocks; }
// Blocks of a part at most; `cost`: sum of prefill_cost over the sequences, times KV heads.  A float sum of up to 4096 terms in
// any order is within 2^-11 of the sum, hence the 1.001.
XATTN_HD int prefill_share(float cost) {
    const float share = cost * (1.001f / kPrefillShares);
    const int blocks = share < 1e9f ? (int)share + 1 : 1000000000;
    return blocks < kPrefillMinBlocks ? kPrefillMinBlocks : blocks;
}
XATTN_HD int prefill_parts(int blocks, int share) { return blocks <= share ? 1 : (int)((unsigned)(blocks + share - 1) / (unsigned)share); }
XATTN_HD int prefill_part_blocks(int blocks, int parts) { return (int)((unsigned)(blocks + parts - 1) / (unsigned)parts); }
// Keys that the new token t sees.
XATTN_HD int prefill_visible(const PrefillSeq& s, int t) { return prefill_clamp(s.kv - s.q + t + 1, 0, s.kv); }
XATTN_HD int prefill_tile_blocks(const PrefillSeq& s, int tile, int group) {
    const unsigned last = (unsigned)(tile + 1) * kPrefillRows - 1;
    const int t = (int)(last / (unsigned)group);
    return (prefill_visible(s, t < s.q ? t : s.q - 1) + kPrefillKeys - 1) / kPrefillKeys;
}
// Upper bounds from what the host knows.
inline long prefill_tiles_bound(long total_q, long batch, long group) {
    return (total_q * group + batch * (kPrefillRows - 1)) / kPrefillRows;
}
inline long prefill_grid(long total_q, long batch, long group, long n_kv_heads) {
    return prefill_tiles_bound(total_q, batch, group) * n_kv_heads + kPrefillShares;
}
// Rows that a tile has at most.
inline int prefill_slot_rows(long total_q, long group) { return total_q * group < kPrefillRows ? (int)(total_q * group) : kPrefillRows; }

}  // namespace xattn
#endif
