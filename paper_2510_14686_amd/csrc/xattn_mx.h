// The cache of 4 bits a value, and the internal interface between the host code of its operators and their kernels.
//
// A head's row of 128 values is four blocks of 32; a block has a scale 2^e, one byte e + 127, and its values are 4-bit codes: a sign and one
// of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale (element format e2m1 and scale format e8m0 of the OCP Microscaling Formats, v1.0).
// Rows lie in tiles of 64 tokens of one KV head, kMxTileBytes long: 4 x 1024 bytes of codes, 16 tokens each, then 256 bytes of scales.
// A range's tiles lie one behind the other, those of all heads of the same tokens together.  Inside, bytes stand as
// the lanes of xattn_decode_mx's waves take them, 16 (codes) or 4 and 16 (scales) at a time, so that every load is one contiguous run:
//   K codes    token 16 s + m, block c:                1024 s + 256 c + 16 m, 16 bytes
//   V codes    token 16 s + 4 g + r, values 8 m .. + 7:  1024 s + 256 g + 16 m + 4 r, 4 bytes
//   K scales   4096 + 4 (16 c + m) + s
//   V scales   4096 + 16 (4 g + c) + 4 s + r
// The lower half of a byte is the value that comes first.
#ifndef XATTN_MX_H_
#define XATTN_MX_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "xattn_kernels.h"
#include "xattn_rope.h"

namespace xattn {

constexpr int kMxTileTokens = 64;
constexpr int kMxCodeBytes = 4096;
constexpr int kMxTileBytes = kMxCodeBytes + 256;
// A block's scale exponent: the least e with all values within 7 * 2^e, so that none is further from its code than half of the
// widest step, 4 to 6.  (Root mean square error of N(0, 1) with 6 / 7 / 8 in 7's place: 0.1153 / 0.1118 / 0.1150.)  From -125 on the least
// code, half of the scale, is a normal number of bf16 and fp32.  At 126 only codes up to 3 are: 4 and 6 are read as infinities.
constexpr int kMxLeastExp = -125, kMxMostExp = 126;
constexpr int kMxNanScale = 255;

// Positions of the token stream (see xattn_plan.h) that a tile takes, whose rounding of piece bounds then is to whole tiles.
constexpr int kMxPositions = kPlanRound;
XATTN_HD int mx_positions(int len) { return len > 0 ? (int)(((unsigned)len + (kMxTileTokens - 1)) / kMxTileTokens) * kMxPositions : 0; }
// Positions of each of `parts` waves of a piece of `len` positions, all but the last one's: whole tiles.
XATTN_HD int mx_part_positions(int len, int parts) { return ((len + parts - 1) / parts + kMxPositions - 1) / kMxPositions * kMxPositions; }

// How a call's work is cut: `waves` waves of a workgroup share a piece, of which there are `pieces`.
struct MxCut {
    int rows, waves, pieces;
};
constexpr int kMxComputeUnits = 256;
// A compute unit holds twelve waves with 16 query rows each, or eight with 32 (registers and LDS).  One workgroup of all of them leaves the fewest
// partial results, and where that many workgroups fill the chip (8 KV heads: 32 pieces) is faster than several small ones: 128 sequences of 1028 to
// 8196 tokens, 16 rows of 8 KV heads 107.4 us, 116.3 in workgroups of four.  Pieces come in multiples of eight, though, and with many KV heads, or a number of them that
// does not go into 256, a quarter of the chip or more may have nothing to do in the last round: small ones then, 16 sequences of 501 to
// 4001 tokens of 40 KV heads 48.4 -> 37.5.
inline MxCut mx_cut(int q_len, int n_q_heads, int n_kv_heads) {
    const int rows_total = n_q_heads / n_kv_heads * q_len, rows = rows_total <= 16 ? 16 : 32;
    const int most = rows == 16 ? 12 : 8, on_a_piece = (rows_total + rows - 1) / rows * n_kv_heads;
    auto used = [&](int at_once, int pieces) {      // per mille of the rounds' places
        const int n = pieces * on_a_piece;
        return (int)(1000L * n / ((n + at_once - 1) / at_once * at_once));
    };
    const int small = kMxComputeUnits * most / 4, pieces = pieces_of(kMxComputeUnits, on_a_piece), more = pieces_of(small, on_a_piece);
    if (used(kMxComputeUnits, pieces) < 800 && used(small, more) > used(kMxComputeUnits, pieces)) return MxCut{rows, 4, more};
    return MxCut{rows, most, pieces};
}

// Decode attention; prm.share and parts are not used.
hipError_t launch_decode_mx(const DecodeParams& prm, const MxCut& cut, hipStream_t stream);

// Rotation and append: prm.k_ptrs and v_ptrs are ranges of tiles, prm.head_dim is 128.
hipError_t launch_rope_mx(const RopeParams& prm, hipStream_t stream);

struct ReadMxParams {
    const void* const* k_ptrs;
    const void* const* v_ptrs;
    const int32_t* q_starts;         // [batch + 1]
    const int32_t* kv_lens;          // [batch]
    uint16_t* k_out;                 // bf16 [total_q, n_kv_heads, 128]
    uint16_t* v_out;
    int batch, total_q, n_kv_heads;
};
hipError_t launch_read_mx(const ReadMxParams& prm, hipStream_t stream);

}  // namespace xattn
#endif
