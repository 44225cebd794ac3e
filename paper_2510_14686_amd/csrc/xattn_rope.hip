// Rotary positions with one to four axes on the new rows of a packed batch, with the append of the turned K and of V to the
// sequences' ranges (xattn_rope_kvcache).
//
//   (x, y) -> (x cos a - y sin a, y cos a + x sin a),  a = pos[axis of i][row] * inv_freq[i],  for every pair i of every head
//
// Bound by memory: a row is read once and written once.  Two prompts of 4096 to 8191, 32 / 8 heads, 299 MB: 51 us, 5.9 TB/s, where a copy
// of 1 GiB makes 5.2; 256 sequences' single tokens, 40 / 8 heads: 6 us, of which the angles and two dependent loads are most.  (Loads
// and stores past the caches: 2048 tokens 11.7 -> 14 us; what is written is read next.)
//   A workgroup takes kTokens rows: a wave per row finds the row's sequence
// and works the angles out, into LDS, once for all heads; then all threads move 32 bytes at a time.
// Angles are reduced to a fraction of a turn in double: a far position times a frequency has more digits than a float (position
// 4000000 would be off by 0.2 rad).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "xattn_device.h"
#include "xattn_launch.h"
#include "xattn_packed.h"
#include "xattn_rope.h"

namespace xattn {
namespace {

// kLanes: pieces of 16 values per head where known, else 0.
template <int kTokens, int kLanes>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeParams prm) {
    __shared__ float cosines[kTokens][kRopeMaxHeadDim / 2], sines[kTokens][kRopeMaxHeadDim / 2];
    __shared__ uint16_t* rows[kTokens][2];      // where K and V of the row go, or null
    __shared__ int known[kTokens];              // whether a sequence has it
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
    const int token0 = blockIdx.x * kTokens;
    const int lanes = kLanes ? kLanes : prm.head_dim / 16, slots = prm.n_q_heads + 2 * prm.n_kv_heads;
    const int items = slots * lanes * kTokens, turned = prm.frequencies / 8;
    // An item: 16 values of a head of a row, in two pieces.
    struct Item {
        int tk, head, c, at0, at1;
        bool is_q, is_k, turn;
        u32x4_t x, y;
    };
    auto fetch = [&](int item) {
        Item r;
        r.c = (int)((unsigned)item % (unsigned)lanes);
        const int slot = (int)((unsigned)item / (unsigned)lanes % (unsigned)slots);
        r.tk = (int)((unsigned)item / (unsigned)lanes / (unsigned)slots);
        r.is_q = slot < prm.n_q_heads;
        r.is_k = !r.is_q && slot < prm.n_q_heads + prm.n_kv_heads;
        r.head = r.is_q ? slot : r.is_k ? slot - prm.n_q_heads : slot - prm.n_q_heads - prm.n_kv_heads;
        r.turn = r.c < turned && (r.is_q || r.is_k);
        const bool apart = r.turn && !prm.pairs;
        r.at0 = apart ? 8 * r.c : 16 * r.c;
        r.at1 = apart ? prm.frequencies + 8 * r.c : 16 * r.c + 8;
        const int64_t row = token0 + r.tk < prm.total_q ? token0 + r.tk : prm.total_q - 1;
        const uint16_t* const from =
            (r.is_q ? prm.q + row * prm.q_stride : r.is_k ? prm.k + row * prm.k_stride : prm.v + row * prm.v_stride) + r.head * prm.head_dim;
        r.x = *reinterpret_cast<const u32x4_t*>(from + r.at0);
        r.y = *reinterpret_cast<const u32x4_t*>(from + r.at1);
        return r;
    };
    // The first one is on its way while the rows' sequences are looked for.
    Item next = fetch((int)threadIdx.x < items ? (int)threadIdx.x : 0);
    if (wave < kTokens) {
        const int row = token0 + wave;
        int start = 0, end = 0;
        const int b = row < prm.total_q ? find_sequence(prm.q_starts, prm.batch, row, lane, start, end) : -1;
        if (b >= 0) {
            const int len = prm.kv_lens[b], at = len >= end - row ? len - (end - row) : -1;
            if (lane < 2) {
                void* const base = lane == 0 ? prm.k_ptrs[b] : prm.v_ptrs[b];
                rows[wave][lane] = at >= 0 ? static_cast<uint16_t*>(base) + (int64_t)at * prm.n_kv_heads * prm.head_dim : nullptr;
            }
            for (int i = lane; i < prm.frequencies; i += 64) {
                const int axis = (prm.axis_of[i >> 4] >> (2 * (i & 15))) & 3;
                const double turns = (double)prm.pos[(int64_t)axis * prm.total_q + row] * (double)prm.inv_freq[i] * 0.15915494309189533577;
                float sine, cosine;
                sincospif(2.0f * (float)(turns - rint(turns)), &sine, &cosine);
                cosines[wave][i] = cosine;
                sines[wave][i] = sine;
            }
        }
        if (lane == 0) known[wave] = b >= 0;
    }
    __syncthreads();

    for (int item = threadIdx.x; item < items; item += kRopeThreads) {
        Item it = next;
        if (item + kRopeThreads < items) next = fetch(item + kRopeThreads);
        if (!known[it.tk]) continue;
        uint16_t* to = it.is_q ? prm.q_out + (int64_t)(token0 + it.tk) * prm.n_q_heads * prm.head_dim : rows[it.tk][it.is_k ? 0 : 1];
        if (to == nullptr) continue;
        to += it.head * prm.head_dim;
        u32x4_t &x = it.x, &y = it.y;
        if (it.turn) {
            float co[8], si[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                co[i] = cosines[it.tk][8 * it.c + i];
                si[i] = sines[it.tk][8 * it.c + i];
            }
            if (prm.pairs) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = bf16_lo(x[i]), b = bf16_hi(x[i]), d = bf16_lo(y[i]), e = bf16_hi(y[i]);
                    x[i] = cvt_bf16(a * co[i] - b * si[i], b * co[i] + a * si[i]);
                    y[i] = cvt_bf16(d * co[4 + i] - e * si[4 + i], e * co[4 + i] + d * si[4 + i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = bf16_lo(x[i]), b = bf16_hi(x[i]), d = bf16_lo(y[i]), e = bf16_hi(y[i]);
                    x[i] = cvt_bf16(a * co[2 * i] - d * si[2 * i], b * co[2 * i + 1] - e * si[2 * i + 1]);
                    y[i] = cvt_bf16(d * co[2 * i] + a * si[2 * i], e * co[2 * i + 1] + b * si[2 * i + 1]);
                }
            }
        }
        *reinterpret_cast<u32x4_t*>(to + it.at0) = x;
        *reinterpret_cast<u32x4_t*>(to + it.at1) = y;
    }
}

}  // namespace

hipError_t launch_rope(const RopeParams& prm, hipStream_t stream) {
    auto with = [&](auto tokens) {
        constexpr int kTokens = decltype(tokens)::value;
        const dim3 grid((unsigned)((prm.total_q + kTokens - 1) / kTokens));
        return prm.head_dim == 128 ? launch(rope_kernel<kTokens, 8>, grid, kRopeThreads, stream, prm)
                                   : launch(rope_kernel<kTokens, 0>, grid, kRopeThreads, stream, prm);
    };
    switch (rope_rows_per_workgroup(prm.total_q, prm.n_q_heads, prm.n_kv_heads, prm.head_dim)) {
        case 1: return with(std::integral_constant<int, 1>());
        case 2: return with(std::integral_constant<int, 2>());
        default: return with(std::integral_constant<int, 4>());
    }
}

}  // namespace xattn
