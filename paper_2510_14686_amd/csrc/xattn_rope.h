// Internal interface between the host code of xattn_rope_kvcache and its kernel.
#ifndef XATTN_ROPE_H_
#define XATTN_ROPE_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace xattn {

constexpr int kRopeMaxHeadDim = 256;
constexpr int kRopeMaxAxes = 4;

struct RopeParams {
    const uint16_t* q;               // bf16, rows of n_q_heads * head_dim values, q_stride apart
    const uint16_t* k;
    const uint16_t* v;
    int64_t q_stride, k_stride, v_stride;
    const int32_t* pos;              // [n_axes, total_q]
    const float* inv_freq;           // [frequencies]
    void* const* k_ptrs;
    void* const* v_ptrs;
    const int32_t* q_starts;         // [batch + 1]
    const int32_t* kv_lens;          // [batch]
    uint16_t* q_out;                 // [total_q, n_q_heads, head_dim]
    int batch, total_q, n_q_heads, n_kv_heads, head_dim;
    int frequencies;                 // half the rotated values of a head
    int pairs;                       // frequency i turns values 2 i and 2 i + 1, not i and frequencies + i
    uint32_t axis_of[kRopeMaxHeadDim / 2 / 16];      // two bits per frequency
};
constexpr int kRopeThreads = 256;

// Rows per workgroup.  A workgroup of few short rows has threads without work, one of more rows than its threads need moves them in more
// turns of its loop.  Of 1 / 2 / 4 rows each, in us: 256 rows of 40 / 8 heads 5.8 / 6.5 / 8.4, 2000 rows 13.1 / 12.2 / 13.2, 16384 rows
// 86.4 / 89.0 / 95.1; 16384 of 64 / 8 heads 120 / 127 / 135, of 16 / 8 47.2 / 41.7 / 43.5; 65536 of 8 / 1 139 / 90 / 69.
// A launch has fewer than 2^32 threads, so 2^24 rows do not get a workgroup each.
inline int rope_rows_per_workgroup(int total_q, int n_q_heads, int n_kv_heads, int head_dim) {
    const int items = (n_q_heads + 2 * n_kv_heads) * (head_dim / 16);      // of a row
    if (total_q < 1024) return 1;
    if (items > 2 * kRopeThreads) return (int64_t)total_q * kRopeThreads < (int64_t)1 << 32 ? 1 : 2;
    return items > kRopeThreads / 2 ? 2 : 4;
}
hipError_t launch_rope(const RopeParams& prm, hipStream_t stream);

}  // namespace xattn
#endif
