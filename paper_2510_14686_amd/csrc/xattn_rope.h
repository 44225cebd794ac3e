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
hipError_t launch_rope(const RopeParams& prm, hipStream_t stream);

}  // namespace xattn
#endif
