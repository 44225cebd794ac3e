// Internal interface between the host code of xattn_prefill and its kernels.
#ifndef XATTN_PREFILL_H_
#define XATTN_PREFILL_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "xattn_prefill_plan.h"

namespace xattn {

struct PrefillParams {
    const uint16_t* q;               // bf16 [total_q, n_q_heads, 128]
    const void* const* k_ptrs;       // device array[batch] of device pointers
    const void* const* v_ptrs;
    const int32_t* q_starts;         // device int32[batch + 1]
    const int32_t* kv_lens;          // device int32[batch]
    int batch, total_q, n_q_heads, n_kv_heads, group;
    float scale_log2;                // |scale| * log2(e), or 1 where the scale is 0
    uint32_t q_and, q_xor;           // applied to pairs of Q's values: a negative scale's sign, a zero scale
    uint16_t* out;                   // bf16 [total_q, n_q_heads, 128]
    float* lse;                      // fp32 [total_q, n_q_heads] or null
    int32_t* table;                  // kPrefillTableBytes: what the merge kernel has to put together
    float* part_ml;                  // fp32 [kPrefillSlots, slot_rows, 2]: reference maximum (log2 domain), sum
    float* part_o;                   // fp32 [kPrefillSlots, slot_rows, 128]
    int slot_rows;
    int exact;                       // weights enter the product with V with all their bits
};
constexpr size_t kPrefillTableBytes = 32 + 32 * (size_t)kPrefillShares;
hipError_t launch_prefill(const PrefillParams& prm, hipStream_t stream);

}  // namespace xattn
#endif
