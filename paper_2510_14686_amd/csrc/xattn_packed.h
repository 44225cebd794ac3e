// Packed batches on the device: which sequence a row belongs to.
#ifndef XATTN_PACKED_H_
#define XATTN_PACKED_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace xattn {
namespace {

// The sequence whose rows [q_starts[b], q_starts[b + 1]) hold `row`, and where its new rows begin and end; -1 without one.
// Wave-uniform: each lane looks at the bounds of batch / 64 sequences, then of one.
__device__ __forceinline__ int find_sequence(const int32_t* __restrict__ q_starts, int batch, int row, int lane, int& start, int& end) {
    const int per = (batch + 63) / 64;
    int first = lane * per, last = first + per < batch ? first + per : batch;
    int s = 0, e = 0;
    if (first < batch) {
        s = q_starts[first];
        e = q_starts[last];
    }
    unsigned long long hit = __ballot(first < batch && s <= row && row < e);
    if (hit == 0) return -1;
    int at = __builtin_ctzll(hit);
    if (per > 1) {
        first = at * per + lane;
        const bool in = lane < per && first < batch;
        s = in ? q_starts[first] : 0;
        e = in ? q_starts[first + 1] : 0;
        hit = __ballot(in && s <= row && row < e);
        if (hit == 0) return -1;      // q_starts does not ascend
        const int l = __builtin_ctzll(hit);
        start = __builtin_amdgcn_readlane(s, l);
        end = __builtin_amdgcn_readlane(e, l);
        return at * per + l;
    }
    start = __builtin_amdgcn_readlane(s, at);
    end = __builtin_amdgcn_readlane(e, at);
    return at;
}

}  // namespace
}  // namespace xattn
#endif
