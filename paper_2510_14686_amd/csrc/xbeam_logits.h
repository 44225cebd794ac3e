// Rows of logits as the kernels read them: 16 bytes at a time, from any address that is aligned to the type.
#ifndef XBEAM_LOGITS_H_
#define XBEAM_LOGITS_H_

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "xattn_device.h"

namespace xattn {
namespace {

struct Bf16 {
    uint16_t bits;
};
__device__ __forceinline__ float to_float(Bf16 x) { return __uint_as_float((uint32_t)x.bits << 16); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(float x) { return x; }

// Sixteen bytes of a row, which may begin anywhere.
typedef uint32_t words_at_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t words_at_4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T> struct Chunk {
    static constexpr int kCount = 16 / (int)sizeof(T);
    u32x4_t x;
    using words = typename std::conditional<sizeof(T) == 4, words_at_4, words_at_2>::type;
    __device__ __forceinline__ void load(const T* p) { x = __builtin_nontemporal_load(reinterpret_cast<const words*>(p)); }
    // Of a row that is read again.
    __device__ __forceinline__ void load_kept(const T* p) { x = *reinterpret_cast<const words*>(p); }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(x[i]);
        else if constexpr (std::is_same<T, Bf16>::value) return i & 1 ? bf16_hi(x[i >> 1]) : bf16_lo(x[i >> 1]);
        else return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? x[i >> 1] >> 16 : x[i >> 1]));
    }
};

}  // namespace
}  // namespace xattn
#endif
