// Internal interface between the host code of xbeam_logprobs and its kernels.
#ifndef XBEAM_LOGPROBS_H_
#define XBEAM_LOGPROBS_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace xattn {

constexpr int kMaxTopK = 512;

struct LogprobsParams {
    const void* logits;
    int dtype;                       // XBEAM_BF16, XBEAM_FP16, XBEAM_FP32
    int64_t row_stride;              // in values
    int rows, vocab;
    float scale_log2;                // scale * log2(e)
    float scale;
    const int32_t* tokens;           // or null, with token_lp
    int top_k;
    float* token_lp;
    float* top_lp;
    int32_t* top_tok;
    float* lse;
    float* entropy;
    char* workspace;                 // of several parts per row
};
// How a call's rows are cut.
struct LogprobsCut {
    int parts, part_size;            // parts of a row, and their logits (a multiple of 512 but for the last)
    size_t workspace;                // bytes; 0 with one part
};
LogprobsCut logprobs_cut(int rows, int vocab, int top_k);
hipError_t launch_logprobs(const LogprobsParams& prm, const LogprobsCut& cut, hipStream_t stream);

}  // namespace xattn
#endif
