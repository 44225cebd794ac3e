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

constexpr int kRowWaves = 8;                     // waves of a workgroup; kFewWaves where rows are short
constexpr int kFewWaves = 2;
// Where no compute unit has two workgroups and a part has more than kManyRounds rounds: 250 rows of 131072 without alternatives 17.8 -> 14.7 us,
// with 20 26.9 -> 24.6, fp32 with 400 47.3 -> 34.7; in shorter ones a longer end costs 2 us (200 rows of 50000 14.7 -> 16.2).
constexpr int kMostWaves = 16;
constexpr int kManyRounds = 10;
constexpr int kStep = 512;                       // values that a wave loads as one row of 8 (or two of 4) per lane
constexpr int kLoads = 2;                        // steps of a wave in a round
constexpr int kAtOnceSize = kRowWaves * kLoads * kStep;      // values that a workgroup's registers hold
constexpr int kParts = 256;                      // workgroups that rows are cut for
constexpr int kFewRounds = 6;                    // of a row that is not cut
constexpr int kMostMerged = 8192;                // candidates that the merge of a row's parts holds

// How a call's rows are cut.
struct LogprobsCut {
    int parts, part_size;            // parts of a row, and their logits (a multiple of kStep but for the last)
    size_t workspace;                // bytes; 0 with one part
};
// A round is kAtOnceSize values and takes a workgroup about 1 us, putting parts together 6 to 8 us (a second launch): rows of more
// than kFewRounds rounds are cut where they are few.  1 / 128 rows of 40000, 20 alternatives 12.3 / 13.8 us whole (of kFewRounds = 3, cut,
// 12.0 / 17.3); 1 / 128 of 60000 12.4 / 17.5 cut (15.3 / 16.3 whole).  kParts 512: 64 of 131072 19.6 -> 25.0.
inline LogprobsCut logprobs_cut(int rows, int vocab, int top_k) {
    const int at_once = (vocab + kAtOnceSize - 1) / kAtOnceSize;
    int parts = kParts / rows < at_once ? kParts / rows : at_once;
    if (top_k > 0 && parts > kMostMerged / top_k) parts = kMostMerged / top_k;
    if (at_once <= kFewRounds) parts = 1;
    if (parts <= 1) return LogprobsCut{1, vocab, 0};
    const int steps = (vocab + kStep - 1) / kStep, size = (steps + parts - 1) / parts * kStep;
    parts = (vocab + size - 1) / size;
    return LogprobsCut{parts, size, parts > 1 ? (size_t)rows * parts * (16 + 8 * (size_t)top_k) : 0};
}
hipError_t launch_logprobs(const LogprobsParams& prm, const LogprobsCut& cut, hipStream_t stream);

}  // namespace xattn
#endif
