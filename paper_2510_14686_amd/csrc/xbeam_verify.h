// Internal interface between the host code of xbeam_verify and its kernels.
#ifndef XBEAM_VERIFY_H_
#define XBEAM_VERIFY_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace xattn {

constexpr int kVerifyThreads = 256;
constexpr int kVerifyStep = 8 * kVerifyThreads;      // logits that a workgroup takes at a time
constexpr int kVerifyMostParts = 64;                 // of a row: a wave puts them together, a lane each
constexpr int kVerifySums = 5;                       // that a row's parts give

struct VerifyParams {
    const void* target;              // [batch * q_len, >= vocab], rows target_stride values apart
    const void* draft;               // [batch * (q_len - 1), >= vocab], or null: drafts are certain
    int64_t target_stride, draft_stride;
    int dtype, vocab;
    float scale, draft_scale;
    const int32_t* draft_tokens;     // [batch, q_len - 1]
    const int32_t* n_drafts;         // [batch], or null: q_len - 1
    const float* uniforms;           // [batch, q_len]; null with greedy
    int batch, q_len, greedy;
    int32_t* tokens;                 // [batch, q_len]
    int32_t* accepted;               // [batch]
    float* token_lp;                 // [batch, q_len] or null
    // workspace
    float2* stats;                   // [rows, parts]: largest logit, sum of exponentials over it
    uint64_t* best;                  // [target rows, parts], greedy
    double* sums;                    // [kVerifySums, batch, cut.parts]: see verify_weigh_kernel
    void* decisions;                 // [batch]
};

// How rows are cut: parts, and logits of each (a multiple of kVerifyStep but for the last).
struct VerifyCut {
    int parts, size;
};
// `rows` rows in about `workgroups` parts.
inline VerifyCut verify_cut(long rows, int vocab, int workgroups) {
    const int steps = (vocab + kVerifyStep - 1) / kVerifyStep;
    long parts = (workgroups + rows - 1) / rows;
    parts = parts < 1 ? 1 : parts > kVerifyMostParts ? kVerifyMostParts : parts;
    parts = parts > steps ? steps : parts;
    const int size = (int)((steps + parts - 1) / parts) * kVerifyStep;
    return VerifyCut{(vocab + size - 1) / size, size};
}
// Workgroups of the two passes, about: read's many are its loads in flight.  (Readers 2048 / 4096 / 8192: 64 sequences of five rows of 131072 logits 67.9 / 66.0 / 65.4 us,
// 48 of four of 100003 32.1 / 30.1 / 29.5.  Pickers 1024 / 2048 / 4096 / 8192: 76.1 / 68.1 / 65.4 / 65.4, 128 of four of 50000 62.5 / 54.1 / 48.9 / 48.8.)
constexpr int kVerifyReaders = 8192, kVerifyPickers = 4096;
struct VerifyLayout {
    VerifyCut read, pick;
    size_t best_off, sums_off, decisions_off, total;
};
inline VerifyLayout verify_layout(int batch, int q_len, int vocab, bool with_draft) {
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const long rows = (long)batch * (2 * q_len - 1);
    VerifyLayout w;
    w.read = verify_cut(with_draft ? rows : (long)batch * q_len, vocab, kVerifyReaders);
    w.pick = verify_cut(batch, vocab, kVerifyPickers);
    w.best_off = up((size_t)rows * w.read.parts * 8);
    w.sums_off = w.best_off + up((size_t)batch * q_len * w.read.parts * 8);
    w.decisions_off = w.sums_off + up((size_t)kVerifySums * batch * w.pick.parts * 8);
    w.total = w.decisions_off + up((size_t)batch * 64);
    return w;
}
hipError_t launch_verify(const VerifyParams& prm, const VerifyLayout& w, hipStream_t stream);

}  // namespace xattn
#endif
