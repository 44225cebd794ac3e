// C-ABI entry points around decode attention: rotary positions with append, prompt attention, log-probabilities.  Argument
// checks, workspaces, launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/xattn.h"
#include "../../include/xbeam.h"
#include "xattn_hip_error.h"
#include "xattn_host.h"
#include "xattn_kernels.h"
#include "xattn_prefill.h"
#include "xattn_rope.h"
#include "xbeam_logprobs.h"

namespace xattn {

namespace {

constexpr int kMaxBatch = 4096;
constexpr int kMaxTotalQ = 1 << 24;
constexpr int kMaxRowsOfHeads = 1 << 30;      // total_q * n_q_heads
constexpr int kMaxHeads = 1024;
constexpr int kMaxRows = 1 << 22;             // of logits: a launch has fewer than 2^32 threads, 512 of them per row

bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

int check_prefill(const char* who, int batch, int total_q, int n_q_heads, int n_kv_heads, int head_dim) {
    const int st = check_packed_batch(who, batch, total_q, n_q_heads, n_kv_heads, head_dim);
    if (st != XATTN_OK) return st;
    if (n_q_heads % n_kv_heads != 0)
        return fail(XATTN_EUNSUPPORTED, "%s: n_q_heads (%d) is not a multiple of n_kv_heads (%d)", who, n_q_heads, n_kv_heads);
    if (head_dim != kHeadDim) return fail(XATTN_EUNSUPPORTED, "%s: head_dim %d: only 128 is supported", who, head_dim);
    return XATTN_OK;
}

struct PrefillLayout {
    int slot_rows;
    size_t ml_off, o_off, total;
};
PrefillLayout prefill_layout(int total_q, int group) {
    PrefillLayout w;
    w.slot_rows = prefill_slot_rows(total_q, group);
    const size_t rows = (size_t)kPrefillSlots * w.slot_rows;
    w.ml_off = align_up(kPrefillTableBytes, 256);
    w.o_off = w.ml_off + align_up(rows * 2 * sizeof(float), 256);
    w.total = w.o_off + rows * kHeadDim * sizeof(float);
    return w;
}

int check_logprobs(const char* who, int rows, int vocab, int top_k) {
    if (rows < 1 || vocab < 1) return fail(XATTN_EINVAL, "%s: rows and vocab must be positive", who);
    if (top_k < 0 || top_k > vocab) return fail(XATTN_EINVAL, "%s: top_k %d is not in [0, vocab]", who, top_k);
    if (top_k > kMaxTopK) return fail(XATTN_EUNSUPPORTED, "%s: top_k %d exceeds %d", who, top_k, kMaxTopK);
    if (vocab > 1 << 24) return fail(XATTN_EUNSUPPORTED, "%s: vocab %d exceeds %d", who, vocab, 1 << 24);
    if (rows > kMaxRows) return fail(XATTN_EUNSUPPORTED, "%s: %d rows exceed %d", who, rows, kMaxRows);
    return XATTN_OK;
}

}  // namespace

int check_packed_batch(const char* who, int batch, int total_q, int n_q_heads, int n_kv_heads, int head_dim) {
    if (batch < 1 || total_q < 1 || n_q_heads < 1 || n_kv_heads < 1 || head_dim < 1)
        return fail(XATTN_EINVAL, "%s: batch, total_q, n_q_heads, n_kv_heads and head_dim must be positive", who);
    if (batch > kMaxBatch) return fail(XATTN_EUNSUPPORTED, "%s: batch %d exceeds %d", who, batch, kMaxBatch);
    if (total_q > kMaxTotalQ) return fail(XATTN_EUNSUPPORTED, "%s: total_q %d exceeds %d", who, total_q, kMaxTotalQ);
    if (n_q_heads > kMaxHeads || n_kv_heads > kMaxHeads)
        return fail(XATTN_EUNSUPPORTED, "%s: %d query heads, %d KV heads: more than %d", who, n_q_heads, n_kv_heads, kMaxHeads);
    if ((long)total_q * n_q_heads > kMaxRowsOfHeads)
        return fail(XATTN_EUNSUPPORTED, "%s: total_q * n_q_heads = %ld exceeds %d", who, (long)total_q * n_q_heads, kMaxRowsOfHeads);
    return XATTN_OK;
}

int make_rope(const char* who, const void* q, const void* k_new, const void* v_new, int64_t q_stride, int64_t k_stride, int64_t v_stride,
              const int32_t* pos, const float* inv_freq, const int32_t* sections, int n_axes, int flags, void* const* k_ptrs,
              void* const* v_ptrs, const int32_t* q_starts, const int32_t* kv_lens, int batch, int total_q, int n_q_heads, int n_kv_heads,
              int head_dim, void* q_out, RopeParams* prm_out) {
    if (!q || !k_new || !v_new || !pos || !sections || !k_ptrs || !v_ptrs || !q_starts || !kv_lens || !q_out)
        return fail(XATTN_EINVAL, "%s: NULL argument", who);
    const int st = check_packed_batch(who, batch, total_q, n_q_heads, n_kv_heads, head_dim);
    if (st != XATTN_OK) return st;
    if (flags & ~(XATTN_ROPE_PAIRS | XATTN_ROPE_DEALT)) return fail(XATTN_EINVAL, "%s: unknown flags 0x%x", who, flags);
    if (head_dim % 16 != 0 || head_dim > kRopeMaxHeadDim)
        return fail(XATTN_EUNSUPPORTED, "%s: head_dim %d is not a multiple of 16 up to %d", who, head_dim, kRopeMaxHeadDim);
    if (n_axes < 1 || n_axes > kRopeMaxAxes) return fail(XATTN_EUNSUPPORTED, "%s: %d axes: one to four are supported", who, n_axes);
    int left[kRopeMaxAxes] = {}, frequencies = 0;
    for (int a = 0; a < n_axes; ++a) {
        if (sections[a] < 0 || sections[a] > head_dim / 2)
            return fail(XATTN_EINVAL, "%s: section %d has %d frequencies of head_dim / 2 = %d", who, a, (int)sections[a], head_dim / 2);
        left[a] = sections[a];
        frequencies += sections[a];
    }
    if (frequencies > head_dim / 2)
        return fail(XATTN_EINVAL, "%s: %d frequencies in all, head_dim %d has %d", who, frequencies, head_dim, head_dim / 2);
    if (frequencies > 0 && !inv_freq) return fail(XATTN_EINVAL, "%s: NULL argument", who);
    if (frequencies % 8 != 0) return fail(XATTN_EUNSUPPORTED, "%s: %d frequencies in all: a multiple of 8 is supported", who, frequencies);
    if (q_stride < (int64_t)n_q_heads * head_dim || k_stride < (int64_t)n_kv_heads * head_dim || v_stride < (int64_t)n_kv_heads * head_dim)
        return fail(XATTN_EINVAL, "%s: a row stride is less than the row's heads * head_dim", who);
    if (q_stride > (int64_t)1 << 32 || k_stride > (int64_t)1 << 32 || v_stride > (int64_t)1 << 32)
        return fail(XATTN_EUNSUPPORTED, "%s: a row stride exceeds 2^32 values", who);
    if (q_stride % 8 != 0 || k_stride % 8 != 0 || v_stride % 8 != 0 || misaligned(q, 16) || misaligned(k_new, 16) || misaligned(v_new, 16) ||
        misaligned(q_out, 16))
        return fail(XATTN_EINVAL, "%s: q, k_new, v_new, q_out and the row strides must be multiples of 16 bytes", who);

    if (q_out == q && q_stride != (int64_t)n_q_heads * head_dim)
        return fail(XATTN_EINVAL, "%s: q_out may be q only where q's rows are contiguous", who);

    RopeParams& prm = *prm_out;
    prm = RopeParams{};
    prm.q = static_cast<const uint16_t*>(q);
    prm.k = static_cast<const uint16_t*>(k_new);
    prm.v = static_cast<const uint16_t*>(v_new);
    prm.q_stride = q_stride;
    prm.k_stride = k_stride;
    prm.v_stride = v_stride;
    prm.pos = pos;
    prm.inv_freq = inv_freq;
    prm.k_ptrs = k_ptrs;
    prm.v_ptrs = v_ptrs;
    prm.q_starts = q_starts;
    prm.kv_lens = kv_lens;
    prm.q_out = static_cast<uint16_t*>(q_out);
    prm.batch = batch;
    prm.total_q = total_q;
    prm.n_q_heads = n_q_heads;
    prm.n_kv_heads = n_kv_heads;
    prm.head_dim = head_dim;
    prm.frequencies = frequencies;
    prm.pairs = flags & XATTN_ROPE_PAIRS ? 1 : 0;
    for (int i = 0, axis = 0; i < frequencies; ++i) {
        while (left[axis] == 0) axis = (axis + 1) % n_axes;
        prm.axis_of[i >> 4] |= (uint32_t)axis << (2 * (i & 15));
        --left[axis];
        if (flags & XATTN_ROPE_DEALT) axis = (axis + 1) % n_axes;
    }
    return XATTN_OK;
}

}  // namespace xattn

using namespace xattn;

extern "C" {

size_t xattn_prefill_workspace_bytes(int batch, int total_q, int n_q_heads, int n_kv_heads, int head_dim) {
    if (check_prefill("xattn_prefill_workspace_bytes", batch, total_q, n_q_heads, n_kv_heads, head_dim) != XATTN_OK) return 0;
    return prefill_layout(total_q, n_q_heads / n_kv_heads).total;
}

int xattn_prefill(const void* q, const void* const* k_ptrs, const void* const* v_ptrs, const int32_t* q_starts,
                  const int32_t* kv_lens, int batch, int total_q, int n_q_heads, int n_kv_heads, int head_dim, float scale,
                  void* out, float* lse, void* stream) {
    const char* const who = "xattn_prefill";
    if (!q || !k_ptrs || !v_ptrs || !q_starts || !kv_lens || !out)
        return fail(XATTN_EINVAL, "%s: q, k_ptrs, v_ptrs, q_starts, kv_lens and out must not be NULL", who);
    int st = check_prefill(who, batch, total_q, n_q_heads, n_kv_heads, head_dim);
    if (st != XATTN_OK) return st;
    // The kernel takes a row's maximum ahead of the scale, which must be positive for that.
    const float scale_log2 = scale == 0.0f ? 1.0f : (float)(std::fabs((double)scale) * 1.4426950408889634074);
    if (!std::isfinite(scale_log2)) return fail(XATTN_EINVAL, "%s: scale, or scale * log2 e, is not finite", who);
    if (misaligned(q, 16) || misaligned(out, 16)) return fail(XATTN_EINVAL, "%s: q and out must be 16-byte aligned", who);

    PrefillParams prm;
    prm.q = static_cast<const uint16_t*>(q);
    prm.k_ptrs = k_ptrs;
    prm.v_ptrs = v_ptrs;
    prm.q_starts = q_starts;
    prm.kv_lens = kv_lens;
    prm.batch = batch;
    prm.total_q = total_q;
    prm.n_q_heads = n_q_heads;
    prm.n_kv_heads = n_kv_heads;
    prm.group = n_q_heads / n_kv_heads;
    prm.scale_log2 = scale_log2;
    prm.q_and = scale == 0.0f ? 0u : 0xffffffffu;
    prm.q_xor = scale < 0.0f ? 0x80008000u : 0u;
    prm.out = static_cast<uint16_t*>(out);
    prm.lse = lse;
    const PrefillLayout w = prefill_layout(total_q, prm.group);
    prm.slot_rows = w.slot_rows;
    struct Call {
        PrefillParams* prm;
        size_t ml_off, o_off;
        hipStream_t stream;
    } call = {&prm, w.ml_off, w.o_off, static_cast<hipStream_t>(stream)};
    return with_workspace(who, w.total, stream, [](void* context, char* ws) {
        const Call& c = *static_cast<Call*>(context);
        c.prm->table = reinterpret_cast<int32_t*>(ws);
        c.prm->part_ml = reinterpret_cast<float*>(ws + c.ml_off);
        c.prm->part_o = reinterpret_cast<float*>(ws + c.o_off);
        c.prm->exact = configured_pv_mode() == 1;
        const hipError_t e = launch_prefill(*c.prm, c.stream);
        return e == hipSuccess ? (int)XATTN_OK : fail_hip(e, "kernel launch");
    }, &call);
}

int xattn_rope_kvcache(const void* q, const void* k_new, const void* v_new, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                       const int32_t* pos, const float* inv_freq, const int32_t* sections, int n_axes, int flags,
                       void* const* k_ptrs, void* const* v_ptrs, const int32_t* q_starts, const int32_t* kv_lens, int batch,
                       int total_q, int n_q_heads, int n_kv_heads, int head_dim, void* q_out, void* stream) {
    RopeParams prm;
    const int st = make_rope("xattn_rope_kvcache", q, k_new, v_new, q_stride, k_stride, v_stride, pos, inv_freq, sections, n_axes, flags, k_ptrs, v_ptrs,
                             q_starts, kv_lens, batch, total_q, n_q_heads, n_kv_heads, head_dim, q_out, &prm);
    if (st != XATTN_OK) return st;
    const hipError_t e = launch_rope(prm, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)XATTN_OK : fail_hip(e, "kernel launch");
}

size_t xbeam_logprobs_workspace_bytes(int rows, int vocab, int top_k) {
    if (check_logprobs("xbeam_logprobs_workspace_bytes", rows, vocab, top_k) != XATTN_OK) return 0;
    const size_t bytes = logprobs_cut(rows, vocab, top_k).workspace;
    return bytes < 256 ? 256 : bytes;
}

int xbeam_logprobs(const void* logits, int dtype, int64_t row_stride, int rows, int vocab, float scale, const int32_t* tokens,
                   int top_k, float* token_lp, float* top_lp, int32_t* top_tok, float* lse, float* entropy, void* stream) {
    const char* const who = "xbeam_logprobs";
    if (!logits) return fail(XATTN_EINVAL, "%s: logits must not be NULL", who);
    int st = check_logprobs(who, rows, vocab, top_k);
    if (st != XATTN_OK) return st;
    if (dtype != XBEAM_BF16 && dtype != XBEAM_FP16 && dtype != XBEAM_FP32) return fail(XATTN_EINVAL, "%s: unknown dtype %d", who, dtype);
    if ((tokens == nullptr) != (token_lp == nullptr)) return fail(XATTN_EINVAL, "%s: tokens and token_lp go together", who);
    if ((top_k > 0) != (top_lp != nullptr) || (top_k > 0) != (top_tok != nullptr))
        return fail(XATTN_EINVAL, "%s: top_lp and top_tok go with a positive top_k, and only with that", who);
    if (!tokens && top_k == 0 && !lse && !entropy) return fail(XATTN_EINVAL, "%s: nothing is asked for", who);
    if (row_stride < vocab) return fail(XATTN_EINVAL, "%s: row_stride is less than vocab", who);
    if (!std::isfinite(scale) || !(scale > 0.0f)) return fail(XATTN_EINVAL, "%s: scale %g is not a positive finite number", who, (double)scale);
    if (scale > 1048576.0f || scale < 1.0f / 1048576.0f) return fail(XATTN_EUNSUPPORTED, "%s: scale %g is not within 2^-20 to 2^20", who, (double)scale);
    if (misaligned(logits, dtype == XBEAM_FP32 ? 4 : 2)) return fail(XATTN_EINVAL, "%s: logits are not aligned to their type", who);

    LogprobsParams prm = {};
    prm.logits = logits;
    prm.dtype = dtype;
    prm.row_stride = row_stride;
    prm.rows = rows;
    prm.vocab = vocab;
    prm.scale = scale;
    prm.scale_log2 = (float)((double)scale * 1.4426950408889634074);
    prm.tokens = tokens;
    prm.top_k = top_k;
    prm.token_lp = token_lp;
    prm.top_lp = top_lp;
    prm.top_tok = top_tok;
    prm.lse = lse;
    prm.entropy = entropy;
    struct Call {
        LogprobsParams* prm;
        LogprobsCut cut;
        hipStream_t stream;
    } call = {&prm, logprobs_cut(rows, vocab, top_k), static_cast<hipStream_t>(stream)};
    auto launch = [](void* context, char* ws) {
        const Call& c = *static_cast<Call*>(context);
        c.prm->workspace = ws;
        const hipError_t e = launch_logprobs(*c.prm, c.cut, c.stream);
        return e == hipSuccess ? (int)XATTN_OK : fail_hip(e, "kernel launch");
    };
    return call.cut.workspace ? with_workspace(who, call.cut.workspace, stream, launch, &call) : launch(&call, nullptr);
}

}  // extern "C"
