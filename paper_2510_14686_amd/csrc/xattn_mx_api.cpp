// C-ABI entry points of the cache of 4 bits a value and of draft verification.  Argument checks, workspaces, launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/xattn.h"
#include "../../include/xbeam.h"
#include "xattn_hip_error.h"
#include "xattn_host.h"
#include "xattn_mx.h"
#include "xbeam_verify.h"

namespace xattn {

namespace {

constexpr int kMxMaxHeads = 1024;
constexpr int kMaxVerifyBatch = 4096, kMaxVerifyQLen = 16, kMaxVerifyVocab = 1 << 24;

bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

int check_verify(const char* who, int batch, int q_len, int vocab) {
    if (batch < 1 || q_len < 1 || vocab < 1) return fail(XATTN_EINVAL, "%s: batch, q_len and vocab must be positive", who);
    if (batch > kMaxVerifyBatch) return fail(XATTN_EUNSUPPORTED, "%s: batch %d exceeds %d", who, batch, kMaxVerifyBatch);
    if (q_len > kMaxVerifyQLen) return fail(XATTN_EUNSUPPORTED, "%s: q_len %d exceeds %d", who, q_len, kMaxVerifyQLen);
    if (vocab > kMaxVerifyVocab) return fail(XATTN_EUNSUPPORTED, "%s: vocab %d exceeds %d", who, vocab, kMaxVerifyVocab);
    return XATTN_OK;
}

int check_scale(const char* who, const char* name, float scale) {
    if (!std::isfinite(scale) || !(scale > 0.0f)) return fail(XATTN_EINVAL, "%s: %s %g is not a positive finite number", who, name, (double)scale);
    if (scale > 1048576.0f || scale < 1.0f / 1048576.0f) return fail(XATTN_EUNSUPPORTED, "%s: %s %g is not within 2^-20 to 2^20", who, name, (double)scale);
    return XATTN_OK;
}

}  // namespace

}  // namespace xattn

using namespace xattn;

extern "C" {

size_t xattn_mx_range_bytes(int64_t tokens, int n_kv_heads, int head_dim) {
    const char* const who = "xattn_mx_range_bytes";
    if (tokens < 0 || n_kv_heads < 1 || head_dim < 1) {
        fail(XATTN_EINVAL, "%s: tokens must not be negative, n_kv_heads and head_dim must be positive", who);
        return 0;
    }
    if (head_dim != kHeadDim || n_kv_heads > kMxMaxHeads || tokens > INT32_MAX) {
        fail(XATTN_EUNSUPPORTED, "%s: head_dim 128, up to 1024 heads and 2^31 - 1 tokens are supported", who);
        return 0;
    }
    return (size_t)((tokens + kMxTileTokens - 1) / kMxTileTokens) * (size_t)n_kv_heads * kMxTileBytes;
}

size_t xattn_decode_mx_workspace_bytes(int batch, int q_len, int n_q_heads, int n_kv_heads, int head_dim) {
    if (check_decode_shape(batch, q_len, n_q_heads, n_kv_heads, head_dim) != XATTN_OK) return 0;
    if (n_kv_heads > kMxMaxHeads) {
        fail(XATTN_EUNSUPPORTED, "xattn_decode_mx_workspace_bytes: %d KV heads: more than %d", n_kv_heads, kMxMaxHeads);
        return 0;
    }
    return decode_layout(batch, q_len, n_q_heads, mx_cut(q_len, n_q_heads, n_kv_heads).pieces).total;
}

int xattn_decode_mx(const void* q, const void* const* k_ptrs, const void* const* v_ptrs, const int32_t* kv_lens, int batch, int q_len,
                    int n_q_heads, int n_kv_heads, int head_dim, float scale, void* out, float* lse, void* stream) {
    const char* const who = "xattn_decode_mx";
    if (!q || !k_ptrs || !v_ptrs || !kv_lens || !out)
        return fail(XATTN_EINVAL, "%s: q, k_ptrs, v_ptrs, kv_lens and out must not be NULL", who);
    const int st = check_decode_shape(batch, q_len, n_q_heads, n_kv_heads, head_dim);
    if (st != XATTN_OK) return st;
    if (n_kv_heads > kMxMaxHeads) return fail(XATTN_EUNSUPPORTED, "%s: %d KV heads: more than %d", who, n_kv_heads, kMxMaxHeads);
    const float scale_log2 = (float)((double)scale * 1.4426950408889634074);
    if (!std::isfinite(scale) || !std::isfinite(scale_log2)) return fail(XATTN_EINVAL, "%s: scale, or scale * log2 e, is not finite", who);
    if (misaligned(q, 16) || misaligned(out, 16)) return fail(XATTN_EINVAL, "%s: q and out must be 16-byte aligned", who);

    DecodeParams prm = {};
    prm.q = static_cast<const uint16_t*>(q);
    prm.k_ptrs = k_ptrs;
    prm.v_ptrs = v_ptrs;
    prm.kv_lens = kv_lens;
    prm.batch = batch;
    prm.q_len = q_len;
    prm.n_q_heads = n_q_heads;
    prm.n_kv_heads = n_kv_heads;
    prm.group = n_q_heads / n_kv_heads;
    prm.inv_group = 1.0f / (float)prm.group;
    prm.scale_log2 = scale_log2;
    prm.out = static_cast<uint16_t*>(out);
    prm.lse = lse;
    const MxCut cut = mx_cut(q_len, n_q_heads, n_kv_heads);
    prm.n_pieces = cut.pieces;
    prm.min_piece_tokens = cut.waves * kMxPositions;
    prm.few = FewPieces{prm.n_pieces, kMxPositions};
    prm.xcd_skew = 0;
    struct Call {
        DecodeParams* prm;
        const MxCut* cut;
        DecodeLayout w;
        hipStream_t stream;
    } call = {&prm, &cut, decode_layout(batch, q_len, n_q_heads, cut.pieces), static_cast<hipStream_t>(stream)};
    return with_workspace(who, call.w.total, stream, [](void* context, char* ws) {
        const Call& c = *static_cast<Call*>(context);
        c.prm->meta = reinterpret_cast<int32_t*>(ws + c.w.meta_off);
        c.prm->part_ml = reinterpret_cast<float*>(ws + c.w.ml_off);
        c.prm->part_o = reinterpret_cast<float*>(ws + c.w.o_off);
        const hipError_t e = launch_decode_mx(*c.prm, *c.cut, c.stream);
        return e == hipSuccess ? (int)XATTN_OK : fail_hip(e, "kernel launch");
    }, &call);
}

int xattn_rope_kvcache_mx(const void* q, const void* k_new, const void* v_new, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                          const int32_t* pos, const float* inv_freq, const int32_t* sections, int n_axes, int flags,
                          void* const* k_ptrs, void* const* v_ptrs, const int32_t* q_starts, const int32_t* kv_lens, int batch,
                          int total_q, int n_q_heads, int n_kv_heads, int head_dim, void* q_out, void* stream) {
    const char* const who = "xattn_rope_kvcache_mx";
    if (head_dim > 0 && head_dim != kHeadDim) return fail(XATTN_EUNSUPPORTED, "%s: head_dim %d: only 128 is supported", who, head_dim);
    RopeParams prm;
    const int st = make_rope(who, q, k_new, v_new, q_stride, k_stride, v_stride, pos, inv_freq, sections, n_axes, flags, k_ptrs, v_ptrs, q_starts, kv_lens,
                             batch, total_q, n_q_heads, n_kv_heads, head_dim, q_out, &prm);
    if (st != XATTN_OK) return st;
    const hipError_t e = launch_rope_mx(prm, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)XATTN_OK : fail_hip(e, "kernel launch");
}

int xattn_read_kvcache_mx(const void* const* k_ptrs, const void* const* v_ptrs, const int32_t* q_starts, const int32_t* kv_lens, int batch,
                          int total_q, int n_kv_heads, int head_dim, void* k_out, void* v_out, void* stream) {
    const char* const who = "xattn_read_kvcache_mx";
    if (!k_ptrs || !v_ptrs || !q_starts || !kv_lens || !k_out || !v_out) return fail(XATTN_EINVAL, "%s: NULL argument", who);
    const int st = check_packed_batch(who, batch, total_q, n_kv_heads, n_kv_heads, head_dim);
    if (st != XATTN_OK) return st;
    if (head_dim != kHeadDim) return fail(XATTN_EUNSUPPORTED, "%s: head_dim %d: only 128 is supported", who, head_dim);
    if (misaligned(k_out, 16) || misaligned(v_out, 16)) return fail(XATTN_EINVAL, "%s: k_out and v_out must be 16-byte aligned", who);
    const ReadMxParams prm = {k_ptrs, v_ptrs, q_starts, kv_lens, static_cast<uint16_t*>(k_out), static_cast<uint16_t*>(v_out), batch, total_q, n_kv_heads};
    const hipError_t e = launch_read_mx(prm, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)XATTN_OK : fail_hip(e, "kernel launch");
}

size_t xbeam_verify_workspace_bytes(int batch, int q_len, int vocab) {
    if (check_verify("xbeam_verify_workspace_bytes", batch, q_len, vocab) != XATTN_OK) return 0;
    const size_t with = verify_layout(batch, q_len, vocab, true).total, without = verify_layout(batch, q_len, vocab, false).total;
    return with > without ? with : without;
}

int xbeam_verify(const void* target, int64_t target_stride, const void* draft, int64_t draft_stride, int dtype, int vocab, float scale,
                 float draft_scale, const int32_t* draft_tokens, const int32_t* n_drafts, const float* uniforms, int batch, int q_len,
                 int flags, int32_t* tokens, int32_t* n_accepted, float* token_lp, void* stream) {
    const char* const who = "xbeam_verify";
    if (!target || !tokens || !n_accepted) return fail(XATTN_EINVAL, "%s: target, tokens and n_accepted must not be NULL", who);
    int st = check_verify(who, batch, q_len, vocab);
    if (st != XATTN_OK) return st;
    if (dtype != XBEAM_BF16 && dtype != XBEAM_FP16 && dtype != XBEAM_FP32) return fail(XATTN_EINVAL, "%s: unknown dtype %d", who, dtype);
    if (flags & ~XBEAM_GREEDY) return fail(XATTN_EINVAL, "%s: unknown flags 0x%x", who, flags);
    const bool greedy = (flags & XBEAM_GREEDY) != 0;
    if (q_len > 1 && !draft_tokens) return fail(XATTN_EINVAL, "%s: draft_tokens must not be NULL with q_len above 1", who);
    if (!greedy && !uniforms) return fail(XATTN_EINVAL, "%s: uniforms must not be NULL without XBEAM_GREEDY", who);
    if (greedy || q_len == 1) draft = nullptr;      // not looked at
    if (target_stride < vocab || (draft && draft_stride < vocab)) return fail(XATTN_EINVAL, "%s: a row stride is less than vocab", who);
    if ((st = check_scale(who, "scale", scale)) != XATTN_OK) return st;
    if (draft && (st = check_scale(who, "draft_scale", draft_scale)) != XATTN_OK) return st;
    const size_t size = dtype == XBEAM_FP32 ? 4 : 2;
    if (misaligned(target, size) || misaligned(draft, size)) return fail(XATTN_EINVAL, "%s: logits are not aligned to their type", who);

    VerifyParams prm = {};
    prm.target = target;
    prm.draft = draft;
    prm.target_stride = target_stride;
    prm.draft_stride = draft_stride;
    prm.dtype = dtype;
    prm.vocab = vocab;
    prm.scale = scale;
    prm.draft_scale = draft_scale;
    prm.draft_tokens = draft_tokens;
    prm.n_drafts = n_drafts;
    prm.uniforms = uniforms;
    prm.batch = batch;
    prm.q_len = q_len;
    prm.greedy = greedy ? 1 : 0;
    prm.tokens = tokens;
    prm.accepted = n_accepted;
    prm.token_lp = token_lp;
    struct Call {
        VerifyParams* prm;
        VerifyLayout w;
        hipStream_t stream;
    } call = {&prm, verify_layout(batch, q_len, vocab, draft != nullptr), static_cast<hipStream_t>(stream)};
    return with_workspace(who, call.w.total, stream, [](void* context, char* ws) {
        const Call& c = *static_cast<Call*>(context);
        c.prm->stats = reinterpret_cast<float2*>(ws);
        c.prm->best = reinterpret_cast<uint64_t*>(ws + c.w.best_off);
        c.prm->sums = reinterpret_cast<double*>(ws + c.w.sums_off);
        c.prm->decisions = ws + c.w.decisions_off;
        const hipError_t e = launch_verify(*c.prm, c.w, c.stream);
        return e == hipSuccess ? (int)XATTN_OK : fail_hip(e, "kernel launch");
    }, &call);
}

}  // extern "C"
