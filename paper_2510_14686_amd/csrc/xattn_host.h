// Internal interface between the host translation units of libxattn.so.
#ifndef XATTN_HOST_H_
#define XATTN_HOST_H_

#include <stddef.h>
#include <stdint.h>

namespace xattn {

// Supplies a workspace of at least `bytes` bytes on device `device` without allocating, or fails with
// a recorded message.
typedef int (*FixedWorkspaceFn)(const char* who, int device, size_t bytes, char** ws_out);

int decode_call(const char* who, FixedWorkspaceFn fixed_workspace, const void* q, const void* const* k_ptrs,
                const void* const* v_ptrs, const int32_t* kv_lens, int batch, int q_len, int n_q_heads,
                int n_kv_heads, int head_dim, float scale, void* out, float* lse, void* stream);

// Runs launch(context, workspace) with at least `bytes` bytes of the workspace that calls on `stream` have (the caller's if one
// was handed over, else the library's own, grown when needed; see xattn_set_workspace), under the lock that keeps the launches of
// one call together.
typedef int (*WorkspaceLaunchFn)(void* context, char* workspace);
int with_workspace(const char* who, size_t bytes, void* stream, WorkspaceLaunchFn launch, void* context);
// XATTN_CFG_PV_MODE, for a launch under that lock.
int configured_pv_mode();

// Bounds on a decode call's sizes, and its workspace: the merge's table, (max, sum) and sums of each partial row.
int check_decode_shape(int batch, int q_len, int n_q_heads, int n_kv_heads, int head_dim);
struct DecodeLayout {
    size_t meta_off, ml_off, o_off, total;
};
DecodeLayout decode_layout(int batch, int q_len, int n_q_heads, int n_pieces);
// Bounds on a packed batch's sizes.
int check_packed_batch(const char* who, int batch, int total_q, int n_q_heads, int n_kv_heads, int head_dim);
// The checks of xattn_rope_kvcache, and what its kernel takes.
struct RopeParams;
int make_rope(const char* who, const void* q, const void* k_new, const void* v_new, int64_t q_stride, int64_t k_stride, int64_t v_stride,
              const int32_t* pos, const float* inv_freq, const int32_t* sections, int n_axes, int flags, void* const* k_ptrs,
              void* const* v_ptrs, const int32_t* q_starts, const int32_t* kv_lens, int batch, int total_q, int n_q_heads, int n_kv_heads,
              int head_dim, void* q_out, RopeParams* prm_out);

}  // namespace xattn
#endif
