// The C-ABI layer around decode attention (csrc/xattn_step_api.cpp) on a stand-in for the HIP runtime and the launches: workspaces
// that cannot be had, streams under capture, what reaches the kernels; and how rows of logits are cut.  Prints "all scenarios ran"
// and exits with 0 if every check held.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../../include/xattn.h"
#include "../../include/xbeam.h"
#include "../../paper_2510_14686_amd/csrc/xattn_host.h"
#include "../../paper_2510_14686_amd/csrc/xattn_kernels.h"
#include "../../paper_2510_14686_amd/csrc/xattn_prefill.h"
#include "../../paper_2510_14686_amd/csrc/xattn_rope.h"
#include "../../paper_2510_14686_amd/csrc/xbeam_logprobs.h"

static hipError_t g_recorded = hipSuccess;      // the runtime's last error
static size_t g_free = (size_t)1 << 40;         // largest allocation that succeeds
static bool g_capturing = false;
static std::vector<size_t> g_allocs;
static hipError_t record(hipError_t e) {
    if (e != hipSuccess) g_recorded = e;
    return e;
}

extern "C" {
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipMalloc(void** p, size_t bytes) {
    if (bytes > g_free) return record(hipErrorOutOfMemory);
    g_allocs.push_back(bytes);
    *p = reinterpret_cast<void*>((uintptr_t)(g_allocs.size() << 44));      // never dereferenced
    return hipSuccess;
}
hipError_t hipGetLastError() { const hipError_t e = g_recorded; g_recorded = hipSuccess; return e; }
const char* hipGetErrorString(hipError_t) { return "stand-in error"; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) {
    *s = g_capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
    return hipSuccess;
}
hipError_t hipEventCreate(hipEvent_t*) { return record(hipErrorUnknown); }
hipError_t hipEventSynchronize(hipEvent_t) { return record(hipErrorUnknown); }
hipError_t hipEventElapsedTime(float*, hipEvent_t, hipEvent_t) { return record(hipErrorUnknown); }
hipError_t hipMemcpy(void*, const void*, size_t, hipMemcpyKind) { return record(hipErrorUnknown); }
}

namespace xattn {
static int g_launches = 0;
static hipError_t g_launch_fails = hipSuccess;
static PrefillParams g_prefill;
static RopeParams g_rope;
static LogprobsParams g_logprobs;
static LogprobsCut g_cut;
static hipError_t launched() {
    if (g_launch_fails != hipSuccess) return g_launch_fails;
    ++g_launches;
    return hipSuccess;
}
bool use_matrix_path(int path) { return path != kPathVector; }
int rows_per_wave(int rows_total, int) { return rows_total <= 16 ? 16 : 32; }
void mla_block_shape(int, int, int* waves, int* tiles) { *waves = 8; *tiles = 1; }
hipError_t launch_decode(const DecodeParams&, hipStream_t, hipEvent_t*) { return launched(); }
hipError_t launch_mla_decode(const MlaParams&, hipStream_t, hipEvent_t*) { return launched(); }
hipError_t launch_write_kvcache(const WriteParams&, hipStream_t) { return launched(); }
hipError_t launch_prefill(const PrefillParams& prm, hipStream_t) { g_prefill = prm; return launched(); }
hipError_t launch_rope(const RopeParams& prm, hipStream_t) { g_rope = prm; return launched(); }
hipError_t launch_logprobs(const LogprobsParams& prm, const LogprobsCut& cut, hipStream_t) {
    g_logprobs = prm;
    g_cut = cut;
    return launched();
}
}  // namespace xattn
using namespace xattn;

static int g_failures = 0;
#define CHECK(cond)                                                                                        \
    do {                                                                                                   \
        if (!(cond)) {                                                                                     \
            std::fprintf(stderr, "CHECK failed at line %d: %s (%s)\n", __LINE__, #cond, xattn_last_error()); \
            ++g_failures;                                                                                  \
        }                                                                                                  \
    } while (0)

static char g_buffer[64] __attribute__((aligned(64)));
static void* const A = g_buffer;
static void** const P = reinterpret_cast<void**>(g_buffer);
static int32_t* const I = reinterpret_cast<int32_t*>(g_buffer);
static float* const F = reinterpret_cast<float*>(g_buffer);
static void* stream(intptr_t s) { return reinterpret_cast<void*>(s); }
static int prefill(intptr_t s, int batch, int total, int hq, int hkv, float scale = 0.1f) {
    return xattn_prefill(A, P, P, I, I, batch, total, hq, hkv, 128, scale, A, nullptr, stream(s));
}
static int logprobs(intptr_t s, int rows, int vocab, int k) {
    return xbeam_logprobs(A, XBEAM_FP32, vocab, rows, vocab, 1.0f, nullptr, k, nullptr, k ? F : nullptr, k ? I : nullptr, F, nullptr, stream(s));
}
static int rope(const int32_t* sections, int n_axes, int flags) {
    return xattn_rope_kvcache(A, A, A, 1024, 256, 256, I, F, sections, n_axes, flags, P, P, I, I, 2, 9, 8, 2, 128, A, stream(9));
}

// A workspace that cannot be had, or would have to be made under capture, fails the call and launches nothing; the next call works.
static void workspaces() {
    g_free = 0;
    const int before = g_launches;
    CHECK(prefill(1, 4, 5000, 32, 8) == XATTN_ENOMEM);
    CHECK(logprobs(1, 1, 131072, 20) == XATTN_ENOMEM);
    CHECK(g_launches == before && g_recorded == hipSuccess);
    CHECK(logprobs(1, 5000, 131072, 20) == XATTN_OK);            // a workgroup per row: no workspace
    g_free = (size_t)1 << 40;
    g_capturing = true;
    CHECK(prefill(2, 4, 5000, 32, 8) == XATTN_ENOMEM);
    CHECK(logprobs(2, 1, 131072, 20) == XATTN_ENOMEM);
    g_capturing = false;
    CHECK(prefill(2, 4, 5000, 32, 8) == XATTN_OK);
    g_capturing = true;
    CHECK(prefill(2, 4096, 1 << 20, 64, 8) == XATTN_OK);         // no shape needs more
    CHECK(logprobs(2, 1, 131072, 20) == XATTN_OK);
    g_capturing = false;
    CHECK(reinterpret_cast<char*>(g_prefill.part_ml) >= reinterpret_cast<char*>(g_prefill.table) + kPrefillTableBytes);
    CHECK(reinterpret_cast<char*>(g_prefill.part_o) >= reinterpret_cast<char*>(g_prefill.part_ml) + (size_t)kPrefillSlots * g_prefill.slot_rows * 8);
    CHECK(reinterpret_cast<char*>(g_prefill.part_o) + (size_t)kPrefillSlots * g_prefill.slot_rows * 512 <=
          reinterpret_cast<char*>(g_prefill.table) + xattn_prefill_workspace_bytes(4096, 1 << 20, 64, 8, 128));
    // a caller's
    for (int total : {1, 20, 5000}) {
        const size_t need = xattn_prefill_workspace_bytes(2, total, 16, 2, 128);
        CHECK(xattn_set_workspace(reinterpret_cast<void*>((uintptr_t)1 << 61), need) == XATTN_OK);
        CHECK(prefill(3, 2, total, 16, 2) == XATTN_OK);
        CHECK(xattn_set_workspace(reinterpret_cast<void*>((uintptr_t)1 << 61), need - 1) == XATTN_OK);
        CHECK(prefill(3, 2, total, 16, 2) == XATTN_ENOMEM);
    }
    CHECK(xattn_set_workspace(nullptr, 0) == XATTN_OK);
    g_launch_fails = hipErrorUnknown;
    CHECK(prefill(2, 4, 5000, 32, 8) == XATTN_EHIP && logprobs(2, 1, 131072, 20) == XATTN_EHIP && logprobs(2, 1, 100, 20) == XATTN_EHIP);
    const int32_t one[] = {64};
    CHECK(rope(one, 1, 0) == XATTN_EHIP);
    g_launch_fails = hipSuccess;
}

// The kernel takes a positive scale: the sign and a zero go into Q.
static void scales() {
    CHECK(prefill(2, 1, 1, 8, 8, 0.5f) == XATTN_OK && g_prefill.q_and == 0xffffffffu && g_prefill.q_xor == 0 && g_prefill.scale_log2 > 0.72f && g_prefill.scale_log2 < 0.73f);
    CHECK(prefill(2, 1, 1, 8, 8, -0.5f) == XATTN_OK && g_prefill.q_xor == 0x80008000u && g_prefill.scale_log2 > 0.72f);
    CHECK(prefill(2, 1, 1, 8, 8, 0.0f) == XATTN_OK && g_prefill.q_and == 0 && g_prefill.scale_log2 > 0.0f);
}

// Which axis a frequency belongs to.
static void axes() {
    const int32_t sections[] = {3, 0, 7, 6};
    CHECK(rope(sections, 4, 0) == XATTN_OK && g_rope.frequencies == 16);
    for (int i = 0; i < 16; ++i) CHECK((int)(g_rope.axis_of[0] >> 2 * i & 3) == (i < 3 ? 0 : i < 10 ? 2 : 3));
    CHECK(rope(sections, 4, XATTN_ROPE_DEALT | XATTN_ROPE_PAIRS) == XATTN_OK && g_rope.pairs == 1);
    const int dealt[] = {0, 2, 3, 0, 2, 3, 0, 2, 3, 2, 3, 2, 3, 2, 3, 2};
    for (int i = 0; i < 16; ++i) CHECK((int)(g_rope.axis_of[0] >> 2 * i & 3) == dealt[i]);
    const int32_t last[] = {0, 64};
    CHECK(rope(last, 2, XATTN_ROPE_DEALT) == XATTN_OK);
    for (int i = 0; i < 64; ++i) CHECK((g_rope.axis_of[i >> 4] >> 2 * (i & 15) & 3) == 1);
}

// The parts of a row cover it once, begin at multiples of a step, and what they leave fits the merge and the workspace.
static void cuts() {
    unsigned seed = 1;
    auto draw = [&](unsigned n) { return (seed = seed * 1664525u + 1013904223u) / 65536u % n; };
    for (int i = 0; i < 200000; ++i) {
        const int vocab = 1 + (int)(((uint64_t)draw(65536) << 8 | draw(256)) >> draw(24)), rows = 1 + (int)(draw(4096) >> draw(12));
        const int k = (int)(draw(513) >> draw(10)) < vocab ? 0 : vocab, top_k = k ? (k < 512 ? k : 512) : (int)draw((unsigned)(vocab < 512 ? vocab : 512) + 1);
        const LogprobsCut c = logprobs_cut(rows, vocab, top_k);
        CHECK(c.parts >= 1 && (int64_t)c.parts * c.part_size >= vocab && (int64_t)(c.parts - 1) * c.part_size < vocab);
        CHECK(c.parts == 1 || (c.part_size % kStep == 0 && c.parts * top_k <= kMostMerged && (int64_t)rows * c.parts <= kParts));
        CHECK(c.workspace == (c.parts == 1 ? 0 : (size_t)rows * c.parts * (16 + 8 * (size_t)top_k)));
        CHECK(c.workspace <= xbeam_logprobs_workspace_bytes(rows, vocab, top_k));
    }
}

int main() {
    workspaces();
    scales();
    axes();
    cuts();
    CHECK(g_recorded == hipSuccess);
    if (g_failures) return 1;
    std::puts("all scenarios ran");
    return 0;
}
