// The C-ABI layer of the 4-bit cache and of draft verification (csrc/xattn_mx_api.cpp) on a stand-in for the HIP runtime and the launches:
// workspaces that cannot be had, streams under capture, what reaches the kernels; how work is cut.  Prints "all scenarios ran" and exits
// with 0 if every check held.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../../include/xattn.h"
#include "../../include/xbeam.h"
#include "../../paper_2510_14686_amd/csrc/xattn_host.h"
#include "../../paper_2510_14686_amd/csrc/xattn_kernels.h"
#include "../../paper_2510_14686_amd/csrc/xattn_mx.h"
#include "../../paper_2510_14686_amd/csrc/xattn_prefill.h"
#include "../../paper_2510_14686_amd/csrc/xattn_rope.h"
#include "../../paper_2510_14686_amd/csrc/xbeam_logprobs.h"
#include "../../paper_2510_14686_amd/csrc/xbeam_verify.h"

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
static DecodeParams g_decode;
static MxCut g_cut;
static RopeParams g_rope;
static ReadMxParams g_read;
static VerifyParams g_verify;
static VerifyLayout g_layout;
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
hipError_t launch_prefill(const PrefillParams&, hipStream_t) { return launched(); }
hipError_t launch_rope(const RopeParams&, hipStream_t) { return launched(); }
hipError_t launch_logprobs(const LogprobsParams&, const LogprobsCut&, hipStream_t) { return launched(); }
hipError_t launch_decode_mx(const DecodeParams& prm, const MxCut& cut, hipStream_t) { g_decode = prm; g_cut = cut; return launched(); }
hipError_t launch_rope_mx(const RopeParams& prm, hipStream_t) { g_rope = prm; return launched(); }
hipError_t launch_read_mx(const ReadMxParams& prm, hipStream_t) { g_read = prm; return launched(); }
hipError_t launch_verify(const VerifyParams& prm, const VerifyLayout& w, hipStream_t) { g_verify = prm; g_layout = w; return launched(); }
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
static int decode(intptr_t s, int batch, int q_len, int hq, int hkv, float scale = 0.1f) {
    return xattn_decode_mx(A, P, P, I, batch, q_len, hq, hkv, 128, scale, A, nullptr, stream(s));
}
static int verify(intptr_t s, int batch, int q_len, int vocab, const void* draft, int flags = 0) {
    return xbeam_verify(A, vocab, draft, vocab, XBEAM_FP32, vocab, 1.0f, 0.5f, I, nullptr, F, batch, q_len, flags, I, I, nullptr, stream(s));
}

// A workspace that cannot be had, or would have to be made under capture, fails the call and launches nothing; the next call works.
static void workspaces() {
    g_free = 0;
    const int before = g_launches;
    CHECK(decode(1, 64, 4, 32, 8) == XATTN_ENOMEM);
    CHECK(verify(1, 8, 5, 131072, A) == XATTN_ENOMEM);
    CHECK(g_launches == before && g_recorded == hipSuccess);
    g_free = (size_t)1 << 40;
    g_capturing = true;
    CHECK(decode(2, 64, 4, 32, 8) == XATTN_ENOMEM);
    CHECK(verify(2, 8, 5, 131072, A) == XATTN_ENOMEM);
    CHECK(g_launches == before);
    g_capturing = false;
    CHECK(decode(2, 64, 1, 32, 8) == XATTN_OK);
    g_capturing = true;      // 32 MiB at least: these need no more
    CHECK(decode(2, 64, 4, 32, 8) == XATTN_OK);
    CHECK(verify(2, 64, 5, 131072, A) == XATTN_OK);
    g_capturing = false;
    for (int q_len : {1, 4, 8}) {      // a caller's
        const size_t need = xattn_decode_mx_workspace_bytes(5, q_len, 64, 8, 128);
        CHECK(xattn_set_workspace(reinterpret_cast<void*>((uintptr_t)1 << 61), need) == XATTN_OK);
        CHECK(decode(3, 5, q_len, 64, 8) == XATTN_OK);
        const char* const base = reinterpret_cast<char*>((uintptr_t)1 << 61);
        const size_t slots = (size_t)g_cut.pieces + 5, rows = (size_t)q_len * 64;
        CHECK(reinterpret_cast<char*>(g_decode.meta) == base && reinterpret_cast<char*>(g_decode.part_ml) >= base + 5 * 8);
        CHECK(reinterpret_cast<char*>(g_decode.part_o) >= reinterpret_cast<char*>(g_decode.part_ml) + slots * rows * 8);
        CHECK(reinterpret_cast<char*>(g_decode.part_o) + slots * rows * 512 <= base + need);
        CHECK(xattn_set_workspace(reinterpret_cast<void*>((uintptr_t)1 << 61), need - 1) == XATTN_OK);
        CHECK(decode(3, 5, q_len, 64, 8) == XATTN_ENOMEM);
    }
    for (int vocab : {7, 5000, 131072, 1 << 24}) {
        const size_t need = xbeam_verify_workspace_bytes(6, 5, vocab);
        CHECK(xattn_set_workspace(reinterpret_cast<void*>((uintptr_t)1 << 61), need) == XATTN_OK);
        const char* const base = reinterpret_cast<char*>((uintptr_t)1 << 61);
        for (int form = 0; form < 3; ++form) {
            CHECK(verify(3, 6, 5, vocab, form == 1 ? nullptr : A, form == 2 ? XBEAM_GREEDY : 0) == XATTN_OK);
            const size_t rows = form == 0 ? 6 * 9 : 6 * 5;
            CHECK(reinterpret_cast<char*>(g_verify.stats) == base);
            CHECK(reinterpret_cast<char*>(g_verify.best) >= base + rows * g_layout.read.parts * sizeof(float2));
            CHECK(reinterpret_cast<char*>(g_verify.sums) >= reinterpret_cast<char*>(g_verify.best) + (size_t)6 * 5 * g_layout.read.parts * 8);
            CHECK(static_cast<char*>(g_verify.decisions) >= reinterpret_cast<char*>(g_verify.sums) + (size_t)3 * 6 * g_layout.pick.parts * 8);
            CHECK(static_cast<char*>(g_verify.decisions) + 6 * 64 <= base + need);
        }
    }
    CHECK(xattn_set_workspace(nullptr, 0) == XATTN_OK);
    g_launch_fails = hipErrorUnknown;
    CHECK(decode(2, 4, 1, 32, 8) == XATTN_EHIP && verify(2, 1, 2, 100, A) == XATTN_EHIP);
    CHECK(xattn_read_kvcache_mx(P, P, I, I, 2, 9, 8, 128, A, A, nullptr) == XATTN_EHIP);
    const int32_t one[] = {64};
    CHECK(xattn_rope_kvcache_mx(A, A, A, 1024, 256, 256, I, F, one, 1, 0, P, P, I, I, 2, 9, 8, 2, 128, A, nullptr) == XATTN_EHIP);
    g_launch_fails = hipSuccess;
}

// What is not looked at does not reach the kernels; scales and sizes do.
static void arguments() {
    CHECK(verify(2, 3, 4, 1000, A, XBEAM_GREEDY) == XATTN_OK && g_verify.greedy == 1 && g_verify.draft == nullptr);
    CHECK(verify(2, 3, 1, 1000, A) == XATTN_OK && g_verify.draft == nullptr);
    CHECK(verify(2, 3, 4, 1000, A) == XATTN_OK && g_verify.draft == A && g_verify.scale == 1.0f && g_verify.draft_scale == 0.5f);
    CHECK(xbeam_verify(A, 1000, nullptr, 0, XBEAM_FP32, 1000, 1.0f, 0.0f, I, I, F, 3, 4, 0, I, I, F, stream(2)) == XATTN_OK);      // draft_scale: not looked at
    CHECK(xbeam_verify(A, 1000, nullptr, 0, XBEAM_FP32, 1000, 1.0f, 0.0f, nullptr, nullptr, F, 3, 1, 0, I, I, F, stream(2)) == XATTN_OK);
    CHECK(xbeam_verify(A, 1000, nullptr, 0, XBEAM_FP32, 1000, 1.0f, 0.0f, I, nullptr, nullptr, 3, 4, XBEAM_GREEDY, I, I, F, stream(2)) == XATTN_OK);
    CHECK(decode(2, 3, 2, 12, 2, -0.5f) == XATTN_OK && g_decode.scale_log2 < -0.72f && g_decode.scale_log2 > -0.73f && g_decode.group == 6);
    CHECK(xattn_read_kvcache_mx(P, P, I, I, 2, 9, 5, 128, A, A, nullptr) == XATTN_OK && g_read.total_q == 9 && g_read.n_kv_heads == 5);
    const int32_t sections[] = {8, 0, 24};
    CHECK(xattn_rope_kvcache_mx(A, A, A, 1024, 256, 256, I, F, sections, 3, XATTN_ROPE_PAIRS, P, P, I, I, 2, 9, 8, 2, 128, A, nullptr) == XATTN_OK);
    CHECK(g_rope.frequencies == 32 && g_rope.pairs == 1 && (g_rope.axis_of[0] >> 2 * 7 & 3) == 0 && (g_rope.axis_of[0] >> 2 * 8 & 3) == 2);
}

// Every shape is cut into workgroups that there are kernels for, pieces in multiples of eight; a piece's tiles are dealt to its waves once.
static void cuts() {
    for (int hkv = 1; hkv <= 128; ++hkv)
        for (int group = 1; group <= 64; ++group)
            for (int q_len = 1; q_len <= 16 && group * q_len <= 64; ++q_len) {
                const MxCut c = mx_cut(q_len, group * hkv, hkv);
                CHECK(c.rows == (group * q_len <= 16 ? 16 : 32) && (c.waves == 4 || c.waves == (c.rows == 16 ? 12 : 8)));
                CHECK(c.pieces >= 8 && c.pieces <= kMaxPieces && (c.pieces % 8 == 0 || hkv == 1));
            }
    for (int parts : {4, 8, 12})
        for (int tiles = 1; tiles < 300; ++tiles) {
            const int len = tiles * kMxPositions, sub = mx_part_positions(len, parts);
            CHECK(sub % kMxPositions == 0 && (long)sub * parts >= len && sub - kMxPositions < (len + parts - 1) / parts);
        }
    for (int len : {-2147483647 - 1, -1, 0, 1, 63, 64, 65, 2147483647}) CHECK(mx_positions(len) == (len <= 0 ? 0 : (int)(((int64_t)len + 63) / 64 * kMxPositions)));
    unsigned seed = 1;
    auto draw = [&](unsigned n) { return (seed = seed * 1664525u + 1013904223u) / 65536u % n; };
    for (int i = 0; i < 100000; ++i) {
        const int vocab = 1 + (int)(((uint64_t)draw(65536) << 8 | draw(256)) >> draw(24)), batch = 1 + (int)(draw(4096) >> draw(12)), q_len = 1 + (int)draw(16);
        for (int with = 0; with < 2; ++with) {
            const VerifyLayout w = verify_layout(batch, q_len, vocab, with != 0);
            for (const VerifyCut& c : {w.read, w.pick})
                CHECK(c.parts >= 1 && c.parts <= kVerifyMostParts && (int64_t)c.parts * c.size >= vocab && (int64_t)(c.parts - 1) * c.size < vocab && c.size % kVerifyStep == 0);
            CHECK(w.total <= xbeam_verify_workspace_bytes(batch, q_len, vocab));
        }
    }
}

int main() {
    workspaces();
    arguments();
    cuts();
    CHECK(g_recorded == hipSuccess);
    if (g_failures) return 1;
    std::puts("all scenarios ran");
    return 0;
}
