// Attention of the new tokens of a batch of prompts (xattn_prefill): causal, grouped heads, sequences of different lengths
// packed one behind the other, keys and values in per-sequence ranges.
//
//   out = softmax(scale Q K^T + causal mask) V in one pass over the keys: with a running reference m and sum l per row,
//   a block of keys adds exp2(s - m) to l and exp2(s - m) V to o, both rescaled when m moves.
//
// The rows of a tile are (new token, query head of the group) pairs of one KV head, so that K and V are read once for the whole
// group, and a tile of a short sequence holds all its rows.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "xattn_device.h"
#include "xattn_launch.h"
#include "xattn_prefill.h"

namespace xattn {
namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef short s16x4v_t __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kWaveRows = kPrefillRows / kWaves;      // 32: the MFMA's columns
constexpr int kBlockBytes = kPrefillKeys * kRowBytes; // 16 KiB of K, or of V
constexpr float kLowest = -3.0e38f;                   // reference of a row that has seen no key
constexpr float kSlackLog2 = 8.0f;                    // how far a row's maximum may exceed its reference

// ------------------------------------------------------------------------------------------------ a workgroup's work
struct PrefillWork {
    PrefillSeq s;
    int b, parts, index;      // index: of the work among the sequence's (per KV head)
    int slot;                 // first slot of the sequence
    bool found;
};
__device__ __forceinline__ PrefillSeq load_seq(const PrefillParams& prm, int b) {
    const bool in = b < prm.batch;
    const int i = in ? b : 0;
    const int start = prm.q_starts[i], end = prm.q_starts[i + 1], kv = prm.kv_lens[i];
    return prefill_seq(in ? start : 0, in ? end : 0, in ? kv : 0, prm.total_q, prm.group);
}
// What work number j (per KV head) is: of all parts (kMerge false), or of all tiles in several parts (kMerge true).  Lane l has
// the sequences l << lg ..; one scan finds j's lane, another the sequence among the lane's.
template <bool kMerge>
__device__ __forceinline__ PrefillWork find_work(const PrefillParams& prm, int j, int lane) {
    const int lg = prm.batch <= 64 ? 0 : 26 - __builtin_clz((unsigned)(prm.batch - 1));
    const int chunk = 1 << lg;
    float cost = 0.0f;
    PrefillSeq s = {};
    for (int i = 0; i < chunk; ++i) {
        s = load_seq(prm, (lane << lg) + i);
        cost += prefill_cost(s);
    }
    const int share = prefill_share(wave_sum(cost) * (float)prm.n_kv_heads);
    auto amounts = [&](const PrefillSeq& q, int& work, int& slots) {
        const int parts = prefill_parts(q.blocks, share);
        const int split = parts > 1 ? q.tiles * parts : 0;
        work = kMerge ? (parts > 1 ? q.tiles : 0) : q.tiles * parts;
        slots = split;
        return parts;
    };
    int work = 0, slots = 0;
    if (chunk == 1) {
        amounts(s, work, slots);
    } else {
        for (int i = 0; i < chunk; ++i) {
            int w, n;
            amounts(load_seq(prm, (lane << lg) + i), w, n);
            work += w;
            slots += n;
        }
    }
    int before = wave_incl_scan_i(work) - work, slots_before = wave_incl_scan_i(slots) - slots;
    unsigned long long hit = __ballot(j >= before && j < before + work);
    PrefillWork r;
    r.found = hit != 0;
    int at = hit ? __builtin_ctzll(hit) : 0;
    r.index = j - __builtin_amdgcn_readlane(before, at);
    r.slot = __builtin_amdgcn_readlane(slots_before, at);
    r.b = at;
    if (chunk > 1) {
        const int first = at << lg;
        s = load_seq(prm, lane < chunk ? first + lane : prm.batch);
        amounts(s, work, slots);
        before = wave_incl_scan_i(work) - work;
        slots_before = wave_incl_scan_i(slots) - slots;
        hit = __ballot(r.index >= before && r.index < before + work);
        at = hit ? __builtin_ctzll(hit) : 0;
        r.index -= __builtin_amdgcn_readlane(before, at);
        r.slot += __builtin_amdgcn_readlane(slots_before, at);
        r.b = first + at;
    }
    r.slot *= prm.n_kv_heads;
    r.s.first = __builtin_amdgcn_readlane(s.first, at);
    r.s.q = __builtin_amdgcn_readlane(s.q, at);
    r.s.kv = __builtin_amdgcn_readlane(s.kv, at);
    r.s.tiles = __builtin_amdgcn_readlane(s.tiles, at);
    r.s.blocks = __builtin_amdgcn_readlane(s.blocks, at);
    r.parts = prefill_parts(r.s.blocks, share);
    return r;
}

// ------------------------------------------------------------------------------------------------ blocks
// Block at key0 of K or V: 1024 chunks of 16 bytes, four per thread, thread t chunk t % 16 of rows t / 16 + 16 i.  The descriptor
// ends with the sequence, so rows behind it (which an xTensor range need not have mapped) read as zero, and begins with the
// block, so a sequence may be larger than 32-bit offsets reach.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t block_rsrc(const char* head, int key0, int kv, int row_bytes) {
    const int keys = kv - key0 < kPrefillKeys ? kv - key0 : kPrefillKeys;
    return make_rsrc(head + (int64_t)key0 * row_bytes, keys > 0 ? (uint32_t)((keys - 1) * row_bytes + kRowBytes) : 0u);
}

// In LDS a row is 256 bytes.  K: chunk c of row r sits at c ^ (r & 15), so that the 16 rows that 16 lanes read a chunk
// of are in different banks; V: 64-byte piece x of row r at x ^ (r & 3), for the four rows of a transposing read.
__device__ __forceinline__ int k_off(int row, int chunk) { return row * kRowBytes + ((chunk ^ (row & 15)) << 4); }
__device__ __forceinline__ int v_off(int row, int chunk) { return row * kRowBytes + ((chunk ^ ((row & 3) << 2)) << 4); }

// S^T = K Q^T by 32x32x16 MFMA: lane (hh, n) = (lane / 32, lane % 32) gives chunk 8 hh .. of key row n and of query row n, and
// has, of query row n, the keys at rows 8 (i / 4) + 4 hh + i % 4 in accumulator i.  Row x of the operand is key tile_row(x) of the
// tile, which makes them the keys 16 (i / 8) + 8 hh + i % 8: accumulators 8 s .. 8 s + 7, as bf16, are the operand of the
// 16 keys of step s in O^T += V^T P^T.
__device__ __forceinline__ int tile_row(int x) { return (x & ~12) | ((x & 4) << 1) | ((x & 8) >> 1); }

__global__ __launch_bounds__(64 * kWaves, 2) void prefill_kernel(PrefillParams prm) {
    __shared__ __attribute__((aligned(16))) char lds[2 * 2 * kBlockBytes];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int head = blockIdx.x % (unsigned)prm.n_kv_heads;
    const PrefillWork w = find_work<false>(prm, (int)(blockIdx.x / (unsigned)prm.n_kv_heads), lane);
    if (!w.found) return;
    // Later tiles see more keys: first.
    const int tile = w.s.tiles - 1 - w.index / w.parts, part = w.index % w.parts;
    const int part_blocks = prefill_part_blocks(w.s.blocks, w.parts), blocks = prefill_tile_blocks(w.s, tile, prm.group);
    const int blk0 = part * part_blocks, blk1 = blk0 + part_blocks < blocks ? blk0 + part_blocks : blocks;
    if (part > 0 && blk0 >= blk1) return;
    const bool whole = blocks <= part_blocks;

    const int row_bytes = prm.n_kv_heads * kRowBytes;
    const char* const k_head = static_cast<const char*>(uniform(prm.k_ptrs[w.b])) + head * kRowBytes;
    const char* const v_head = static_cast<const char*>(uniform(prm.v_ptrs[w.b])) + head * kRowBytes;

    // This lane's query row.
    const int rows = w.s.q * prm.group, wave_row = tile * kPrefillRows + wave * kWaveRows, row = wave_row + n;
    const bool wave_on = wave_row < rows, row_on = row < rows;
    const int t = (int)((unsigned)row / (unsigned)prm.group), h = head * prm.group + (row - t * prm.group);
    const int64_t q_row = (int64_t)(w.s.first + t) * prm.n_q_heads + h;
    const int lim = row_on ? prefill_visible(w.s, t) : 0;
    const int last_row = wave_row + kWaveRows < rows ? wave_row + kWaveRows - 1 : rows - 1;
    const int lim_first = prefill_visible(w.s, (int)((unsigned)wave_row / (unsigned)prm.group));
    const int lim_last = wave_on ? prefill_visible(w.s, (int)((unsigned)last_row / (unsigned)prm.group)) : 0;

    bf16x8_t qop[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
        u32x4_t x = {0u, 0u, 0u, 0u};
        if (row_on) x = *reinterpret_cast<const u32x4_t*>(prm.q + q_row * kHeadDim + s * 16 + hh * 8);
        qop[s] = __builtin_bit_cast(bf16x8_t, (x & prm.q_and) ^ prm.q_xor);
    }

    f32x16_t o[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] = f32x16_t{};
    float m = kLowest, l = 0.0f;

    // Loads of a block, and their way into LDS.
    const int load_row = tid >> 4, load_chunk = tid & 15;
    uint32_t load_off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) load_off[i] = (uint32_t)((load_row + 16 * i) * row_bytes + load_chunk * 16);
    u32x4_t stage[8];
    auto load_block = [&](int blk) {
        const __amdgpu_buffer_rsrc_t rk = block_rsrc(k_head, blk * kPrefillKeys, w.s.kv, row_bytes);
        const __amdgpu_buffer_rsrc_t rv = block_rsrc(v_head, blk * kPrefillKeys, w.s.kv, row_bytes);
#pragma unroll
        for (int i = 0; i < 4; ++i) stage[i] = __builtin_amdgcn_raw_buffer_load_b128(rk, (int)load_off[i], 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) stage[4 + i] = __builtin_amdgcn_raw_buffer_load_b128(rv, (int)load_off[i], 0, 0);
    };
    auto store_block = [&](char* to) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<u32x4_t*>(to + k_off(load_row, load_chunk) + 16 * i * kRowBytes) = stage[i];
            *reinterpret_cast<u32x4_t*>(to + kBlockBytes + v_off(load_row, load_chunk) + 16 * i * kRowBytes) = stage[4 + i];
        }
    };

    // Where the lane reads.  Keys: row tile_row(n), chunk 2 s + hh.  Values, by transposing reads: a 16-lane group's lane 4 j + i
    // points at 4 columns of key row j, and lane x receives column x of the group's 16 in four keys.  Columns are taken in an
    // order that gives a lane 16 neighbouring ones of each 32: slots 8 q + 4 hh + e of the MFMA are columns 16 hh + 4 q + e.
    const int k_row = tile_row(n);
    const int k_read = k_row * kRowBytes + ((hh ^ (k_row & 15)) << 4);
    const int piece = 4 * ((lane >> 4) & 1) + (lane & 3), v_row = 8 * hh + ((lane >> 2) & 3);
    const int v_read = kBlockBytes + v_row * kRowBytes + ((v_row & 3) << 6) + (4 * (piece & 1) + (piece >> 1)) * 8;

    if (blk0 < blk1) {
        load_block(blk0);
        store_block(lds);
    }
    __syncthreads();
    for (int blk = blk0; blk < blk1; ++blk) {
        const char* const cur = lds + ((blk - blk0) & 1) * (2 * kBlockBytes);
        char* const next = lds + ((blk - blk0 + 1) & 1) * (2 * kBlockBytes);
        const bool more = blk + 1 < blk1;
        if (more) load_block(blk + 1);
        const int key0 = blk * kPrefillKeys;
        if (key0 < lim_last) {
            f32x16_t s[2];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                s[kt] = f32x16_t{};
#pragma unroll
                for (int st = 0; st < 8; ++st) {
                    const bf16x8_t a = *reinterpret_cast<const bf16x8_t*>(cur + (k_read ^ (st << 5)) + kt * 32 * kRowBytes);
                    s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qop[st], s[kt], 0, 0, 0);
                }
            }
            if (key0 + kPrefillKeys > lim_first) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        s[kt][i] = key0 + 32 * kt + 16 * (i >> 3) + 8 * hh + (i & 7) < lim ? s[kt][i] : kNegInf;
            }
            float mx = s[0][0];
#pragma unroll
            for (int i = 1; i < 32; ++i) mx = fmaxf(mx, s[i >> 4][i & 15]);
            float a, b;
            swap32(mx, a, b);
            mx = fmaxf(a, b) * prm.scale_log2;
            // The reference moves only when a row exceeds it by 2^8: then a weight is 2^8 at most, which neither the sums nor
            // bf16 mind, and most blocks need no rescaling of o.
            if (__ballot(mx > m + kSlackLog2) != 0) {
                const float to = fmaxf(m, mx), by = fast_exp2(m - to);
                m = to;
                l *= by;
#pragma unroll
                for (int c = 0; c < 4; ++c) o[c] *= by;
            }
            float p[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                p[i] = fast_exp2(__builtin_fmaf(s[i >> 4][i & 15], prm.scale_log2, -m));
                l += p[i];
            }
#pragma unroll
            for (int st = 0; st < 4; ++st) {
                const u32x4_t pw = {cvt_bf16(p[8 * st], p[8 * st + 1]), cvt_bf16(p[8 * st + 2], p[8 * st + 3]),
                                    cvt_bf16(p[8 * st + 4], p[8 * st + 5]), cvt_bf16(p[8 * st + 6], p[8 * st + 7])};
                const bf16x8_t pb = __builtin_bit_cast(bf16x8_t, pw);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const char* const at = cur + (v_read ^ (c << 6)) + st * 16 * kRowBytes;
                    const u32x2_t v0 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4v_t*)at));
                    const u32x2_t v1 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4v_t*)(at + 4 * kRowBytes)));
                    o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, u32x4_t{v0.x, v0.y, v1.x, v1.y}), pb, o[c], 0, 0, 0);
                }
            }
        }
        if (more) store_block(next);
        __syncthreads();
    }

    float la, lb;
    swap32(l, la, lb);
    l = la + lb;
    if (!row_on) return;
    // Column 32 c + 16 hh + i of the row is o[c][i].
    if (whole) {
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        uint16_t* const to = prm.out + q_row * kHeadDim + 16 * hh;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            uint32_t x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = cvt_bf16(o[c][2 * i] * inv, o[c][2 * i + 1] * inv);
            *reinterpret_cast<u32x4_t*>(to + 32 * c) = u32x4_t{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<u32x4_t*>(to + 32 * c + 8) = u32x4_t{x[4], x[5], x[6], x[7]};
        }
        if (prm.lse && hh == 0) prm.lse[q_row] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : kNegInf;
        return;
    }
    const int64_t slot_row = (int64_t)(w.slot + (head * w.s.tiles + tile) * w.parts + part) * prm.slot_rows + wave * kWaveRows + n;
    float* const to = prm.part_o + slot_row * kHeadDim + 16 * hh;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4_t*>(to + 32 * c + 4 * i) = f32x4_t{o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]};
    if (hh == 0) *reinterpret_cast<f32x2_t*>(prm.part_ml + slot_row * 2) = f32x2_t{m, l};
}

// The rows of tiles in several parts: blockIdx.x the tile among those, blockIdx.y a quarter of its rows, a wave per row at a
// time, two columns per lane.
constexpr int kMergeSplit = 4;
__global__ __launch_bounds__(256) void prefill_merge_kernel(PrefillParams prm) {
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
    const int head = blockIdx.x % (unsigned)prm.n_kv_heads;
    const PrefillWork w = find_work<true>(prm, (int)(blockIdx.x / (unsigned)prm.n_kv_heads), lane);
    if (!w.found) return;
    const int tile = w.index, part_blocks = prefill_part_blocks(w.s.blocks, w.parts);
    const int parts = (prefill_tile_blocks(w.s, tile, prm.group) + part_blocks - 1) / part_blocks;
    if (parts <= 1) return;
    const int rows = w.s.q * prm.group;
    const int64_t first_slot = w.slot + (int64_t)(head * w.s.tiles + tile) * w.parts;
    for (int i = blockIdx.y * (kPrefillRows / kMergeSplit) + wave; i < (int)(blockIdx.y + 1) * (kPrefillRows / kMergeSplit); i += 4) {
        const int row = tile * kPrefillRows + i;
        if (row >= rows) return;
        float top = kLowest;
        for (int s = lane; s < parts; s += 64) top = fmaxf(top, prm.part_ml[((first_slot + s) * prm.slot_rows + i) * 2]);
        top = wave_max(top);
        float l = 0.0f;
        f32x2_t o = {0.0f, 0.0f};
        for (int s0 = 0; s0 < parts; s0 += 64) {
            float by = 0.0f;
            if (s0 + lane < parts) {
                const f32x2_t ml = *reinterpret_cast<const f32x2_t*>(prm.part_ml + ((first_slot + s0 + lane) * prm.slot_rows + i) * 2);
                by = fast_exp2(ml.x - top);
                l += by * ml.y;
            }
            const int count = parts - s0 < 64 ? parts - s0 : 64;
            for (int s = 0; s < count; ++s) {
                const f32x2_t x = *reinterpret_cast<const f32x2_t*>(prm.part_o + ((first_slot + s0 + s) * prm.slot_rows + i) * kHeadDim + 2 * lane);
                o += x * lane_value(by, s);
            }
        }
        l = wave_sum(l);
        const int t = (int)((unsigned)row / (unsigned)prm.group);
        const int64_t q_row = (int64_t)(w.s.first + t) * prm.n_q_heads + head * prm.group + (row - t * prm.group);
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        reinterpret_cast<uint32_t*>(prm.out + q_row * kHeadDim)[lane] = cvt_bf16(o.x * inv, o.y * inv);
        if (prm.lse && lane == 0) prm.lse[q_row] = l > 0.0f ? (top + __builtin_amdgcn_logf(l)) * kLn2 : kNegInf;
    }
}

}  // namespace

hipError_t launch_prefill(const PrefillParams& prm, hipStream_t stream) {
    const long grid = prefill_grid(prm.total_q, prm.batch, prm.group, prm.n_kv_heads);
    hipError_t e = launch(prefill_kernel, dim3((unsigned)grid), 64 * kWaves, stream, prm);
    if (e != hipSuccess) return e;
    return launch(prefill_merge_kernel, dim3(kPrefillShares, kMergeSplit), 256, stream, prm);
}

}  // namespace xattn
