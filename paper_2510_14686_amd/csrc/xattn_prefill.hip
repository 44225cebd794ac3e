// Attention of the new tokens of a batch of prompts (xattn_prefill): causal, grouped heads, sequences of different lengths
// packed one behind the other, keys and values in per-sequence ranges.
//
//   out = softmax(scale Q K^T + causal mask) V in one pass over the keys: with a running reference m and sum l per row,
//   a block of keys adds exp2(s - m) to l and exp2(s - m) V to o, both rescaled when m moves.
//
// The rows of a tile are (new token, query head of the group) pairs of one KV head, so that K and V are read once for the whole
// group, and a tile of a short sequence holds all its rows.
//
// Many new tokens are bound by the matrix pipes at the clock that the card's power leaves them: one prompt of 16001, 32 / 8 heads,
// 1.85 to 1.95 ms, 1080 to 1140 TFLOP/s, against the 1360 of a bf16 matrix product of 16384 in a library; the pipes are busy 64 % of the
// time at 1.6 GHz.  Few are bound by reading the keys: 64 sequences of 4096 and one new token each, 171 us, 6.3 TB/s.  A handful of
// short sequences takes 9 us of finding the work and a few blocks' latencies, and 2 us of merge.
//   A wave has 32 rows, so that its scores, weights and sums need 200 registers and two waves share a SIMD, one in its softmax while
// the other multiplies.  64 rows a wave halve what is read from LDS, but need 420 registers: with one wave per SIMD, the two halves of
// its rows interleaved, the prompt of 16001 takes 2200 us where this takes 1845, and one of 2048 77 us where this takes 49.
//   32 keys at a time make the weights beside the next scores: with 64 the two sets of scores do not fit, and in turn, without
// the overlap, 2246 us where this took 2004 then.
//   Weights enter the second product as one bf16 each, off by 2^-8 of it at most, as the values of V themselves may be.  On request (kExact)
// as three bf16 parts, all 24 bits of them: the prompt of 16001 takes 1.72 times as long, 64 sequences of 4096 and one new token each 172 us
// instead of 170, a prompt of 1000 among decoding sequences 138 instead of 122, four short sequences 12.9 instead of 10.8 (the products
// are a part of each step's latency there).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

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
constexpr int kHalfBytes = kBlockBytes / 2;
constexpr int kAhead = 4;                             // steps of the next scores ahead of the row maxima
constexpr float kSlackLog2 = 8.0f;                    // how far a row's maximum may exceed its reference

// ------------------------------------------------------------------------------------------------ a workgroup's work
struct PrefillWork {
    PrefillSeq s;
    int b, parts, index;      // index: of the work among the sequence's (per KV head)
    int slot, split;          // of the sequence: first slot, tiles of earlier sequences that are in several parts (per KV head)
    int splits;               // tiles in several parts, per KV head
    const char *k, *v;        // the sequence's ranges
    bool found;
};
__device__ __forceinline__ PrefillSeq load_seq(const PrefillParams& prm, int b) {
    const bool in = b < prm.batch;
    const int i = in ? b : 0;
    const int start = prm.q_starts[i], end = prm.q_starts[i + 1], kv = prm.kv_lens[i];
    return prefill_seq(in ? start : 0, in ? end : 0, in ? kv : 0, prm.total_q, prm.group);
}
struct Amounts {
    int work, slots, split;
};
__device__ __forceinline__ Amounts amounts_of(const PrefillSeq& s, int share) {
    const int parts = prefill_parts(s.blocks, share);
    return Amounts{s.tiles * parts, parts > 1 ? s.tiles * parts : 0, parts > 1 ? s.tiles : 0};
}
// What work number j (per KV head) is.  Lane l has the sequences l << lg ..; one scan finds j's lane, another the sequence among the
// lane's.  Up to 64 sequences, one per lane, are taken in the order of their lengths, longest first: workgroups start in the order of their
// numbers, and long work that starts late ends late.
__device__ __forceinline__ PrefillWork find_work(const PrefillParams& prm, int j, int lane) {
    const int lg = prm.batch <= 64 ? 0 : 26 - __builtin_clz((unsigned)(prm.batch - 1));
    const int chunk = 1 << lg;
    PrefillWork r;
    PrefillSeq s = load_seq(prm, lane << lg);
    float cost = prefill_cost(s);
    Amounts mine;
    int b = lane << lg, share;
    u32x2_t k = {0u, 0u}, v = {0u, 0u};
    if (chunk == 1) {
        const int i = lane < prm.batch ? lane : 0;
        k = *reinterpret_cast<const u32x2_t*>(prm.k_ptrs + i);
        v = *reinterpret_cast<const u32x2_t*>(prm.v_ptrs + i);
        share = prefill_share(wave_sum(cost) * (float)prm.n_kv_heads);
        const int key = s.tiles > 0 ? s.blocks : -1;
        int before = 0;
        for (int l = 0; l < prm.batch; ++l) {
            const int other = __builtin_amdgcn_readlane(key, l);
            before += other > key || (other == key && l < lane);
        }
        if (lane >= prm.batch) before = lane;
        // lane `before` becomes this one's
        auto to = [&](int x) { return __builtin_amdgcn_ds_permute(before * 4, x); };
        s = PrefillSeq{to(s.first), to(s.q), to(s.kv), to(s.tiles), to(s.blocks)};
        b = to(b);
        mine = amounts_of(s, share);
    } else {
        for (int i = 1; i < chunk; ++i) cost += prefill_cost(load_seq(prm, (lane << lg) + i));
        share = prefill_share(wave_sum(cost) * (float)prm.n_kv_heads);
        mine = Amounts{0, 0, 0};
        for (int i = 0; i < chunk; ++i) {
            const Amounts a = amounts_of(load_seq(prm, (lane << lg) + i), share);
            mine.work += a.work;
            mine.slots += a.slots;
            mine.split += a.split;
        }
    }
    int work = wave_incl_scan_i(mine.work), slots = wave_incl_scan_i(mine.slots), split = wave_incl_scan_i(mine.split);
    r.splits = __builtin_amdgcn_readlane(split, 63);
    // Where all work is on its way at once, two workgroups to a compute unit, the later half comes in reverse: long work shares a
    // compute unit with short work.
    const int all = __builtin_amdgcn_readlane(work, 63), half = (all + 1) / 2;
    if (all * prm.n_kv_heads <= kPrefillShares && j >= half && j < all) j = all - 1 - (j - half);
    unsigned long long hit = __ballot(j >= work - mine.work && j < work);
    r.found = hit != 0;
    int at = hit ? __builtin_ctzll(hit) : 0;
    r.index = j - __builtin_amdgcn_readlane(work - mine.work, at);
    r.slot = __builtin_amdgcn_readlane(slots - mine.slots, at);
    r.split = __builtin_amdgcn_readlane(split - mine.split, at);
    if (chunk > 1) {
        const int first = at << lg;
        b = first + lane;
        s = load_seq(prm, lane < chunk ? b : prm.batch);
        mine = amounts_of(s, share);
        work = wave_incl_scan_i(mine.work);
        slots = wave_incl_scan_i(mine.slots);
        split = wave_incl_scan_i(mine.split);
        hit = __ballot(r.index >= work - mine.work && r.index < work);
        at = hit ? __builtin_ctzll(hit) : 0;
        r.index -= __builtin_amdgcn_readlane(work - mine.work, at);
        r.slot += __builtin_amdgcn_readlane(slots - mine.slots, at);
        r.split += __builtin_amdgcn_readlane(split - mine.split, at);
    }
    r.slot *= prm.n_kv_heads;
    r.b = __builtin_amdgcn_readlane(b, at);
    r.s.first = __builtin_amdgcn_readlane(s.first, at);
    r.s.q = __builtin_amdgcn_readlane(s.q, at);
    r.s.kv = __builtin_amdgcn_readlane(s.kv, at);
    r.s.tiles = __builtin_amdgcn_readlane(s.tiles, at);
    r.s.blocks = __builtin_amdgcn_readlane(s.blocks, at);
    r.parts = prefill_parts(r.s.blocks, share);
    if (chunk == 1) {
        auto lane_ptr = [&](const u32x2_t& x) {
            return reinterpret_cast<const char*>((uintptr_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)x.x, r.b) |
                                                             (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)x.y, r.b) << 32));
        };
        r.k = lane_ptr(k);
        r.v = lane_ptr(v);
    } else if (r.found) {
        r.k = static_cast<const char*>(uniform(prm.k_ptrs[r.b]));
        r.v = static_cast<const char*>(uniform(prm.v_ptrs[r.b]));
    }
    return r;
}

// For the merge kernel, in the workspace: how many tiles are in several parts, and of each where its rows and its parts are.
struct SplitTile {
    int first, q;             // the sequence's packed rows
    int tile, head, slot, parts;
    int unused[2];
};
__device__ __forceinline__ int* split_count(const PrefillParams& prm) { return prm.table; }
__device__ __forceinline__ SplitTile* split_tiles(const PrefillParams& prm) { return reinterpret_cast<SplitTile*>(prm.table + 8); }

// ------------------------------------------------------------------------------------------------ blocks
// Block at key0 of K or V, loaded into LDS without passing through registers: a wave's load fills 1024 consecutive bytes, four rows,
// lane l the l-th 16 bytes.  The descriptor ends with the sequence, so rows behind it (which an xTensor range need not have mapped) read
// as zero, and begins with the block, so a sequence may be larger than 32-bit offsets reach.
__device__ __forceinline__ u32x4_t block_rsrc(const char* head, int key0, int kv, int row_bytes) {
    const int keys = kv - key0 < kPrefillKeys ? kv - key0 : kPrefillKeys;
    const uint64_t base = (uint64_t)(uintptr_t)(head + (int64_t)key0 * row_bytes);
    return u32x4_t{(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu, keys > 0 ? (uint32_t)((keys - 1) * row_bytes + kRowBytes) : 0u, 0x00020000u};
}
// The loads are assembly because the compiler would wait for all of them ahead of every read of LDS; wait_loads() and the barrier
// behind it are what makes a block visible.  m0 is the address in LDS; a wait state goes between its write and the load.
// kOnce: non-temporal.
template <bool kOnce>
__device__ __forceinline__ void load_lds(u32x4_t rsrc, uint32_t lds_addr, uint32_t voff, uint32_t soff) {
    if constexpr (kOnce) asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds" : : "{m0}"(lds_addr), "v"(voff), "s"(rsrc), "s"(soff) : "memory");
    else asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "{m0}"(lds_addr), "v"(voff), "s"(rsrc), "s"(soff) : "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// In LDS a row is 256 bytes.  K: chunk c of row r sits at c ^ (r & 15), so that the 16 rows that 16 lanes read a chunk
// of are in different banks; V: 64-byte piece x of row r at x ^ (r & 3), for the four rows of a transposing read.

// S^T = K Q^T by 32x32x16 MFMA: lane (hh, n) = (lane / 32, lane % 32) gives chunk 8 hh .. of key row n and of query row n, and
// has, of query row n, the keys at rows 8 (i / 4) + 4 hh + i % 4 in accumulator i.  Row x of the operand is key tile_row(x) of the
// tile, which makes them the keys 16 (i / 8) + 8 hh + i % 8: accumulators 8 s .. 8 s + 7, as bf16, are the operand of the
// 16 keys of step s in O^T += V^T P^T.
__device__ __forceinline__ int tile_row(int x) { return (x & ~12) | ((x & 4) << 1) | ((x & 8) >> 1); }

template <bool kExact>
__global__ __launch_bounds__(64 * kWaves, 2) void prefill_kernel(PrefillParams prm) {
    __shared__ __attribute__((aligned(1024))) char lds[2 * 2 * kBlockBytes];      // K, K, V, V
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int head = uniform((int)(blockIdx.x % (unsigned)prm.n_kv_heads));
    const PrefillWork w = find_work(prm, uniform((int)(blockIdx.x / (unsigned)prm.n_kv_heads)), lane);
    if (blockIdx.x == 0 && tid == 0) *split_count(prm) = w.splits * prm.n_kv_heads;
    if (!w.found) return;
    // Later tiles see more keys: first.
    const int tile = uniform(w.s.tiles - 1 - w.index / w.parts), part = uniform(w.index % w.parts);
    const int part_blocks = uniform(prefill_part_blocks(w.s.blocks, w.parts)), blocks = uniform(prefill_tile_blocks(w.s, tile, prm.group));
    const int blk0 = part * part_blocks, blk1 = blk0 + part_blocks < blocks ? blk0 + part_blocks : blocks;
    if (part > 0 && blk0 >= blk1) return;
    const bool whole = blocks <= part_blocks;
    const int first_slot = w.slot + (head * w.s.tiles + tile) * w.parts;
    if (w.parts > 1 && part == 0 && tid == 0)
        split_tiles(prm)[(w.split + tile) * prm.n_kv_heads + head] =
            SplitTile{w.s.first, w.s.q, tile, head, first_slot, whole ? 1 : (blocks + part_blocks - 1) / part_blocks, {0, 0}};

    const int row_bytes = prm.n_kv_heads * kRowBytes;
    const char* const k_head = static_cast<const char*>(uniform(static_cast<const void*>(w.k + head * kRowBytes)));
    const char* const v_head = static_cast<const char*>(uniform(static_cast<const void*>(w.v + head * kRowBytes)));
    const int kv = uniform(w.s.kv);

    // This lane's query row.
    const int rows = w.s.q * prm.group, wave_row = tile * kPrefillRows + wave * kWaveRows, row = wave_row + n;
    const bool wave_on = wave_row < rows, row_on = row < rows;
    const int t = (int)((unsigned)row / (unsigned)prm.group), h = head * prm.group + (row - t * prm.group);
    const int64_t q_row = (int64_t)(w.s.first + t) * prm.n_q_heads + h;
    const int lim = row_on ? prefill_visible(w.s, t) : 0;
    const int last_row = wave_row + kWaveRows < rows ? wave_row + kWaveRows - 1 : rows - 1;
    const int lim_first = uniform(prefill_visible(w.s, (int)((unsigned)wave_row / (unsigned)prm.group)));
    const int lim_last = uniform(wave_on ? prefill_visible(w.s, (int)((unsigned)last_row / (unsigned)prm.group)) : 0);

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

    // This wave's loads of a block: rows 16 wave + 4 i + lane / 16, i < 4, of K and of V.
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    const int load_row = 16 * wave + (lane >> 4), load_chunk = lane & 15;
    uint32_t k_load[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) k_load[i] = (uint32_t)((load_row + 4 * i) * row_bytes + ((load_chunk ^ ((load_row + 4 * i) & 15)) << 4));
    const uint32_t v_load = (uint32_t)(load_row * row_bytes + ((load_chunk ^ ((load_row & 3) << 2)) << 4));
    // K of the part's block j is in buffer j & 1.  V comes and goes by half blocks of 32 keys, half g = 2 j + h to place g & 3; a load
    // is of two, from an odd one on.
    // What a single tile reads, as of a decoding sequence, is read once: non-temporal (64 of 4096 keys, one new token, 8 KV heads 196 ->
    // 173 us); K and V of several tiles are to stay in the L2.
    const bool once = uniform(w.s.tiles) == 1;
    const int n_blocks = blk1 - blk0, first_key = blk0 * kPrefillKeys;
    auto load_k_as = [&](auto as, int j) {
        const u32x4_t rsrc = block_rsrc(k_head, (blk0 + j) * kPrefillKeys, kv, row_bytes);
        const uint32_t to = lds0 + (j & 1) * kBlockBytes + wave * 4096;
#pragma unroll
        for (int i = 0; i < 4; ++i) load_lds<decltype(as)::value>(rsrc, to + i * 1024, k_load[i], 0u);
    };
    auto load_v_as = [&](auto as, int g, int place) {
        const u32x4_t rsrc = block_rsrc(v_head, blk0 * kPrefillKeys + g * 32, kv, row_bytes);
        const uint32_t to = lds0 + 2 * kBlockBytes + (place & 3) * kHalfBytes + (wave & 1) * 4096;
#pragma unroll
        for (int i = 0; i < 4; ++i) load_lds<decltype(as)::value>(rsrc, to + i * 1024, v_load, (uint32_t)(4 * i * row_bytes));
    };
    auto load_next = [&](auto as, int j) {      // block j of K, and halves 2 j - 1 and 2 j of V
        if (j < n_blocks) load_k_as(as, j);
        load_v_as(as, 2 * j - 1, 2 * j - 1 + (wave >> 1));
    };

    // Where the lane reads.  Keys: row tile_row(n), chunk 2 s + hh.  Values, by transposing reads: a 16-lane group's lane 4 j + i
    // points at 4 columns of key row j, and lane x receives column x of the group's 16 in four keys.  Columns are taken in an
    // order that gives a lane 16 neighbouring ones of each 32: slots 8 q + 4 hh + e of the MFMA are columns 16 hh + 4 q + e.
    const int k_row = tile_row(n);
    const int k_read = k_row * kRowBytes + ((hh ^ (k_row & 15)) << 4);
    const int piece = 4 * ((lane >> 4) & 1) + (lane & 3), v_row = 8 * hh + ((lane >> 2) & 3);
    const int v_read = 2 * kBlockBytes + v_row * kRowBytes + ((v_row & 3) << 6) + (4 * (piece & 1) + (piece >> 1)) * 8;
    // (The addresses of all reads of a half, but for what the half adds to them, a constant in each of the four forms of it.)
    const char *k_at[8], *v_at[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) k_at[i] = lds + (k_read ^ (i << 5));
#pragma unroll
    for (int c = 0; c < 4; ++c) v_at[c] = lds + (v_read ^ (c << 6));

    // The scores of half kG (of 4 in LDS), in eight steps.
    auto key_operand = [&](auto half, int i) {
        constexpr int kG = decltype(half)::value & 3;
        return *reinterpret_cast<const bf16x8_t*>(k_at[i] + (kG >> 1) * kBlockBytes + (kG & 1) * kHalfBytes);
    };
    auto score_step = [&](f32x16_t& s, const bf16x8_t& a, int i) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qop[i], i == 0 ? f32x16_t{} : s, 0, 0, 0);
    };
    // Columns 32 c .. 32 c + 31 of keys 16 st .. 16 st + 15 of a half.
    auto value_operand = [&](auto half, int st, int c) {
        const char* const at = v_at[c] + decltype(half)::value * kHalfBytes + st * 16 * kRowBytes;
        const u32x2_t v0 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4v_t*)at));
        const u32x2_t v1 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4v_t*)(at + 4 * kRowBytes)));
        return __builtin_bit_cast(bf16x8_t, u32x4_t{v0.x, v0.y, v1.x, v1.y});
    };
    // The scores of the half from key0 on become weights, while the matrix pipe works on those of the half after it, and add its values up.
    auto half = [&](auto which, f32x16_t& s, f32x16_t& next, int key0) {
        constexpr int kG = decltype(which)::value;
        bf16x8_t ka[8], va[2][4];
        if (key0 + 32 > lim_first) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = key0 + 16 * (i >> 3) + 8 * hh + (i & 7) < lim ? s[i] : kNegInf;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) ka[i] = key_operand(std::integral_constant<int, kG + 1>(), i);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) score_step(next, ka[i], i);
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
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
#pragma unroll
        for (int c = 0; c < 4; ++c) va[0][c] = value_operand(which, 0, c);
#pragma unroll
        for (int i = kAhead; i < 8; ++i) score_step(next, ka[i], i);
        float p[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            p[i] = fast_exp2(__builtin_fmaf(s[i], prm.scale_log2, -m));
            l += p[i];
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) va[1][c] = value_operand(which, 1, c);
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const bf16x8_t pb = __builtin_bit_cast(bf16x8_t, u32x4_t{cvt_bf16(p[8 * st], p[8 * st + 1]), cvt_bf16(p[8 * st + 2], p[8 * st + 3]),
                                                                     cvt_bf16(p[8 * st + 4], p[8 * st + 5]), cvt_bf16(p[8 * st + 6], p[8 * st + 7])});
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[st][c], pb, o[c], 0, 0, 0);
            if constexpr (kExact) {
                // What bf16 leaves of the weights, then what it leaves of that.
                u32x4_t part = __builtin_bit_cast(u32x4_t, pb);
#pragma unroll
                for (int again = 0; again < 2; ++again) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float &a = p[8 * st + 2 * i], &b = p[8 * st + 2 * i + 1];
                        a -= bf16_lo(part[i]);
                        b -= bf16_hi(part[i]);
                        part[i] = cvt_bf16(a, b);
                    }
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[st][c], __builtin_bit_cast(bf16x8_t, part), o[c], 0, 0, 0);
                }
            }
        }
    };

    // Round j: the weights of half 2 j beside the scores of half 2 j + 1, then the weights of that beside the scores of 2 j + 2 (behind the
    // last one, of whatever the buffer holds: they are not used).  What the second half of the round and the first of the next one read is
    // loaded meanwhile, block j + 1 of K and halves 2 j + 1 and 2 j + 2 of V, into buffers that were last read ahead of the barrier.  A wave
    // whose rows see no more keys goes on with its share of the loads and the barriers.
    if (n_blocks > 0) {
        load_k_as(std::false_type(), 0);
        if (wave < 2) load_v_as(std::false_type(), 0, 0);      // one half, by two waves
        wait_loads();
        __syncthreads();
        load_next(std::false_type(), 1);
        f32x16_t s0, s1;
#pragma unroll
        for (int i = 0; i < 8; ++i) score_step(s0, key_operand(std::integral_constant<int, 0>(), i), i);
        auto round = [&](auto odd, int j) {
            constexpr int kG = 2 * decltype(odd)::value;
            const int key0 = first_key + j * kPrefillKeys;
            if (key0 < lim_last) half(std::integral_constant<int, kG>(), s0, s1, key0);
            wait_loads();
            __syncthreads();
            if (j + 1 < n_blocks) {
                if (once) load_next(std::true_type(), j + 2);
                else load_next(std::false_type(), j + 2);
            }
            if (key0 + 32 < lim_last) half(std::integral_constant<int, kG + 1>(), s1, s0, key0 + 32);
        };
        for (int j = 0;;) {
            round(std::integral_constant<int, 0>(), j);
            if (++j >= n_blocks) break;
            round(std::integral_constant<int, 1>(), j);
            if (++j >= n_blocks) break;
        }
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
    const int64_t slot_row = (int64_t)(first_slot + part) * prm.slot_rows + wave * kWaveRows + n;
    float* const to = prm.part_o + slot_row * kHeadDim + 16 * hh;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4_t*>(to + 32 * c + 4 * i) = f32x4_t{o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]};
    if (hh == 0) *reinterpret_cast<f32x2_t*>(prm.part_ml + slot_row * 2) = f32x2_t{m, l};
}

// The rows of tiles in several parts.  A workgroup takes 16 / kWavesPerRow rows at a time, so many that all workgroups have some: few
// tiles are in many parts each, whose rows several waves put together.  A lane holds two columns.
constexpr int kMergeWaves = 16, kMergeGroups = 512;
__global__ __launch_bounds__(64 * kMergeWaves) void prefill_merge_kernel(PrefillParams prm) {
    __shared__ f32x2_t sums[kMergeWaves][64];
    __shared__ f32x2_t tops[kMergeWaves];
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
    const int tiles = uniform(*split_count(prm));
    if (tiles == 0) return;
    int per_row = 1;          // waves
    while (per_row < kMergeWaves && tiles * (kPrefillRows / kMergeWaves) * per_row * 2 <= kMergeGroups) per_row *= 2;
    const int rows_at_once = kMergeWaves / per_row, steps = kPrefillRows / rows_at_once;
    for (int unit = blockIdx.x; unit < tiles * steps; unit += kMergeGroups) {
        const SplitTile w = split_tiles(prm)[unit % tiles];      // the tiles' first rows first: some tiles have no others
        const int i = unit / tiles * rows_at_once + wave / per_row, row = w.tile * kPrefillRows + i, mine = wave % per_row;
        // (Of bounds in q_starts that do not ascend, an entry may not have been written: nothing outside the buffers then.)
        const bool known = w.parts > 1 && w.parts <= kPrefillSlots && (unsigned)w.slot <= (unsigned)(kPrefillSlots - w.parts) && (unsigned)w.head < (unsigned)prm.n_kv_heads &&
                           (unsigned)w.first <= (unsigned)prm.total_q && (unsigned)w.q <= (unsigned)(prm.total_q - w.first) && (unsigned)w.tile < 1u << 24;
        const bool on = known && row < w.q * prm.group;
        float top = kLowest, l = 0.0f;
        f32x2_t o = {0.0f, 0.0f};
        if (on) {
            // Parts mine, mine + per_row, ..., 64 of them at a time.
            for (int s0 = mine; s0 < w.parts; s0 += 64 * per_row) {
                const int at = s0 + lane * per_row;
                f32x2_t ml = {kLowest, 0.0f};
                if (at < w.parts) ml = *reinterpret_cast<const f32x2_t*>(prm.part_ml + ((int64_t)(w.slot + at) * prm.slot_rows + i) * 2);
                const float higher = fmaxf(top, wave_max(ml.x)), by = fast_exp2(ml.x - higher), old = fast_exp2(top - higher);
                top = higher;
                l = l * old + by * ml.y;
                o *= old;
                const int count = (w.parts - s0 + per_row - 1) / per_row < 64 ? (w.parts - s0 + per_row - 1) / per_row : 64;
                const float* from = prm.part_o + ((int64_t)(w.slot + s0) * prm.slot_rows + i) * kHeadDim + 2 * lane;
                const int64_t stride = (int64_t)per_row * prm.slot_rows * kHeadDim;
                for (int s = 0; s < count; s += 8) {
                    f32x2_t x[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u) x[u] = *reinterpret_cast<const f32x2_t*>(from + (s + u < count ? s + u : s) * stride);
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        const float weight = s + u < count ? lane_value(by, s + u) : 0.0f;
                        o.x = __builtin_fmaf(x[u].x, weight, o.x);
                        o.y = __builtin_fmaf(x[u].y, weight, o.y);
                    }
                }
            }
            l = wave_sum(l);
        }
        if (per_row > 1) {
            __syncthreads();      // the last unit's are read
            sums[wave][lane] = o;
            if (lane == 0) tops[wave] = f32x2_t{top, l};
            __syncthreads();
            if (mine == 0) {
                float m = top;
                for (int u = 1; u < per_row; ++u) m = fmaxf(m, tops[wave + u].x);
                const float own = fast_exp2(top - m);
                o *= own;
                l *= own;
                top = m;
                for (int u = 1; u < per_row; ++u) {
                    const f32x2_t ml = tops[wave + u], x = sums[wave + u][lane];
                    const float by = fast_exp2(ml.x - m);
                    l += by * ml.y;
                    o += x * by;
                }
            }
        }
        if (!on || mine != 0) continue;
        const int t = (int)((unsigned)row / (unsigned)prm.group);
        const int64_t q_row = (int64_t)(w.first + t) * prm.n_q_heads + w.head * prm.group + (row - t * prm.group);
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        reinterpret_cast<uint32_t*>(prm.out + q_row * kHeadDim)[lane] = cvt_bf16(o.x * inv, o.y * inv);
        if (prm.lse && lane == 0) prm.lse[q_row] = l > 0.0f ? (top + __builtin_amdgcn_logf(l)) * kLn2 : kNegInf;
    }
}

}  // namespace

hipError_t launch_prefill(const PrefillParams& prm, hipStream_t stream) {
    const long grid = prefill_grid(prm.total_q, prm.batch, prm.group, prm.n_kv_heads);
    hipError_t e = launch(prm.exact ? prefill_kernel<true> : prefill_kernel<false>, dim3((unsigned)grid), 64 * kWaves, stream, prm);
    if (e != hipSuccess) return e;
    return launch(prefill_merge_kernel, dim3(kMergeGroups), 64 * kMergeWaves, stream, prm);
}

}  // namespace xattn
