// Split-KV decode attention over a cache of 4 bits a value (xattn_decode_mx; the cache: xattn_mx.h).
//
//   s_j = scale <q, k_j>;  out = sum_j softmax(s)_j v_j;  lse = ln sum_j exp(s_j)      with k_j = 2^e code, v_j likewise, per block of 32 values
//
// The stream of keys is cut as xattn_decode's is, in whole tiles: a workgroup takes a piece of it for one KV head, its waves (mx_cut) a
// run of tiles each; a sequence that the waves cut among themselves is put together in LDS, one that pieces cut by the merge kernel.
//
// Bound by HBM with many keys: 64 sequences of 512 to 4096, 32 / 8 heads, 35.2 us; 16 of 16384 to 32768, 64 / 8 heads, 76 us (5.9 TB/s); 128 of
// 1028 to 8196, four tokens, 32 / 8 heads, 107 us (5.8 TB/s); with few by the dependent steps of two kernels, 9 to 10 us.  With 32 rows to a KV head by the issue of
// conversions, softmax and products (187 MB in 54 us, 3.8 TB/s in the kernel; vector units 62 %, matrix pipes 35 %), with 64, whose two workgroups a piece each convert all codes,
// twice per byte (100 MB in 54 us).  What the code owes to that:
//  - Codes become bf16 by a conversion with the scale, exactly, two to an instruction, and enter bf16 matrix products.  The scaled products
//    that take codes as they are would want q in 8 bits: in three parts of e4m3 their sums are off by 7e-5 of sum |q k|, these by 1e-7.
//  - Codes lie as the products' lanes hold them, so every load is 16 bytes a lane of one run of 1 KiB and nothing passes through LDS.
//  - A wave holds one tile, and where its K (V) has been used the next one's loads go out into its place; twelve waves a compute unit
//    wait for theirs in turn.  (Two tiles in registers and eight waves: 38.0 us in place of 35.5, 79.6 of 76.)
//  - Softmax weights enter the value product as two bf16, 16 bits.  With one, 8 bits, a call takes 2 to 3 % less, with 64 rows to a KV head 12 %.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "xattn_device.h"
#include "xattn_launch.h"
#include "xattn_matrix.h"
#include "xattn_mx.h"

namespace xattn {
namespace {

struct TileUnit {
    static __device__ __forceinline__ int positions(int raw) { return mx_positions(raw); }
    static __device__ __forceinline__ int stream(int raw, int seg_cost) { return raw > 0 ? mx_positions(raw) + seg_cost : 0; }
};

// How far, in powers of two, a score may exceed its row's reference before that moves.  (0: 64 sequences of 512 to 4096 35.2 -> 37.1 us, 32 rows to a KV
// head 45.9 -> 47.2; sums stay within 2^8 times a row's keys.)
constexpr float kSlack = 8.0f;

// Fixed work of a (piece, sequence) segment, in positions: a tile's.  (None / one / two / four tiles' worth: 64 sequences of 512 to 4096 37.2 / 35.2 / 36.3 /
// 37.0 us; 222 of 16 to 60000 66.3 / 65.2 / 64.5 / 67.1; 256 of up to 400 21.9 / 21.3 / 20.5 / 22.7.)
constexpr int kMxSegCost = kMxPositions;

// Lane (kb, n) = (lane / 16, lane % 16) of a tile: K's block kb of tokens 16 s + n; V's values 8 n .. 8 n + 7 of tokens 16 s + 4 kb + r.
struct MxTile {
    u32x4_t k[4], v[4], vs;
    uint32_t ks;
};
// From the tile at kt (vt); `on` false: from nowhere.  The loads go out either way, so that how many are on their way is always known and no wait is
// for more than it needs.
__device__ __forceinline__ void load_k(MxTile& t, const char* kt, bool on, int lane) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(kt, on ? kMxTileBytes : 0);
#pragma unroll
    for (int s = 0; s < 4; ++s) t.k[s] = load_b128_nt(r, lane * 16, 1024 * s);
    t.ks = __builtin_amdgcn_raw_buffer_load_b32(r, lane * 4, kMxCodeBytes, 2);
}
__device__ __forceinline__ void load_v(MxTile& t, const char* vt, bool on, int lane) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(vt, on ? kMxTileBytes : 0);
    t.vs = load_b128_nt(r, ((lane >> 4) * 4 + ((lane & 15) >> 2)) * 16, kMxCodeBytes);
#pragma unroll
    for (int s = 0; s < 4; ++s) t.v[s] = load_b128_nt(r, lane * 16, 1024 * s);
}

// The scale in byte i of four as a float's exponent.  The conversion takes no more of a scale than that; what stands in the other bits does not matter
// (masking them off: 24 instructions of a tile's 430).
__device__ __forceinline__ float scale_of(uint32_t bytes, int i) { return __uint_as_float(i == 3 ? bytes >> 1 : bytes << (23 - 8 * i)); }
// The codes in byte i of four, times the scale, as two bf16: exact.
template <int kByte>
__device__ __forceinline__ uint32_t unpack(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, kByte));
}

// One tile against kTiles times 16 query rows.  s[t][i][j] is the score of key 16 i + 4 kb + j for row n: a lane holds keys of one row, and the
// products of these with V take them from where they are.
template <int kTiles, typename NextK, typename NextV>
__device__ __forceinline__ void mx_tile(MatrixState (&st)[kTiles], const MxTile& r, const bf16x8_t (&qop)[kTiles][4], float scale_log2, int key0, int L,
                                        const int (&lim)[kTiles], int kb, NextK next_k, NextV next_v) {
    f32x4_t s[kTiles][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float scale = scale_of(r.ks, i);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) s[t][i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int step = 0; step < 4; ++step) {
            const uint32_t w = r.k[i][step];
            const u32x4_t a = {unpack<0>(w, scale), unpack<1>(w, scale), unpack<2>(w, scale), unpack<3>(w, scale)};
#pragma unroll
            for (int t = 0; t < kTiles; ++t) s[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), qop[t][step], s[t][i], 0, 0, 0);
        }
    }
    next_k();
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        if (__builtin_amdgcn_ballot_w64(key0 + kMxTileTokens > lim[t]) != 0) {      // only tiles that reach a limit
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[t][i][j] = key0 + 16 * i + 4 * kb + j < lim[t] ? s[t][i][j] : kNegInf;
        }
        float mx = kNegInf;
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, fmaxf(fmaxf(s[t][i][0], s[t][i][1]), fmaxf(s[t][i][2], s[t][i][3])));
        if (__builtin_amdgcn_ballot_w64(mx * scale_log2 > st[t].m + kSlack) != 0) {
            mx = kb_max(mx) * scale_log2;
            const bool moves = mx > st[t].m;
            const float alpha = moves ? fast_exp2(st[t].m - mx) : 1.0f;
            st[t].m = moves ? mx : st[t].m;
            st[t].l *= alpha;
#pragma unroll
            for (int e = 0; e < 8; ++e) st[t].o[e] *= alpha;
        }
        const float m_use = st[t].m == kNegInf ? 0.0f : st[t].m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s[t][i][j] = fast_exp2(__builtin_fmaf(s[t][i][j], scale_log2, -m_use));
            st[t].l += (s[t][i][0] + s[t][i][1]) + (s[t][i][2] + s[t][i][3]);
        }
    }
    // What stands behind the sequence's last key may be anything: its weight is 0, and with a scale of 2^-127 so is the product.
    u32x4_t vs = r.vs;
    if (key0 + kMxTileTokens > L) {
        auto known = [&](int i) {
            const int left = L - (key0 + 16 * i + 4 * kb);
            return left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << 8 * left) - 1;
        };
        vs = u32x4_t{vs.x & known(0), vs.y & known(1), vs.z & known(2), vs.w & known(3)};
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        u32x4_t hi[kTiles], lo[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x2_t p = {s[t][2 * h + (i >> 1)][2 * (i & 1)], s[t][2 * h + (i >> 1)][2 * (i & 1) + 1]};
                const bf16x2_t b = __builtin_convertvector(p, bf16x2_t);
                const f32x2_t rest = p - __builtin_convertvector(b, f32x2_t);
                hi[t][i] = __builtin_bit_cast(uint32_t, b);
                lo[t][i] = cvt_bf16(rest[0], rest[1]);
            }
        float scale[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) scale[i] = scale_of(vs[2 * h + (i >> 2)], i & 3);
        // A byte of the codes at a time, of eight tokens: two of the lane's eight values.
        auto two = [&](auto byte) {
            constexpr int kByte = decltype(byte)::value;
            uint32_t x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = unpack<kByte>(r.v[2 * h + (i >> 2)][i & 3], scale[i]);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                u32x4_t a;
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], half ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    f32x4_t& o = st[t].o[2 * kByte + half];
                    o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, hi[t]), o, 0, 0, 0);
                    o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, lo[t]), o, 0, 0, 0);
                }
            }
        };
        two(std::integral_constant<int, 0>());
        two(std::integral_constant<int, 1>());
        two(std::integral_constant<int, 2>());
        two(std::integral_constant<int, 3>());
        __builtin_amdgcn_sched_barrier(0);
    }
    next_v();
}

// A segment in flight: its Q operand, its limits and its first tile.  seg.j0 and j1 are positions of the stream, seg.L tokens.
template <int kTiles>
struct MxCtx {
    Segment seg;
    const char* kp;      // the segment's first tile
    const char* vp;
    bf16x8_t qop[kTiles][4];
    int lim[kTiles];     // first key that row n of the tile may not see
    MxTile first;
};
template <int kTiles>
__device__ __forceinline__ void mx_begin(MxCtx<kTiles>& c, const DecodeParams& prm, const Segment& seg, int lane) {
    const int kb = lane >> 4, n = lane & 15;
    c.seg = seg;
    const int64_t at = ((int64_t)(seg.j0 / kMxPositions) * prm.n_kv_heads + seg.kvh) * kMxTileBytes;
    c.kp = static_cast<const char*>(seg.kp) + at;
    c.vp = static_cast<const char*>(seg.vp) + at;
    load_k(c.first, c.kp, true, lane);
    load_v(c.first, c.vp, true, lane);
    // The kernel takes a positive scale: a negative one's sign and a zero go into Q.
    const uint32_t q_and = prm.scale_log2 == 0.0f ? 0u : 0xffffffffu, q_xor = prm.scale_log2 < 0.0f ? 0x80008000u : 0u;
    // Q through a descriptor over the sequence's rows: rows past n_rows lie past its end and read as zero.
    const int seq_rows = prm.q_len * prm.n_q_heads;
    const __amdgpu_buffer_rsrc_t rq = make_rsrc(prm.q + (long)seg.b * seq_rows * kHeadDim, (uint32_t)(seq_rows * kRowBytes));
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const bool row_ok = 16 * t + n < seg.n_rows;
        const int r = row_ok ? 16 * t + n : 0;
        const int qoff = (row_ok ? seq_row(prm, seg, r) : seq_rows) * kRowBytes + kb * 64;
#pragma unroll
        for (int step = 0; step < 4; ++step)
            c.qop[t][step] = __builtin_bit_cast(bf16x8_t, (__builtin_amdgcn_raw_buffer_load_b128(rq, qoff + 16 * step, 0, 0) & q_and) ^ q_xor);
        c.lim[t] = seg.L - prm.q_len + row_token(prm, seg.row0 + r) + 1;
    }
}

template <int kTiles>
__device__ __forceinline__ void mx_run(MatrixState (&st)[kTiles], MxCtx<kTiles>& c, const DecodeParams& prm, int lane) {
    const int kb = lane >> 4;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
#pragma unroll
        for (int e = 0; e < 8; ++e) st[t].o[e] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        st[t].m = kNegInf;
        st[t].l = 0.0f;
    }
    const int64_t step = (int64_t)prm.n_kv_heads * kMxTileBytes;
    const int first = c.seg.j0 / kMxPositions, n_tiles = c.seg.j1 / kMxPositions - first;
    const float scale_log2 = prm.scale_log2 == 0.0f ? 1.0f : fabsf(prm.scale_log2);
    auto k_at = [&](int i) { return c.kp + i * step; };
    auto v_at = [&](int i) { return c.vp + i * step; };
    auto tile = [&](int i, MxTile& r) {
        const bool more = i + 1 < n_tiles;
        mx_tile<kTiles>(st, r, c.qop, scale_log2, (first + i) * kMxTileTokens, c.seg.L, c.lim, kb,
                        [&] { load_k(r, k_at(i + 1), more, lane); __builtin_amdgcn_sched_barrier(0); }, [&] { load_v(r, v_at(i + 1), more, lane); });
    };
    for (int i = 0; i < n_tiles; ++i) tile(i, c.first);
}

// grid.x = workgroups of pieces times groups of R query rows, grid.z = KV heads.  (What the plan needs are arguments of their own: see
// split_decode_kernel, whose walk over a piece this one shares.)
template <int R, int kWaves>
__global__ __launch_bounds__(64 * kWaves, R == 16 ? 3 : 2) void decode_mx_kernel(const int32_t* __restrict__ kv_lens, const void* const* k_ptrs, const void* const* v_ptrs,
                                                                 int batch, int n_pieces, int min_piece, int few_pieces, int few_min,
                                                                 int xcd_skew, int grid_x, DecodeParams prm) {
    constexpr int kTiles = R / 16;
    constexpr int kStates = (kWaves - 1) * kTiles;
    __shared__ __attribute__((aligned(16))) char lds[kWaves * kLdsPerWave + kStates * kLdsPerState];
    const int lane = threadIdx.x & 63;
    const int part = uniform((int)(threadIdx.x >> 6));
    SeqWindow win;
    const WavePlan wp = wave_plan<TileUnit>(kv_lens, k_ptrs, v_ptrs, batch, n_pieces, min_piece, kMxSegCost, xcd_skew, FewPieces{few_pieces, few_min}, lane,
                                            &win, kWaves);
    const Plan& pl = wp.pl;
    const int bid = blockIdx.x, rows_total = prm.group * prm.q_len;
    const DecodeWork work = decode_work(pl, grid_x, 1, rows_total, R, bid, 0);
    const int p = work.piece, rows = work.rows;
    const int piece0 = piece_bound(pl, p), piece1 = piece_bound(pl, p + 1);
    const int sub = mx_part_positions(piece1 - piece0, kWaves), s0 = piece0 + part * sub, s1 = s0 + sub < piece1 ? s0 + sub : piece1;
    if (__builtin_expect(64 * (grid_x - 1 - bid) < batch && blockIdx.z == 0 && part == kWaves - 1, 0)) {
        for (int g = grid_x - 1 - bid; 64 * g < batch; g += grid_x)
            wave_write_meta<TileUnit>(wp, kv_lens, batch, prm.q_len * prm.n_q_heads, g, lane, prm.meta);
    }
    if (!work.any || piece0 >= piece1) return;      // the whole workgroup
    const bool active = s0 < s1;
    Walk walk;
    if (active) wave_locate<TileUnit>(wp, kv_lens, k_ptrs, v_ptrs, batch, s0, lane, &win, walk.b, walk.j);
    walk.remaining = uniform(s1 - s0);

    Segment seg;
    seg.kvh = blockIdx.z;
    seg.row0 = work.row0;
    seg.n_rows = rows_total - seg.row0 < rows ? rows_total - seg.row0 : rows;
    // The next (piece, sequence) intersection, in stream order; false when the piece is done.
    auto next_seg = [&](Segment& out, int& positions, auto first) {
        constexpr bool kFirst = decltype(first)::value;
        PieceSeg ps;
        int tokens = 0;
        auto len_of = [&](int b) {
            if constexpr (kFirst) tokens = window_len(win, kv_lens, b);
            else tokens = uniform(clamp_len(kv_lens[b]));
            return mx_positions(tokens);
        };
        if (!next_segment(walk, batch, pl.seg_cost, len_of, ps)) return false;
        out = seg;
        out.b = uniform(ps.b);
        out.kp = kFirst ? window_ptr(win, win.k, k_ptrs, out.b) : uniform(k_ptrs[out.b]);
        out.vp = kFirst ? window_ptr(win, win.v, v_ptrs, out.b) : uniform(v_ptrs[out.b]);
        out.L = uniform(tokens);
        out.j0 = uniform(ps.j0);
        out.j1 = uniform(ps.j1);
        out.slot = uniform(p) + out.b;
        out.whole = uniform(ps.whole);
        positions = uniform(ps.L);
        return true;
    };
    char* const lds_wave = lds + part * kLdsPerWave;
    auto run_piece = [&](auto tiles) {
        constexpr int kT = decltype(tiles)::value;
        auto state_of = [&](int of_part, int t) { return lds + kWaves * kLdsPerWave + ((of_part - 1) * kT + t) * kLdsPerState; };
        MatrixState st[kT];
        MxCtx<kT> cur;
        int positions = 0;
        auto put = [&] {
#pragma unroll
            for (int t = 0; t < kT; ++t) state_put(st[t], state_of(part, t), lane);
        };
        bool have = false;
        if (active) {
            Segment first;
            have = uniform(next_seg(first, positions, std::true_type())) != 0;
            if (have) mx_begin(cur, prm, first, lane);
        }
        if (have) {
            for (;;) {
                mx_run<kT>(st, cur, prm, lane);
                Segment nxt_seg;
                int nxt_positions;
                if (uniform(next_seg(nxt_seg, nxt_positions, std::false_type())) == 0) break;
                MxCtx<kT> nxt;
                mx_begin(nxt, prm, nxt_seg, lane);     // its loads go out before cur's stores
                if (part > 0 && cur.seg.j0 > 0) {
                    put();
                } else {
#pragma unroll
                    for (int t = 0; t < kT; ++t) matrix_finish<true>(st[t], cur.seg, t, prm, lane, lds_wave);
                }
                cur = nxt;
                positions = nxt_positions;
            }
        }
        // The last segment: what the wave before began goes to LDS, what this wave begins is put together there.
        PartRun run = {false, 0, false};
        if (have) run = part_run(part, cur.seg.j0, cur.seg.j1, positions, piece1 - s1, sub);
        if (have && run.prev) put();
        __syncthreads();
        if (!have || run.prev) return;
        for (int q = part + 1; q <= part + run.next; ++q)
#pragma unroll
            for (int t = 0; t < kT; ++t) state_add(st[t], state_of(q, t), lane);
        cur.seg.whole = cur.seg.j0 == 0 && run.ends;
#pragma unroll
        for (int t = 0; t < kT; ++t) matrix_finish<false>(st[t], cur.seg, t, prm, lane, lds_wave);
    };
    if (kTiles == 2 && rows == 16) run_piece(std::integral_constant<int, 1>());
    else run_piece(std::integral_constant<int, kTiles>());
}

template <int R, int kWaves>
hipError_t launch_with(const DecodeParams& prm, hipStream_t stream) {
    const int grid_x = decode_grid_x(prm.n_pieces, 1, prm.group * prm.q_len, R);
    return launch(decode_mx_kernel<R, kWaves>, dim3((unsigned)grid_x, 1, (unsigned)prm.n_kv_heads), 64 * kWaves, stream, prm.kv_lens, prm.k_ptrs, prm.v_ptrs,
                  prm.batch, prm.n_pieces, prm.min_piece_tokens, prm.few.pieces, prm.few.min_piece, prm.xcd_skew, grid_x, prm);
}

}  // namespace

hipError_t launch_decode_mx(const DecodeParams& prm, const MxCut& cut, hipStream_t stream) {
    hipError_t e;
    if (cut.rows == 16) e = cut.waves == 12 ? launch_with<16, 12>(prm, stream) : launch_with<16, 4>(prm, stream);
    else e = cut.waves == 8 ? launch_with<32, 8>(prm, stream) : launch_with<32, 4>(prm, stream);
    return e != hipSuccess ? e : launch_decode_merge(prm, stream);
}

}  // namespace xattn
