// What the split-KV decode kernels on matrix instructions share: a wave's segment, the running state of 16 query rows, and where that
// goes: results or partial results in memory, or another wave's state by way of LDS.
#ifndef XATTN_MATRIX_H_
#define XATTN_MATRIX_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "xattn_device.h"
#include "xattn_kernels.h"

namespace xattn {
namespace {

// One (piece, sequence) intersection as seen by one wave.
struct Segment {
    int b, L;            // sequence and its length
    int j0, j1;          // keys [j0, j1) of the sequence
    const void* kp;      // the sequence's K and V ranges
    const void* vp;
    int slot;            // partial-result slot (piece + sequence index)
    bool whole;          // the segment is the whole sequence: write the final result
    int kvh;             // this wave's KV head
    int row0, n_rows;    // query rows [row0, row0 + n_rows) of the head's group * q_len rows
};

// Lane (kb, n) = (lane / 16, lane % 16).
struct MatrixState {
    f32x4_t o[8];     // O^T tiles: o[e][j] = column 8*(4*kb + j) + e of row n
    float m, l;       // row n: running max (all kb groups agree), this lane's share of the running sum
};

// Row r of the segment's rows <-> (token t, head kvh*G + g).  r / G as a product with 1 / G: (r + 1/2) / G is
// at least 1 / (2 G) >= 2^-7 away from an integer (G <= 64), far more than the product's rounding.
__device__ __forceinline__ int row_token(const DecodeParams& prm, int r) { return (int)(((float)r + 0.5f) * prm.inv_group); }
__device__ __forceinline__ int seq_row(const DecodeParams& prm, const Segment& seg, int r) {      // row within the sequence
    const int rr = seg.row0 + r;
    const int t = row_token(prm, rr);
    return t * prm.n_q_heads + seg.kvh * prm.group + (rr - t * prm.group);
}

// Stores the 16 rows of tile t of the segment; rows past the last get an offset past the descriptor's end,
// and their stores are dropped.
constexpr uint32_t kPastTheEnd = 0x40000000u;
template <bool kWriteThrough>
__device__ __forceinline__ void matrix_finish(const MatrixState& st, const Segment& seg, int tile, const DecodeParams& prm,
                                              int lane, char* lds_wave) {
    const int kb = lane >> 4, n = lane & 15;
    const int seq_rows = prm.q_len * prm.n_q_heads;
    const int n_rows = seg.n_rows - 16 * tile;
    const float l = kb_sum(st.l);
    // Store through LDS so that every store instruction writes whole contiguous rows (a lane's own
    // accumulators are 16-byte pieces of 16 different rows).
    auto fence = [] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    if (seg.whole) {
        constexpr int kPitch = kRowBytes + 16;                   // bf16 rows, padded against bank conflicts
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint4 w;
            w.x = cvt_bf16(st.o[0][j] * inv, st.o[1][j] * inv);
            w.y = cvt_bf16(st.o[2][j] * inv, st.o[3][j] * inv);
            w.z = cvt_bf16(st.o[4][j] * inv, st.o[5][j] * inv);
            w.w = cvt_bf16(st.o[6][j] * inv, st.o[7][j] * inv);
            *reinterpret_cast<uint4*>(lds_wave + n * kPitch + (4 * kb + j) * 16) = w;
        }
        fence();
#pragma unroll
        for (int i = 0; i < 4; ++i) {                             // 4 rows of 256 bytes per store instruction
            if (4 * i >= n_rows) break;
            const int r = 4 * i + (lane >> 4);
            const uint32_t off = (uint32_t)seq_row(prm, seg, 16 * tile + r) * kRowBytes + (lane & 15) * 16;
            const u32x4_t w = *reinterpret_cast<const u32x4_t*>(lds_wave + r * kPitch + (lane & 15) * 16);
            store_b128<kWriteThrough>(prm.out + (long)seg.b * seq_rows * kHeadDim, (uint32_t)(seq_rows * kRowBytes),
                          off | (r < n_rows ? 0u : kPastTheEnd), w);
        }
        if (n < n_rows && prm.lse && kb == 0)
            prm.lse[(long)seg.b * seq_rows + seq_row(prm, seg, 16 * tile + n)] = l > 0.0f ? (st.m + __log2f(l)) * kLn2 : kNegInf;
    } else {
        constexpr int kPitch = kRowBytes + 16;                   // half a row in fp32, padded: lanes kb < 2 hold the first halves
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if ((kb >> 1) == half) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float4* w = reinterpret_cast<float4*>(lds_wave + n * kPitch + (4 * (kb & 1) + j) * 32);
                    w[0] = make_float4(st.o[0][j], st.o[1][j], st.o[2][j], st.o[3][j]);
                    w[1] = make_float4(st.o[4][j], st.o[5][j], st.o[6][j], st.o[7][j]);
                }
            }
            fence();
#pragma unroll
            for (int i = 0; i < 4; ++i) {                         // 256 bytes of 4 rows per store instruction
                if (4 * i >= n_rows) break;
                const int r = 4 * i + (lane >> 4);
                const uint32_t off = (uint32_t)seq_row(prm, seg, 16 * tile + r) * (kHeadDim * 4) + half * kRowBytes + (lane & 15) * 16;
                const u32x4_t w = *reinterpret_cast<const u32x4_t*>(lds_wave + r * kPitch + (lane & 15) * 16);
                store_b128<kWriteThrough>(prm.part_o + (long)seg.slot * seq_rows * kHeadDim, (uint32_t)(seq_rows * kHeadDim * 4),
                                          off | (r < n_rows ? 0u : kPastTheEnd), w);
            }
            if (half == 0) fence();
        }
        if (n < n_rows && kb == 0) {
            const long prow = (long)seg.slot * seq_rows + seq_row(prm, seg, 16 * tile + n);
            reinterpret_cast<float2*>(prm.part_ml)[prow] = make_float2(st.m, l);
        }
    }
    fence();      // the next tile, or the next segment's K blocks, reuse this LDS
}

// The state of a tile, left in LDS by the wave that holds a later run of the sequence's keys, and added to the own one by the
// wave that holds the first.
__device__ __forceinline__ void state_put(const MatrixState& st, char* area, int lane) {
#pragma unroll
    for (int e = 0; e < 8; ++e) *reinterpret_cast<f32x4_t*>(area + e * 1024 + lane * 16) = st.o[e];
    *reinterpret_cast<float2*>(area + 8192 + lane * 8) = make_float2(st.m, st.l);
}
__device__ __forceinline__ void state_add(MatrixState& st, const char* area, int lane) {
    const float2 ml = *reinterpret_cast<const float2*>(area + 8192 + lane * 8);
    const float m = fmaxf(st.m, ml.x), m_use = m == kNegInf ? 0.0f : m;
    const float mine = fast_exp2(st.m - m_use), other = fast_exp2(ml.x - m_use);
    st.m = m;
    st.l = st.l * mine + ml.y * other;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const f32x4_t o = *reinterpret_cast<const f32x4_t*>(area + e * 1024 + lane * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) st.o[e][j] = __builtin_fmaf(o[j], other, st.o[e][j] * mine);
    }
}

}  // namespace
}  // namespace xattn
#endif
