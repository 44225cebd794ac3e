// Rows into and out of a cache of 4 bits a value (xattn_rope_kvcache_mx, xattn_read_kvcache_mx; the cache: xattn_mx.h).
//
//   append  (x, y) -> (x cos a - y sin a, y cos a + x sin a) as in xattn_rope.hip; q rounded to bf16, k and v to codes with a scale per 32 values
//   read    code * scale, exact in bf16
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "xattn_device.h"
#include "xattn_launch.h"
#include "xattn_mx.h"
#include "xattn_packed.h"

namespace xattn {
namespace {

// Where token `at` of head h is: its tile, and inside it its codes of values 8 m .. 8 m + 7 and the scale of block m / 4.
struct MxPlace {
    int64_t codes, scale;
};
template <bool kV>
__device__ __forceinline__ MxPlace mx_place(int at, int head, int n_kv_heads, int m) {
    const int64_t tile = ((int64_t)(at / kMxTileTokens) * n_kv_heads + head) * kMxTileBytes;
    const int s = at >> 4 & 3, u = at & 15, c = m >> 2;
    if (kV) return MxPlace{tile + 1024 * s + 256 * (u >> 2) + 16 * m + 4 * (u & 3), tile + kMxCodeBytes + 16 * (4 * (u >> 2) + c) + 4 * s + (u & 3)};
    return MxPlace{tile + 1024 * s + 256 * c + 16 * u + 4 * (m & 3), tile + kMxCodeBytes + 4 * (16 * c + u) + s};
}

// The largest of the four lanes of a block.
template <int kCtrl>
__device__ __forceinline__ double dpp_d(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, kCtrl, 0xf, 0xf, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), kCtrl, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double block_max(double x) {
    x = fmax(x, dpp_d<0xB1>(x));
    return fmax(x, dpp_d<0x4E>(x));
}

// Eight values of a block as codes, and the block's scale byte.  Called by the block's four lanes.  The values come in double, since their last
// bit can decide a code; a float with the rest of the digits in its last bit rounds the same way.
__device__ __forceinline__ uint32_t encode(const double (&x)[8], int& scale_byte) {
    double most = 0.0;
    bool finite = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double a = fabs(x[i]);
        finite = finite && a < __builtin_inf();
        most = fmax(most, a);
    }
    most = block_max(finite ? most : __builtin_inf());
    const uint64_t bits = __builtin_bit_cast(uint64_t, most);
    int e = (int)(bits >> 52) - 1023 - 2 + ((bits & 0xfffffffffffffull) > 0xc000000000000ull ? 1 : 0);
    e = e < kMxLeastExp ? kMxLeastExp : e > kMxMostExp ? kMxMostExp : e;
    scale_byte = most < __builtin_inf() ? e + 127 : kMxNanScale;
    const double up = __builtin_bit_cast(double, (uint64_t)(1023 - e) << 52);
    uint32_t codes = 0;
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double y = x[i] * up;
        const float t = __double2float_rz(y);
        f[i] = __uint_as_float(__float_as_uint(t) | ((double)t != y ? 1u : 0u));
    }
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[0], f[1], 1.0f, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[2], f[3], 1.0f, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[4], f[5], 1.0f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[6], f[7], 1.0f, 3);
}

__device__ __forceinline__ void widen(u32x4_t x, double (&d)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        d[2 * i] = (double)bf16_lo(x[i]);
        d[2 * i + 1] = (double)bf16_hi(x[i]);
    }
}

template <int kTokens>
__global__ __launch_bounds__(kRopeThreads) void rope_mx_kernel(RopeParams prm) {
    constexpr int kPairs = kHeadDim / 2;
    __shared__ double cosines[kTokens][kPairs], sines[kTokens][kPairs];
    __shared__ int places[kTokens];             // row of the cache, or -1
    __shared__ char* bases[kTokens][2];
    __shared__ int known[kTokens];              // whether a sequence has it
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
    const int token0 = blockIdx.x * kTokens, F = prm.frequencies;
    if (wave < kTokens) {
        const int row = token0 + wave;
        int start = 0, end = 0;
        const int b = row < prm.total_q ? find_sequence(prm.q_starts, prm.batch, row, lane, start, end) : -1;
        if (b >= 0) {
            const int len = prm.kv_lens[b];
            if (lane == 0) places[wave] = len >= end - row ? len - (end - row) : -1;
            if (lane < 2) bases[wave][lane] = static_cast<char*>(lane == 0 ? prm.k_ptrs[b] : prm.v_ptrs[b]);
            for (int i = lane; i < F; i += 64) {
                const int axis = (prm.axis_of[i >> 4] >> (2 * (i & 15))) & 3;
                // a fraction of a turn, of the rounded product to all its digits
                const double angle = (double)prm.pos[(int64_t)axis * prm.total_q + row] * (double)prm.inv_freq[i];
                const double turns = angle * 0.15915494309189533577;
                const double rest = __builtin_fma(angle, 0.15915494309189533577, -turns) + angle * -9.8393383375912173e-18;
                double sine, cosine;
                sincospi(2.0 * ((turns - rint(turns)) + rest), &sine, &cosine);
                cosines[wave][i] = cosine;
                sines[wave][i] = sine;
            }
        }
        if (lane == 0) known[wave] = b >= 0;
    }
    __syncthreads();

    // q: 16 values of a head at a time, in two pieces
    const int q_items = prm.n_q_heads * (kHeadDim / 16), turned = F / 8;
    for (int item = threadIdx.x; item < kTokens * q_items; item += kRopeThreads) {
        const int tk = item / q_items, rest = item - tk * q_items, head = rest >> 3, c = rest & 7;
        if (!known[tk]) continue;
        const int64_t row = token0 + tk;
        const bool turn = c < turned, apart = turn && !prm.pairs;
        const int at0 = apart ? 8 * c : 16 * c, at1 = apart ? F + 8 * c : 16 * c + 8;
        const uint16_t* const from = prm.q + row * prm.q_stride + head * kHeadDim;
        u32x4_t x = *reinterpret_cast<const u32x4_t*>(from + at0), y = *reinterpret_cast<const u32x4_t*>(from + at1);
        if (turn) {
            float co[8], si[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                co[i] = (float)cosines[tk][8 * c + i];
                si[i] = (float)sines[tk][8 * c + i];
            }
            if (prm.pairs) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = bf16_lo(x[i]), b = bf16_hi(x[i]), d = bf16_lo(y[i]), e = bf16_hi(y[i]);
                    x[i] = cvt_bf16(a * co[i] - b * si[i], b * co[i] + a * si[i]);
                    y[i] = cvt_bf16(d * co[4 + i] - e * si[4 + i], e * co[4 + i] + d * si[4 + i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = bf16_lo(x[i]), b = bf16_hi(x[i]), d = bf16_lo(y[i]), e = bf16_hi(y[i]);
                    x[i] = cvt_bf16(a * co[2 * i] - d * si[2 * i], b * co[2 * i + 1] - e * si[2 * i + 1]);
                    y[i] = cvt_bf16(d * co[2 * i] + a * si[2 * i], e * co[2 * i + 1] + b * si[2 * i + 1]);
                }
            }
        }
        uint16_t* const to = prm.q_out + (row * prm.n_q_heads + head) * kHeadDim;
        *reinterpret_cast<u32x4_t*>(to + at0) = x;
        *reinterpret_cast<u32x4_t*>(to + at1) = y;
    }

    // k and v: 8 values of a head at a time, 16 lanes a head
    const int kv_items = prm.n_kv_heads * 16;
    for (int item = threadIdx.x; item < 2 * kTokens * kv_items; item += kRopeThreads) {
        const int tk2 = item / kv_items, rest = item - tk2 * kv_items, head = rest >> 4, m = rest & 15, tk = tk2 >> 1;
        const bool is_v = (tk2 & 1) != 0;
        if (!known[tk] || places[tk] < 0) continue;
        const int64_t row = token0 + tk;
        const uint16_t* const from = (is_v ? prm.v + row * prm.v_stride : prm.k + row * prm.k_stride) + head * kHeadDim;
        double x[8];
        widen(*reinterpret_cast<const u32x4_t*>(from + 8 * m), x);
        if (!is_v && 8 * m < 2 * F) {
            if (prm.pairs) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const double co = cosines[tk][4 * m + i], si = sines[tk][4 * m + i], a = x[2 * i], b = x[2 * i + 1];
                    x[2 * i] = a * co - b * si;
                    x[2 * i + 1] = b * co + a * si;
                }
            } else {
                const bool second = 8 * m >= F;
                const int first = second ? 8 * m - F : 8 * m;
                double other[8];
                widen(*reinterpret_cast<const u32x4_t*>(from + (second ? 8 * m - F : 8 * m + F)), other);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const double co = cosines[tk][first + i], si = sines[tk][first + i];
                    x[i] = second ? x[i] * co + other[i] * si : x[i] * co - other[i] * si;
                }
            }
        }
        int scale;
        const uint32_t codes = encode(x, scale);
        const MxPlace to = is_v ? mx_place<true>(places[tk], head, prm.n_kv_heads, m) : mx_place<false>(places[tk], head, prm.n_kv_heads, m);
        char* const base = bases[tk][is_v ? 1 : 0];
        *reinterpret_cast<uint32_t*>(base + to.codes) = codes;
        if ((m & 3) == 0) *reinterpret_cast<uint8_t*>(base + to.scale) = (uint8_t)scale;
    }
}

// A workgroup takes 16 rows of one head, 16 lanes a row: rows that follow each other share the lines of the cache.
constexpr int kReadRows = 16;
__global__ __launch_bounds__(256) void read_mx_kernel(ReadMxParams prm) {
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), m = lane & 15;
    const int head = blockIdx.y, row0 = blockIdx.x * kReadRows + 4 * wave;
    int start = 0, end = 0, b = -1;
    for (int i = 0; i < 4; ++i) {
        const int row = row0 + i;
        if (row >= prm.total_q) return;
        if (b < 0 || row < start || row >= end) b = find_sequence(prm.q_starts, prm.batch, row, lane, start, end);
        if (b < 0) continue;
        const int len = prm.kv_lens[b];
        if (lane >> 4 != i) continue;
        u32x4_t k = {0u, 0u, 0u, 0u}, v = {0u, 0u, 0u, 0u};
        if (len >= end - row) {
            const int at = len - (end - row);
            const char* const kp = static_cast<const char*>(prm.k_ptrs[b]);
            const char* const vp = static_cast<const char*>(prm.v_ptrs[b]);
            const MxPlace pk = mx_place<false>(at, head, prm.n_kv_heads, m), pv = mx_place<true>(at, head, prm.n_kv_heads, m);
            const uint32_t kc = *reinterpret_cast<const uint32_t*>(kp + pk.codes), vc = *reinterpret_cast<const uint32_t*>(vp + pv.codes);
            const float ks = __uint_as_float((uint32_t)*reinterpret_cast<const uint8_t*>(kp + pk.scale) << 23);
            const float vs = __uint_as_float((uint32_t)*reinterpret_cast<const uint8_t*>(vp + pv.scale) << 23);
            auto unpack = [](uint32_t codes, float scale) {
                return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
            };
            k = unpack(kc, ks);
            v = unpack(vc, vs);
        }
        const int64_t to = ((int64_t)row * prm.n_kv_heads + head) * kHeadDim + 8 * m;
        *reinterpret_cast<u32x4_t*>(prm.k_out + to) = k;
        *reinterpret_cast<u32x4_t*>(prm.v_out + to) = v;
    }
}

}  // namespace

hipError_t launch_rope_mx(const RopeParams& prm, hipStream_t stream) {
    auto with = [&](auto tokens) {
        constexpr int kTokens = decltype(tokens)::value;
        return launch(rope_mx_kernel<kTokens>, dim3((unsigned)((prm.total_q + kTokens - 1) / kTokens)), kRopeThreads, stream, prm);
    };
    switch (rope_rows_per_workgroup(prm.total_q, prm.n_q_heads, prm.n_kv_heads, prm.head_dim)) {
        case 1: return with(std::integral_constant<int, 1>());
        case 2: return with(std::integral_constant<int, 2>());
        default: return with(std::integral_constant<int, 4>());
    }
}

hipError_t launch_read_mx(const ReadMxParams& prm, hipStream_t stream) {
    return launch(read_mx_kernel, dim3((unsigned)((prm.total_q + kReadRows - 1) / kReadRows), (unsigned)prm.n_kv_heads), 256, stream, prm);
}

}  // namespace xattn
