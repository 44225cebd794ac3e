// Rows into and out of a cache of 4 bits a value (xattn_rope_kvcache_mx, xattn_read_kvcache_mx; the cache: xattn_mx.h).
//
//   append  (x, y) -> (x cos a - y sin a, y cos a + x sin a) as in xattn_rope.hip; q rounded to bf16, k and v to codes with a scale per 32 values
//   read    code * scale, exact in bf16 (infinity from 2^128 on)
//
// A prompt's append is bound by HBM and, beside it, the arithmetic of codes: two prompts of 4096 to 8191 tokens, 32 / 8 heads, three axes, 273 MB in
// 62 us, 4.4 TB/s.  K is rotated in 64 bits, since a value next to the border of two codes goes to one or the other by its last digit; q, which is
// rounded to bf16, in 32.  V, which is not turned, takes 32 bits with the same codes.
// q, k and v are read past the caches, which keep the codes and the turned q for the calls behind: from the kernel that writes q, k and v to the end of xattn_prefill, by way of
// xattn_read_kvcache_mx, 8 prompts of 1024 tokens, 32 / 8 heads, 178.8 us and 179.8 with plain loads, 64 of 256 282.9 and 298.2, two of 6000 655 and 663.  With q written past the caches, too, this
// call alone is shorter (two of 6000 behind that kernel 54.5 -> 43), but what reads q is longer: 181.5, 284.3 and 662 together, of 64 / 8 heads one of 2048 114.4 -> 116.8 (256 of 16, 40 / 8 heads,
// 189.6 -> 186.3); steps with xattn_decode_mx level.  A step's kernel takes 5 us, and the host's call binds it.
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
__device__ __forceinline__ uint32_t block_max(uint32_t x) {
    const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true);
    x = x > y ? x : y;
    const uint32_t z = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true);
    return x > z ? x : z;
}

// Eight values of a block as codes, and the block's scale byte.  Called by the block's four lanes.
struct Encoded {
    uint32_t codes;
    int scale;
};
// The exponent of the scale, of the largest value's: 1.f * 2^e is within 7 * 2^(e - 2) up to 1.75 * 2^e.
__device__ __forceinline__ int scale_exp(int e, bool above) {
    e += above ? -1 : -2;
    return e < kMxLeastExp ? kMxLeastExp : e > kMxMostExp ? kMxMostExp : e;
}
__device__ __forceinline__ uint32_t convert(const float (&f)[8], float scale) {
    uint32_t codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, f[0], f[1], scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[2], f[3], scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[4], f[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[6], f[7], scale, 3);
}
// Rotated values in double, whose last bit can decide a code: a float with whether anything was cut off in its last bit rounds the same way.
__device__ __forceinline__ Encoded encode(const double (&x)[8]) {
    double most = 0.0, zero = 0.0;      // zero: NaN where a value is no number or infinite
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        most = fmax(most, fabs(x[i]));
        zero = __builtin_fma(x[i], 0.0, zero);
    }
    most = block_max(zero == 0.0 ? most : __builtin_inf());
    const uint64_t bits = __builtin_bit_cast(uint64_t, most);
    const int e = scale_exp((int)(bits >> 52) - 1023, (bits & 0xfffffffffffffull) > 0xc000000000000ull);
    const double up = __builtin_bit_cast(double, (uint64_t)(1023 - e) << 52);
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // the 29 lowest bits of the significand cut off, what is left is a float's (or less than its least normal number, far below half a code)
        const double y = x[i] * up;
        const uint64_t u = __builtin_bit_cast(uint64_t, y);
        const double cut = __builtin_bit_cast(double, u & ~0x1fffffffull);
        f[i] = __uint_as_float(__float_as_uint((float)cut) | (((uint32_t)u & 0x1fffffffu) != 0u ? 1u : 0u));
    }
    return Encoded{convert(f, 1.0f), most < __builtin_inf() ? e + 127 : kMxNanScale};
}
// Eight bf16 as they are.
__device__ __forceinline__ Encoded encode(u32x4_t x) {
    uint32_t most = 0;      // the sizes order as their bits do; NaN and infinities are the largest
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = x[i] & 0x7fffu, hi = x[i] >> 16 & 0x7fffu;
        most = lo > most ? lo : most;
        most = hi > most ? hi : most;
        f[2 * i] = bf16_lo(x[i]);
        f[2 * i + 1] = bf16_hi(x[i]);
    }
    most = block_max(most);
    const int e = scale_exp((int)(most >> 7) - 127, (most & 0x7fu) > 0x60u);
    return Encoded{convert(f, __uint_as_float((uint32_t)(e + 127) << 23)), most < 0x7f80u ? e + 127 : kMxNanScale};
}

// Values that are read once: past the caches, which keep what else is in them.
__device__ __forceinline__ u32x4_t load_once(const uint16_t* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)); }

__device__ __forceinline__ void widen(u32x4_t x, double (&d)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        d[2 * i] = (double)bf16_lo(x[i]);
        d[2 * i + 1] = (double)bf16_hi(x[i]);
    }
}
// What the lane eight further in its row of 16 holds.
__device__ __forceinline__ u32x4_t across(u32x4_t x) {
    u32x4_t y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x[i], 0x128, 0xf, 0xf, true);      // row_ror:8
    return y;
}

template <int kTokens>
__global__ __launch_bounds__(kRopeThreads) void rope_mx_kernel(RopeParams prm) {
    constexpr int kPairs = kHeadDim / 2;
    __shared__ double cosines[kTokens][kPairs], sines[kTokens][kPairs];      // for k, whose codes take all digits
    __shared__ __attribute__((aligned(16))) float q_cosines[kTokens][kPairs], q_sines[kTokens][kPairs];
    __shared__ int places[kTokens];             // row of the cache, or -1
    __shared__ char* bases[kTokens][2];
    __shared__ int known[kTokens];              // whether a sequence has it
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
    const int token0 = blockIdx.x * kTokens, F = prm.frequencies, turned = F / 8;
    const bool halves = F == kPairs && !prm.pairs;      // value i turns with value 64 + i: another lane of the head has it
    // q: 16 values of a head at a time, in two pieces
    const int q_items = prm.n_q_heads * (kHeadDim / 16);
    struct QItem {
        int tk, at0, at1, c;
        bool turn;
        int64_t at;
        u32x4_t x, y;
    };
    auto fetch_q = [&](int item) {
        QItem r;
        r.tk = kTokens == 1 ? 0 : (int)((unsigned)item / (unsigned)q_items);
        const int rest = item - r.tk * q_items, head = rest >> 3;
        r.c = rest & 7;
        const int64_t row = token0 + r.tk < prm.total_q ? token0 + r.tk : prm.total_q - 1;
        r.turn = r.c < turned;
        const bool apart = r.turn && !prm.pairs;
        r.at0 = apart ? 8 * r.c : 16 * r.c;
        r.at1 = apart ? F + 8 * r.c : 16 * r.c + 8;
        r.at = (row * prm.n_q_heads + head) * kHeadDim;
        const uint16_t* const from = prm.q + row * prm.q_stride + head * kHeadDim;
        r.x = load_once(from + r.at0);
        r.y = load_once(from + r.at1);
        return r;
    };
    // k and v: 8 values of a head at a time, 16 lanes a head
    const int kv_items = prm.n_kv_heads * 16;
    struct KvItem {
        int tk, head, m;
        bool is_v, second;
        u32x4_t x, other;
    };
    auto fetch_kv = [&](int item) {
        KvItem r;
        const int tk2 = (int)((unsigned)item / (unsigned)kv_items), rest = item - tk2 * kv_items;
        r.tk = tk2 >> 1;
        r.is_v = (tk2 & 1) != 0;
        r.head = rest >> 4;
        r.m = rest & 15;
        r.second = 8 * r.m >= F;
        const int64_t row = token0 + r.tk < prm.total_q ? token0 + r.tk : prm.total_q - 1;
        const uint16_t* const from = (r.is_v ? prm.v + row * prm.v_stride : prm.k + row * prm.k_stride) + r.head * kHeadDim;
        r.x = load_once(from + 8 * r.m);
        r.other = r.x;
        if (!halves && !prm.pairs && !r.is_v && r.m < 2 * turned) r.other = *reinterpret_cast<const u32x4_t*>(from + (r.second ? 8 * r.m - F : 8 * r.m + F));
        return r;
    };
    // The first of each are on their way while the rows' sequences are looked for and the angles worked out.
    const int q_all = kTokens * q_items, kv_all = 2 * kTokens * kv_items, tid = threadIdx.x;
    QItem next_q = fetch_q(tid < q_all ? tid : 0);
    KvItem next_kv = fetch_kv(tid < kv_all ? tid : 0);
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
                q_cosines[wave][i] = (float)cosine;
                q_sines[wave][i] = (float)sine;
            }
        }
        if (lane == 0) known[wave] = b >= 0;
    }
    __syncthreads();

    for (int item = tid; item < q_all; item += kRopeThreads) {
        QItem it = next_q;
        if (item + kRopeThreads < q_all) next_q = fetch_q(item + kRopeThreads);
        if (!known[it.tk]) continue;
        u32x4_t &x = it.x, &y = it.y;
        if (it.turn) {
            float co[8], si[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                co[i] = q_cosines[it.tk][8 * it.c + i];
                si[i] = q_sines[it.tk][8 * it.c + i];
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
        *reinterpret_cast<u32x4_t*>(prm.q_out + it.at + it.at0) = x;
        *reinterpret_cast<u32x4_t*>(prm.q_out + it.at + it.at1) = y;
    }

    for (int item = tid; item < kv_all; item += kRopeThreads) {
        const KvItem it = next_kv;
        if (item + kRopeThreads < kv_all) next_kv = fetch_kv(item + kRopeThreads);
        if (!known[it.tk] || places[it.tk] < 0) continue;
        Encoded e;
        MxPlace to;
        if (it.is_v) {
            e = encode(it.x);
            to = mx_place<true>(places[it.tk], it.head, prm.n_kv_heads, it.m);
        } else {
            double x[8];
            widen(it.x, x);
            if (it.m < 2 * turned) {
                if (prm.pairs) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const double co = cosines[it.tk][4 * it.m + i], si = sines[it.tk][4 * it.m + i], a = x[2 * i], b = x[2 * i + 1];
                        x[2 * i] = a * co - b * si;
                        x[2 * i + 1] = b * co + a * si;
                    }
                } else {
                    const int first = it.second ? 8 * it.m - F : 8 * it.m;
                    double other[8];      // with the sign of the sine's product: a first half's is subtracted
                    widen((halves ? across(it.x) : it.other) ^ (it.second ? 0u : 0x80008000u), other);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = x[i] * cosines[it.tk][first + i] + other[i] * sines[it.tk][first + i];
                }
            }
            e = encode(x);
            to = mx_place<false>(places[it.tk], it.head, prm.n_kv_heads, it.m);
        }
        char* const base = bases[it.tk][it.is_v ? 1 : 0];
        *reinterpret_cast<uint32_t*>(base + to.codes) = e.codes;
        if ((it.m & 3) == 0) *reinterpret_cast<uint8_t*>(base + to.scale) = (uint8_t)e.scale;
    }
}

// A wave takes four rows, 16 lanes a row, of four heads (grid.y): a row's sequence is looked for once for them, and rows that follow each other share
// the lines of the cache.  (All heads in a workgroup: 500 rows of 40 heads 7.2 -> 10.6 us, large calls level.)  Bound by HBM: 28672 rows of 8
// heads 33.4 us, 4.5 TB/s, 26.4 where the results lie in the caches already.
// Results stay in the caches for what reads them next.  Past them this call alone would be shorter, 24.1 us, but not with an xattn_prefill behind it: 28672 rows and 128 tokens
// 102.6 -> 104.4, four of 4096 and 64 57.4 -> 59.0, and where a kernel in front has filled the caches 109.6 -> 114 and 60.5 -> 70.5.  (Better so are 16 tokens behind 28672 rows, 65.1 ->
// 62.2, and 16384 rows of 40 heads for as many query heads, 177 -> 167; behind writes 75.2 -> 74.5 and 199 -> 209.)
constexpr int kReadRows = 16, kReadHeads = 4;
__global__ __launch_bounds__(256) void read_mx_kernel(ReadMxParams prm) {
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), m = lane & 15;
    const int row0 = blockIdx.x * kReadRows + 4 * wave;
    int start = 0, end = 0, b = -1, at = -1;      // at: the lane's row in its sequence, -1 where that would be negative, -2 without a sequence
    const char *kp = nullptr, *vp = nullptr;
    for (int i = 0; i < 4; ++i) {
        const int row = row0 + i;
        if (b < 0 || row >= end) b = row < prm.total_q ? find_sequence(prm.q_starts, prm.batch, row, lane, start, end) : -1;
        int place = -2;
        const char *k = nullptr, *v = nullptr;
        if (b >= 0) {
            const int len = prm.kv_lens[b];
            place = len >= end - row ? len - (end - row) : -1;
            k = static_cast<const char*>(prm.k_ptrs[b]);
            v = static_cast<const char*>(prm.v_ptrs[b]);
        }
        if (lane >> 4 == i) {
            at = place;
            kp = k;
            vp = v;
        }
    }
    if (at == -2) return;
    const MxPlace pk = mx_place<false>(at < 0 ? 0 : at, 0, prm.n_kv_heads, m), pv = mx_place<true>(at < 0 ? 0 : at, 0, prm.n_kv_heads, m);
    auto unpack = [](uint32_t codes, uint32_t scale) {
        const float s = __uint_as_float(scale << 23);
        return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0)),
                       __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1)),
                       __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2)),
                       __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3))};
    };
    const int64_t to = ((int64_t)(row0 + (lane >> 4)) * prm.n_kv_heads) * kHeadDim + 8 * m;
    const int head0 = blockIdx.y * kReadHeads;
    uint32_t kc[kReadHeads], vc[kReadHeads], ks[kReadHeads], vs[kReadHeads];
#pragma unroll
    for (int h = 0; h < kReadHeads; ++h) {
        const bool on = head0 + h < prm.n_kv_heads && at >= 0;
        const int64_t tile = (int64_t)(head0 + h) * kMxTileBytes;
        kc[h] = vc[h] = ks[h] = vs[h] = 0;
        if (on) {
            kc[h] = *reinterpret_cast<const uint32_t*>(kp + pk.codes + tile);
            ks[h] = *reinterpret_cast<const uint8_t*>(kp + pk.scale + tile);
            vc[h] = *reinterpret_cast<const uint32_t*>(vp + pv.codes + tile);
            vs[h] = *reinterpret_cast<const uint8_t*>(vp + pv.scale + tile);
        }
    }
#pragma unroll
    for (int h = 0; h < kReadHeads; ++h) {
        if (head0 + h >= prm.n_kv_heads) break;
        uint16_t* const k = prm.k_out + to + (head0 + h) * kHeadDim;
        uint16_t* const v = prm.v_out + to + (head0 + h) * kHeadDim;
        *reinterpret_cast<u32x4_t*>(k) = unpack(kc[h], ks[h]);
        *reinterpret_cast<u32x4_t*>(v) = unpack(vc[h], vs[h]);
    }
}

// Rows per workgroup.  Fewer rows, more workgroups whose waits pass at once; more rows, fewer threads without work.  Of 1 / 2 / 4 rows each, in us: 256 rows of 40 / 8 heads
// 6.4 / 8.3 / 11.6, 1024 9.7 / 11.5 / 14.2, 1536 16.0 / 14.0 / 17.6, 2048 19.4 / 16.8 / 19.4, 8192 58.3 / 51.0 / 50.2; of 64 / 8 1024 11.5 / 13.5 / 18.8, 8192 69.6 / 62.5 / 66.0; of
// 8 / 2 1024 6.3 / 6.6 / 6.2, 1536 8.4 / 7.1 / 7.1, 4096 16.3 / 12.4 / 9.7, 8192 30.5 / 22.6 / 17.7.
int rows_per_workgroup(const RopeParams& prm) {
    if (prm.total_q < 1536) return 1;
    return (prm.n_q_heads + 2 * prm.n_kv_heads) * (kHeadDim / 16) > kRopeThreads / 2 ? 2 : 4;
}

}  // namespace

hipError_t launch_rope_mx(const RopeParams& prm, hipStream_t stream) {
    auto with = [&](auto tokens) {
        constexpr int kTokens = decltype(tokens)::value;
        return launch(rope_mx_kernel<kTokens>, dim3((unsigned)((prm.total_q + kTokens - 1) / kTokens)), kRopeThreads, stream, prm);
    };
    switch (rows_per_workgroup(prm)) {
        case 1: return with(std::integral_constant<int, 1>());
        case 2: return with(std::integral_constant<int, 2>());
        default: return with(std::integral_constant<int, 4>());
    }
}

hipError_t launch_read_mx(const ReadMxParams& prm, hipStream_t stream) {
    const int rows = (prm.total_q + kReadRows - 1) / kReadRows, heads = (prm.n_kv_heads + kReadHeads - 1) / kReadHeads;
    return launch(read_mx_kernel, dim3((unsigned)rows, (unsigned)heads), 256, stream, prm);
}

}  // namespace xattn
