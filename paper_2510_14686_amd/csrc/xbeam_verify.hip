// Verification of drafted tokens against a model's probabilities from given random numbers (xbeam_verify).
//
//   p_t = softmax(scale * target_t), q_t = softmax(draft_scale * draft_t).  Draft x_t stands if all before it do and u_t q_t(x_t) < p_t(x_t).
//   At the first t that falls, the new token comes from w = max(0, p_t - q_t), without one that falls from w = p behind the last draft:
//   the least i with sum_{j <= i} w_j > u W.  E[emitted] is p's whatever q is.
//
// Steps, a kernel each:
//   read     every row once, in parts: a reference and the sum of exponentials, in 32 bits
//   decide   which drafts stand; the end of it with XBEAM_GREEDY
//   weigh    the sums of p, q and max(0, p - q) of the row that the new token comes from, part by part, in 64 bits
//   pick     the part that the random number falls into, and the token in it
// 64 bits because the borders between 100000 tokens lie 10^-5 apart on average and closer where it matters: with sums in 32 bits one token in
// a hundred would be another one's neighbour.  The row's probabilities are worked out anew in every pass: to keep them would be 8 bytes per logit.
// 64 sequences of four drafts, 131072 logits in bf16, 151 MB: 57.4 us, of which read 30 (5 TB/s, HBM), decide 4.6, weigh 19.8 (the 64-bit exponentials, a wave's
// instruction taking 8 cycles), pick 5.  With 64 bits in the first pass already and none but pick behind it 20 us more; one sequence alone, four kernels
// of dependent steps, 17.  exp2_d needs its eight multiply-adds: rounding by a large constant instead of rndne, cvt and ldexp is slower.  Greedy, 84 MB:
// 32.3 us, of which read 27.5 (exponentials and keys, the vector units busy throughout).
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "../../include/xbeam.h"
#include "xattn_device.h"
#include "xattn_launch.h"
#include "xbeam_logits.h"
#include "xbeam_verify.h"

namespace xattn {
namespace {

constexpr double kLog2e = 1.4426950408889634074;
constexpr int kWaves = kVerifyThreads / 64;

// What the first pass says about a sequence.
struct Decision {
    double factor, draft_factor;     // of p's and q's exponents, in log2 units
    double top, draft_top;           // their references: the rows' largest logits times the factor
    double ratio;                    // with kRest: of the sums of p's and q's weights, from 32 bits
    int row;                         // token t that the new one is drawn at, or -1: no probabilities there
    int accepted;
    int mode;                        // kPlain, kRest, kWithout
    int without;                     // token left out
};
constexpr int kPlain = 0, kRest = 1, kWithout = 2;
static_assert(sizeof(Decision) <= 64, "verify_layout");

// Eight logits from p on, as far as there are so many; the others -inf.
template <bool kKeep = false, typename T>
__device__ __forceinline__ void load_logits(const T* p, int left, float (&x)[8]) {
    if (left >= 8) {
        constexpr int kCount = Chunk<T>::kCount;
#pragma unroll
        for (int c = 0; c < 8 / kCount; ++c) {
            Chunk<T> chunk;
            if constexpr (kKeep) chunk.load_kept(p + c * kCount);
            else chunk.load(p + c * kCount);
#pragma unroll
            for (int i = 0; i < kCount; ++i) x[c * kCount + i] = chunk.get(i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < left ? to_float(p[i]) : kNegInf;
    }
}

template <int kCtrl, int kRows>
__device__ __forceinline__ double dpp_add_d(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, kCtrl, kRows, 0xf, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), kCtrl, kRows, 0xf, true);
    return x + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Inclusive sums over the lanes, as wave_incl_scan_i makes them.
__device__ __forceinline__ double wave_scan_d(double x) {
    x = dpp_add_d<0x111, 0xf>(x);
    x = dpp_add_d<0x112, 0xf>(x);
    x = dpp_add_d<0x114, 0xf>(x);
    x = dpp_add_d<0x118, 0xf>(x);
    x = dpp_add_d<0x142, 0xa>(x);
    return dpp_add_d<0x143, 0xc>(x);
}
__device__ __forceinline__ double lane_d(double x, int lane) {      // lane: wave-uniform
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum_d(double x) { return lane_d(wave_scan_d(x), 63); }

// 2^y, to 2^-45 of it: 2^n by the exponent, 2^f for |f| <= 1/2 by the polynomial that meets it at the ten Chebyshev nodes there.  0 from -2000 on
// down and for NaN.
__device__ __forceinline__ double exp2_d(double y) {
    y = fmax(y, -2000.0);
    const double n = rint(y), f = y - n;
    double p = 1.0205905413765595e-07;
    p = __builtin_fma(p, f, 1.325964524488711e-06);
    p = __builtin_fma(p, f, 1.5252672924850737e-05);
    p = __builtin_fma(p, f, 1.540343375125101e-04);
    p = __builtin_fma(p, f, 1.3333558200794592e-03);
    p = __builtin_fma(p, f, 9.618129193934313e-03);
    p = __builtin_fma(p, f, 5.550410866465167e-02);
    p = __builtin_fma(p, f, 2.402265069564034e-01);
    p = __builtin_fma(p, f, 6.931471805599462e-01);
    p = __builtin_fma(p, f, 1.0000000000000135);
    return ldexp(p, (int)n);
}
// log2 of a positive number, to 2^-43: the instruction's 32 bits, and what is left of x over 2^that, 1 + r with |r| < 2^-20.
__device__ __forceinline__ double log2_d(double x) {
    const int e = __builtin_amdgcn_frexp_exp(x);
    const double y = __builtin_amdgcn_frexp_mant(x), l = (double)__builtin_amdgcn_logf((float)y);
    const double r = __builtin_fma(y, exp2_d(-l), -1.0);
    return x > 0.0 && x < __builtin_inf() ? (double)e + l + (r - 0.5 * r * r) * kLog2e : x == 0.0 ? -__builtin_inf() : __builtin_nan("");
}

// Order of logits as whole numbers: value, then the lowest index; NaN below everything.
__device__ __forceinline__ uint64_t token_key(float x, int index) {
    const uint32_t u = __float_as_uint(x + 0.0f), k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return (uint64_t)(x == x ? k : 0u) << 32 | (uint32_t)~index;
}

// The exponent of a logit x, in log2 units and over that of its row's largest one m, is (x - m) times this: the same rounded factor wherever the first pass'
// sums are used.
__device__ __forceinline__ float exponent_scale(float scale) { return (float)((double)scale * kLog2e); }

// A sum's exponents are x c - r with one rounding, r = m c as rounded.  What that cut off is half of r's last digit and shared by all weights of the sum: 2^6 in 32 bits
// where m c is 2^30, 2^-17 in 64 where it is 2^36.  Further from 0 this is a lesser c with which m c is just that: logits next to m in their type are
// 2^6 and 2^12 powers of two below it with that one too, and weigh nothing among 2^24 tokens.
template <typename F>
__device__ __forceinline__ F factor_at(F c, F m, F most) {
    if (__builtin_expect(__ballot(fabs(m) * c > most) != 0, 0) && fabs(m) * c > most) c = most / fabs(m);
    return c;
}

__device__ __forceinline__ int drafts_of(const VerifyParams& prm, int b) {
    const int n = prm.n_drafts ? prm.n_drafts[b] : prm.q_len - 1;
    return n < 0 ? 0 : n < prm.q_len ? n : prm.q_len - 1;
}

// ---------------------------------------------------------------------------------- read
// grid.x = rows, those of the target, then those of the draft; grid.y = parts.  Up to kKeepBytes of logits stay in the caches (kKeep) for the kernels
// that read a row of them again: 48 sequences of four rows of 100003 in fp32 (77 MB) 29.8 -> 27.8 us, 64 of four of 128256 in bf16 (66 MB) 33.5 -> 32.6, 128 of seven of
// 50000 (90 MB) 42.4 -> 42.1; but 48 of nine of 131072 (113 MB) 49.5 -> 50.0, 64 of them (151 MB) 56.5 -> 59.
constexpr int64_t kKeepBytes = 96 << 20;
template <typename T, bool kGreedy, bool kKeep>
__global__ __launch_bounds__(kVerifyThreads) void verify_read_kernel(VerifyParams prm, VerifyCut cut) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, part = blockIdx.y;
    const int target_rows = prm.batch * prm.q_len, row = blockIdx.x;
    const bool is_draft = row >= target_rows;
    const int r = is_draft ? row - target_rows : row, per = is_draft ? prm.q_len - 1 : prm.q_len;
    const int b = r / per, t = r - b * per, n = drafts_of(prm, b);
    if (t >= n + (is_draft ? 0 : 1)) return;      // a row that no token is drawn from or judged by
    const T* const p = static_cast<const T*>(is_draft ? prm.draft : prm.target) + (int64_t)r * (is_draft ? prm.draft_stride : prm.target_stride);
    const float c = exponent_scale(is_draft ? prm.draft_scale : prm.scale);
    const int first = part * cut.size, end = first + cut.size < prm.vocab ? first + cut.size : prm.vocab;
    float m = kNegInf, f = c, ref = 0.0f, cut_off = 0.0f, sum = 0.0f;      // sum of 2^(x f - ref), ref + cut_off = m f
    uint64_t best = 0;
    // Four steps' loads go out together, and the running reference is looked at once for them.
    auto steps = [&](auto count, int i) {
        constexpr int kCount = decltype(count)::value;
        float x[kCount][8];
#pragma unroll
        for (int k = 0; k < kCount; ++k) load_logits<kKeep>(p + i + k * kVerifyStep, end - i - k * kVerifyStep, x[k]);
        float top = x[0][0];
#pragma unroll
        for (int k = 0; k < kCount; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, x[k][j]);
        if (top > m) {
            f = factor_at(c, top, 0x1p30f);
            ref = top * f;
            const float off = __builtin_fmaf(top, f, -ref);
            sum *= fast_exp2(m == kNegInf ? 0.0f : (m - top) * c + (off - cut_off));
            m = top;
            cut_off = off;
        }
#pragma unroll
        for (int k = 0; k < kCount; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum += fast_exp2(__builtin_fmaf(x[k][j], f, -ref));
                if constexpr (kGreedy) {
                    const int at = i + k * kVerifyStep + j;
                    const uint64_t key = at < end ? token_key(x[k][j], at) : 0;
                    best = key > best ? key : best;
                }
            }
    };
    int i = first + 8 * tid;
    for (; i + 3 * kVerifyStep < end; i += 4 * kVerifyStep) steps(std::integral_constant<int, 4>(), i);
    for (; i < end; i += kVerifyStep) steps(std::integral_constant<int, 1>(), i);
    __shared__ float tops[kWaves], sums[kWaves];
    __shared__ uint64_t keys[kWaves];
    const float top = wave_max(m);
    // a lane of nothing but -inf has 0, one with a NaN NaN
    const float s = wave_sum(sum * (m == kNegInf ? (sum == sum ? 0.0f : sum) : fast_exp2((m - top) * c - cut_off)));
    if constexpr (kGreedy) {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint64_t other = __shfl_xor(best, d, 64);
            best = other > best ? other : best;
        }
        if (lane == 0) keys[wave] = best;
    }
    if (lane == 0) {
        tops[wave] = top;
        sums[wave] = s;
    }
    __syncthreads();
    if (tid > 0) return;
    float all = tops[0];
    for (int w = 1; w < kWaves; ++w) all = fmaxf(all, tops[w]);
    float total = 0.0f;
    for (int w = 0; w < kWaves; ++w) {
        total += tops[w] == kNegInf ? sums[w] : sums[w] * fast_exp2((tops[w] - all) * c);
        if constexpr (kGreedy) best = keys[w] > best ? keys[w] : best;
    }
    prm.stats[(int64_t)row * cut.parts + part] = make_float2(all, total);
    if constexpr (kGreedy) prm.best[(int64_t)row * cut.parts + part] = best;
}

// ---------------------------------------------------------------------------------- decide
// A row's largest logit and log2 of its sum, which counts that as 1; no finite number where it has no probabilities.  By one wave.
struct RowSum {
    double log2_sum, top;
};
__device__ __forceinline__ RowSum row_sum(float2 mine, double c) {
    const float top = wave_max(mine.x);
    const double s = wave_sum_d(mine.x == kNegInf ? (double)mine.y : (double)mine.y * exp2_d(((double)mine.x - (double)top) * c));
    return RowSum{log2_d(s), (double)top};
}
template <typename T>
__device__ __forceinline__ double logit_at(const void* rows, int64_t stride, int64_t row, int token) { return (double)to_float(static_cast<const T*>(rows)[row * stride + token]); }

// A workgroup per sequence, a wave per row: which drafts stand, and the outputs that are known with that.
constexpr int kDecideWaves = 8;
template <typename T, bool kGreedy>
__global__ __launch_bounds__(64 * kDecideWaves) void verify_decide_kernel(VerifyParams prm, VerifyCut cut) {
    __shared__ double lses[16], tops[16], draft_tops[16], ratios[16], lps[16];
    __shared__ int stands[16], tokens[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), b = blockIdx.x, n = drafts_of(prm, b);
    const double c = (double)exponent_scale(prm.scale), dc = (double)exponent_scale(prm.draft_scale);
    auto stats_of = [&](int64_t row, bool on) {
        float2 mine = make_float2(kNegInf, 0.0f);
        if (on && lane < cut.parts) mine = prm.stats[row * cut.parts + lane];
        return mine;
    };
    for (int t = wave; t <= n; t += kDecideWaves) {
        const int64_t row = (int64_t)b * prm.q_len + t, draft_row = (int64_t)b * (prm.q_len - 1) + t;
        const bool judges = t < n, with_draft = !kGreedy && judges && prm.draft;
        const float2 mine = stats_of(row, true);
        const float2 drafts = stats_of((int64_t)prm.batch * prm.q_len + draft_row, with_draft);
        const int x = judges ? prm.draft_tokens[draft_row] : -1;
        const bool is_token = x >= 0 && x < prm.vocab;
        const double at = is_token ? logit_at<T>(prm.target, prm.target_stride, row, x) : 0.0;
        const double draft_at = is_token && with_draft ? logit_at<T>(prm.draft, prm.draft_stride, draft_row, x) : 0.0;
        const RowSum p = row_sum(mine, c);
        const double lp = (at - p.top) * c - p.log2_sum;
        double draft_top = 0.0, ratio = 0.0;
        int best = -1;
        bool fine = false;
        if constexpr (kGreedy) {
            uint64_t key = lane < cut.parts ? prm.best[row * cut.parts + lane] : 0;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const uint64_t other = __shfl_xor(key, d, 64);
                key = other > key ? other : key;
            }
            best = (int)~(uint32_t)key;
            fine = judges && x == best && lp == lp;
        } else if (judges) {
            double lq = 0.0;
            if (prm.draft) {
                const RowSum q = row_sum(drafts, dc);
                draft_top = q.log2_sum - q.log2_sum == 0.0 ? q.top : __builtin_nan("");
                lq = (draft_at - q.top) * dc - q.log2_sum;
                ratio = exp2_d(p.log2_sum - q.log2_sum);
            }
            // u q < p, where the row has probabilities: NaN and infinities are neither
            fine = is_token && draft_top == draft_top && (double)prm.uniforms[row] * exp2_d(lq) < (lp == lp ? exp2_d(lp) : 0.0);
        }
        if (lane == 0) {
            lses[t] = p.log2_sum;
            tops[t] = p.top;
            draft_tops[t] = draft_top;
            ratios[t] = ratio;
            lps[t] = lp;
            stands[t] = fine;
            tokens[t] = kGreedy && !fine ? best : x;
        }
    }
    __syncthreads();
    Decision d;
    d.accepted = 0;
    while (d.accepted < n && stands[d.accepted]) ++d.accepted;
    const int at = d.accepted;
    d.factor = factor_at((double)prm.scale * kLog2e, tops[at], 0x1p36);
    d.draft_factor = factor_at((double)prm.draft_scale * kLog2e, draft_tops[at], 0x1p36);
    d.top = tops[at] * d.factor;
    d.draft_top = draft_tops[at] * d.draft_factor;
    d.ratio = ratios[at];
    d.row = lses[at] - lses[at] == 0.0 ? at : -1;
    d.mode = kGreedy || at == n || !(d.draft_top == d.draft_top) ? kPlain : prm.draft ? kRest : kWithout;
    d.without = d.mode == kWithout && tokens[at] < prm.vocab ? tokens[at] : -1;
    if (tid < prm.q_len) {
        int token = tid < at ? tokens[tid] : -1;
        float lp = tid < at ? (float)(lps[tid] / kLog2e) : 0.0f;
        if (kGreedy && tid == at) {
            token = d.row >= 0 ? tokens[at] : -1;
            lp = d.row >= 0 ? (float)(((logit_at<T>(prm.target, prm.target_stride, (int64_t)b * prm.q_len + at, token) - tops[at]) * c - lses[at]) / kLog2e) : __builtin_nanf("");
        }
        prm.tokens[(int64_t)b * prm.q_len + tid] = token;
        if (prm.token_lp) prm.token_lp[(int64_t)b * prm.q_len + tid] = lp;
    }
    if (tid == 0) {
        prm.accepted[b] = at;
        if (!kGreedy) static_cast<Decision*>(prm.decisions)[b] = d;
    }
}

// ---------------------------------------------------------------------------------- weigh
// The rows that a sequence's new token comes from.
template <typename T>
struct Source {
    const T* p;
    const T* q;
    double c, dc;
};
template <typename T>
__device__ __forceinline__ Source<T> source_of(const VerifyParams& prm, int b, const Decision& d) {
    Source<T> s;
    s.p = static_cast<const T*>(prm.target) + ((int64_t)b * prm.q_len + d.row) * prm.target_stride;
    s.q = d.mode == kRest ? static_cast<const T*>(prm.draft) + ((int64_t)b * (prm.q_len - 1) + d.row) * prm.draft_stride : nullptr;
    s.c = d.factor;
    s.dc = d.draft_factor;
    return s;
}
// Unnormalised weights of eight tokens.
__device__ __forceinline__ void weights(const float (&x)[8], double c, double top, double (&w)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = exp2_d(__builtin_fma((double)x[j], c, -top));
}

// With P and Q for the weights of p and q as they come and r for the ratio of their sums, max(0, p - q) is max(0, P - r Q) but for a factor.  Its sum
// needs r first, yet the row is read once: the first pass says r0, off by 2^-21 of r at most in 600 pairs of rows of 5000 to 131072 logits, up to 100 from 0, with
// scales of their own from 1/4 to 4 (its sums are relative to the largest logit itself, so how far that lies from 0 and which factor it has do not count).  A token with
// P - r0 Q further from 0 than |r - r0| Q stays on its side, and the sum over those above is, exactly,
//     A - (r - r0) B      A = sum (P - r0 Q), B = sum Q      over tokens with P > r0 Q
// The others change it by |r - r0| Q each at most: the fifth sum is of Q over all within kNear r0 Q, and where that leaves more than kMayMiss of the sum open, or
// r is further off than kNear, pick sums anew with r, alone.  That happens where p and q are nearly the same, and now and then where one of the steps of the grid
// that logits of 16 bits lie on meets r (within kNear in one row of 4000 in bf16, of 500 in fp16, which mostly still leaves less open than that).  It costs 60 us
// at 131072 logits.  (A pass of its own with r, always: 64 sequences of nine rows 64.7 us in place of 56.5, one of them 20.6 in place of 17.9.)
constexpr double kNear = 0x1p-20, kMayMiss = 0x1p-30;

// grid.x = parts, grid.y = sequences.
template <typename T>
__global__ __launch_bounds__(kVerifyThreads) void verify_weigh_kernel(VerifyParams prm, VerifyCut cut) {
    __shared__ double space[kVerifySums][kWaves];
    const int tid = threadIdx.x, part = blockIdx.x, b = blockIdx.y;
    const Decision d = static_cast<const Decision*>(prm.decisions)[b];
    if (d.row < 0) return;
    const Source<T> s = source_of<T>(prm, b, d);
    const int first = part * cut.size, end = first + cut.size < prm.vocab ? first + cut.size : prm.vocab;
    double sums[kVerifySums] = {0.0, 0.0, 0.0, 0.0, 0.0};      // P, Q, A, B, near
    const double near = kNear * d.ratio;
    for (int i = first + 8 * tid; i < end; i += kVerifyStep) {
        float x[8], y[8];
        double w[8], v[8];
        load_logits(s.p + i, end - i, x);
        if (s.q) load_logits(s.q + i, end - i, y);
        weights(x, s.c, d.top, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[0] += i + j == d.without ? 0.0 : w[j];
        if (s.q) {
            weights(y, s.dc, d.draft_top, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double left = __builtin_fma(-d.ratio, v[j], w[j]);
                sums[1] += v[j];
                sums[2] += fmax(left, 0.0);
                sums[3] += left > 0.0 ? v[j] : 0.0;
                sums[4] += fabs(left) <= near * v[j] ? v[j] : 0.0;
            }
        }
    }
    const int n = s.q ? kVerifySums : 1;
    for (int k = 0; k < n; ++k) {
        const double sum = wave_sum_d(sums[k]);
        if ((tid & 63) == 0) space[k][tid >> 6] = sum;
    }
    __syncthreads();
    if (tid >= n) return;
    double all = space[tid][0];
    for (int w = 1; w < kWaves; ++w) all += space[tid][w];
    prm.sums[((int64_t)tid * prm.batch + b) * cut.parts + part] = all;
}

// ---------------------------------------------------------------------------------- pick
// A workgroup per sequence: the part that holds the random number's share of the sum, then step by step the logits of that part.  Bound by the
// fetching of its own instructions, each of which it needs once: four logits per thread (of 512) instead of eight.
constexpr int kPickThreads = 512, kPickWaves = kPickThreads / 64, kPickLogits = kVerifyStep / kPickThreads;
template <typename T>
__global__ __launch_bounds__(kPickThreads) void verify_pick_kernel(VerifyParams prm, VerifyCut cut) {
    __shared__ double totals[kPickWaves];
    __shared__ double again[kVerifyMostParts];
    __shared__ int tops[kPickWaves], heres[kPickWaves];      // a wave's last token with a weight, and the first beyond the goal
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), b = blockIdx.x;
    const double u = (double)prm.uniforms[(int64_t)b * prm.q_len + prm.q_len - 1];
    double sums[kVerifySums];      // all that may be needed, in one round trip
#pragma unroll
    for (int k = 0; k < kVerifySums; ++k) sums[k] = lane < cut.parts && (k == 0 || prm.draft) ? prm.sums[((int64_t)k * prm.batch + b) * cut.parts + lane] : 0.0;
    const Decision d = static_cast<const Decision*>(prm.decisions)[b];
    constexpr int kNone = 0x7fffffff;
    int last = -1;
    const int64_t out = (int64_t)b * prm.q_len + d.accepted;
    const double upto_p = wave_scan_d(sums[0]), all_p = lane_d(upto_p, 63), ratio = all_p / wave_sum_d(sums[1]);
    const Source<T> s = source_of<T>(prm, b, d);
    const bool drafted = d.row >= 0 && d.mode == kRest;
    const double less = ratio - d.ratio;
    double left = fmax(__builtin_fma(-less, sums[3], sums[2]), 0.0), upto_left = wave_scan_d(left), all_left = lane_d(upto_left, 63);
    if (uniform(drafted && !(fabs(less) <= 0.999 * kNear * d.ratio && fabs(less) * wave_sum_d(sums[4]) <= kMayMiss * all_left))) {
        for (int part = wave; part < cut.parts; part += kPickWaves) {
            const int first = part * cut.size, end = first + cut.size < prm.vocab ? first + cut.size : prm.vocab;
            double sum = 0.0;
            for (int i = first + 8 * lane; i < end; i += 8 * 64) {
                float x[8], y[8];
                double w[8], v[8];
                load_logits(s.p + i, end - i, x);
                load_logits(s.q + i, end - i, y);
                weights(x, s.c, d.top, w);
                weights(y, s.dc, d.draft_top, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += fmax(__builtin_fma(-ratio, v[j], w[j]), 0.0);
            }
            sum = wave_sum_d(sum);
            if (lane == 0) again[part] = sum;
        }
        __syncthreads();
        left = lane < cut.parts ? again[lane] : 0.0;
        upto_left = wave_scan_d(left);
        all_left = lane_d(upto_left, 63);
    }
    // p nowhere above q: nothing could have fallen but by rounding
    bool rest = drafted && all_left > 0.0;
    const double all = rest ? all_left : all_p;
    double upto = rest ? upto_left : upto_p, mine = rest ? left : sums[0];
    auto none = [&] {
        if (tid == 0) {
            // without a token that has all of p, it comes back: rounding alone let it fall
            const bool back = d.row >= 0 && d.mode == kWithout;
            prm.tokens[out] = back ? d.without : -1;
            if (prm.token_lp) prm.token_lp[out] = back ? 0.0f : __builtin_nanf("");
        }
    };
    if (d.row < 0 || !(all > 0.0) || !(all < __builtin_inf())) return none();
    auto finish = [&](int token, double logit) {
        prm.tokens[out] = token;
        if (prm.token_lp) {
            double z = all_p;      // without the token left out
            const double less = d.without < 0 ? (double)kNegInf : (double)to_float(s.p[d.without]);
            if (less > kNegInf) z += exp2_d(__builtin_fma(less, s.c, -d.top));
            prm.token_lp[out] = (float)((__builtin_fma(logit, s.c, -d.top) - log2_d(z)) / kLog2e);
        }
    };
    double goal = u * all;
    // A - (r - r0) B may leave something by rounding in a part whose tokens all have P <= r Q: 1e-28 of the sum, which a random number of 0 falls into.  Then it
    // is the next part with a weight, or where none is left the last one before it.
    while (last < 0) {
        unsigned long long some = __ballot(mine > 0.0);
        if (some == 0 && rest) {      // rounding in all parts
            rest = false;
            mine = sums[0];
            upto = upto_p;
            goal = u * all_p;
            some = __ballot(mine > 0.0);
        }
        if (some == 0) return none();
        const unsigned long long hit = some & __ballot(upto > goal);
        const int part = uniform(hit ? __builtin_ctzll(hit) : 63 - __builtin_clzll(some));
        double before = lane_d(upto - mine, part);
        mine = lane == part ? 0.0 : mine;
        const int first = part * cut.size, end = first + cut.size < prm.vocab ? first + cut.size : prm.vocab;
        for (int step = first; step < end; step += kVerifyStep) {
            const int i = step + kPickLogits * tid;
            float x[kPickLogits], y[kPickLogits];
            double w[kPickLogits];
#pragma unroll
            for (int j = 0; j < kPickLogits; ++j) {
                x[j] = i + j < end ? to_float(s.p[i + j]) : kNegInf;
                y[j] = rest && i + j < end ? to_float(s.q[i + j]) : kNegInf;
            }
            double sum = 0.0;
            int top = -1;
#pragma unroll
            for (int j = 0; j < kPickLogits; ++j) {
                w[j] = i + j == d.without ? 0.0 : exp2_d(__builtin_fma((double)x[j], s.c, -d.top));
                if (rest) w[j] = fmax(__builtin_fma(-ratio, exp2_d(__builtin_fma((double)y[j], s.dc, -d.draft_top)), w[j]), 0.0);
                sum += w[j];
                top = w[j] > 0.0 ? i + j : top;
            }
            const double scan = wave_scan_d(sum);
            const unsigned long long with = __ballot(top >= 0);
            top = with ? __builtin_amdgcn_readlane(top, 63 - __builtin_clzll(with | 1)) : -1;
            __syncthreads();      // the step before has been read
            if (lane == 63) {
                totals[wave] = scan;
                tops[wave] = top;
            }
            __syncthreads();
            double at = before + (scan - sum);
            for (int q = 0; q < kPickWaves; ++q) {
                at += q < wave ? totals[q] : 0.0;
                before += totals[q];
                last = tops[q] > last ? tops[q] : last;
            }
            int here = kNone;
            float logit = 0.0f;
#pragma unroll
            for (int j = 0; j < kPickLogits; ++j) {
                at += w[j];
                const bool is = at > goal && w[j] > 0.0 && here == kNone;
                logit = is ? x[j] : logit;
                here = is ? i + j : here;
            }
            const unsigned long long beyond = __ballot(here != kNone);
            const int first_here = __builtin_amdgcn_readlane(here, beyond ? __builtin_ctzll(beyond) : 0);
            if (lane == 0) heres[wave] = first_here;
            __syncthreads();
            int found = kNone;
            for (int q = 0; q < kPickWaves; ++q) found = heres[q] < found ? heres[q] : found;
            if (found == kNone) continue;
            if (here == found) finish(here, (double)logit);
            return;
        }
    }
    if (tid == 0) finish(last, (double)to_float(s.p[last]));      // the part's last one, where rounding leaves the goal just behind it
}

template <typename T, bool kGreedy>
hipError_t launch_first(const VerifyParams& prm, const VerifyLayout& w, hipStream_t stream) {
    const long rows = (long)prm.batch * (prm.draft ? 2 * prm.q_len - 1 : prm.q_len);
    const dim3 grid((unsigned)rows, (unsigned)w.read.parts);
    hipError_t e;
    if (!kGreedy && rows * prm.vocab * (int64_t)sizeof(T) <= kKeepBytes) e = launch(verify_read_kernel<T, kGreedy, !kGreedy>, grid, kVerifyThreads, stream, prm, w.read);
    else e = launch(verify_read_kernel<T, kGreedy, false>, grid, kVerifyThreads, stream, prm, w.read);
    return e != hipSuccess ? e : launch(verify_decide_kernel<T, kGreedy>, dim3((unsigned)prm.batch), 64 * kDecideWaves, stream, prm, w.read);
}
template <typename T>
hipError_t launch_type(const VerifyParams& prm, const VerifyLayout& w, hipStream_t stream) {
    if (prm.greedy) return launch_first<T, true>(prm, w, stream);
    const dim3 grid((unsigned)w.pick.parts, (unsigned)prm.batch);
    hipError_t e = launch_first<T, false>(prm, w, stream);
    if (e == hipSuccess) e = launch(verify_weigh_kernel<T>, grid, kVerifyThreads, stream, prm, w.pick);
    return e != hipSuccess ? e : launch(verify_pick_kernel<T>, dim3((unsigned)prm.batch), kPickThreads, stream, prm, w.pick);
}

}  // namespace

hipError_t launch_verify(const VerifyParams& prm, const VerifyLayout& w, hipStream_t stream) {
    switch (prm.dtype) {
        case XBEAM_BF16: return launch_type<Bf16>(prm, w, stream);
        case XBEAM_FP16: return launch_type<__half>(prm, w, stream);
        default: return launch_type<float>(prm, w, stream);
    }
}

}  // namespace xattn
