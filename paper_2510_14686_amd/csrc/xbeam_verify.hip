// Verification of drafted tokens against a model's probabilities from given random numbers (xbeam_verify).
//
//   p_t = softmax(scale * target_t), q_t = softmax(draft_scale * draft_t).  Draft x_t stands if all before it do and u_t q_t(x_t) < p_t(x_t).
//   At the first t that falls, the new token comes from w = max(0, p_t - q_t), without one that falls from w = p behind the last draft:
//   the least i with sum_{j <= i} w_j > u W.  E[emitted] is p's whatever q is.
//
// Three passes (four with a draft's probabilities):
//   read     every row once, in parts: a reference and the sum of exponentials, in 32 bits; what a draft's fate is decided by
//   weigh    which drafts stand, and the sums of p and q of the row that the new token comes from, part by part, in 64 bits
//   rest     the sums of max(0, p - q), part by part
//   pick     the part that the random number falls into, and the token in it
// 64 bits because the borders between 100000 tokens lie 10^-5 apart on average and closer where it matters: with sums in 32 bits one token in
// a hundred would be another one's neighbour.  The row's probabilities are worked out anew in every pass: to keep them would be 8 bytes per logit.
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
    double top, draft_top;           // references of p's and q's exponents: the rows' maxima times scale * log2 e
    int row;                         // token t that the new one is drawn at, or -1: no probabilities there
    int accepted;
    int mode;                        // kPlain, kRest, kWithout
    int without;                     // token left out
};
constexpr int kPlain = 0, kRest = 1, kWithout = 2;
static_assert(sizeof(Decision) <= 64, "verify_layout");

// Eight logits from p on, as far as there are so many; the others -inf.
template <typename T>
__device__ __forceinline__ void load_logits(const T* p, int left, float (&x)[8]) {
    if (left >= 8) {
        constexpr int kCount = Chunk<T>::kCount;
#pragma unroll
        for (int c = 0; c < 8 / kCount; ++c) {
            Chunk<T> chunk;
            chunk.load(p + c * kCount);
#pragma unroll
            for (int i = 0; i < kCount; ++i) x[c * kCount + i] = chunk.get(i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < left ? to_float(p[i]) : kNegInf;
    }
}

__device__ __forceinline__ double wave_sum_d(double x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d, 64);
    return x;
}
__device__ __forceinline__ double wave_max_d(double x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x = fmax(x, __shfl_xor(x, d, 64));
    return x;
}

// 2^y for y <= 0, to 2^-51 of it: 2^n by the exponent, 2^f for |f| <= 1/2 by twelve terms of its series.
__device__ __forceinline__ double exp2_d(double y) {
    y = fmax(y, -1100.0);
    const double n = rint(y), f = y - n;
    double p = 2.5678435993488202e-11;                         // (ln 2)^k / k!
    p = __builtin_fma(p, f, 4.4455382718708116e-10);
    p = __builtin_fma(p, f, 7.0549116208011233e-09);
    p = __builtin_fma(p, f, 1.0178086009239699e-07);
    p = __builtin_fma(p, f, 1.3215486790144309e-06);
    p = __builtin_fma(p, f, 1.5252733804059841e-05);
    p = __builtin_fma(p, f, 1.5403530393381609e-04);
    p = __builtin_fma(p, f, 1.3333558146428443e-03);
    p = __builtin_fma(p, f, 9.6181291076284772e-03);
    p = __builtin_fma(p, f, 5.5504108664821580e-02);
    p = __builtin_fma(p, f, 2.4022650695910072e-01);
    p = __builtin_fma(p, f, 6.9314718055994531e-01);
    p = __builtin_fma(p, f, 1.0);
    return ldexp(p, (int)n);
}

// Order of logits as whole numbers: value, then the lowest index; NaN below everything.
__device__ __forceinline__ uint64_t token_key(float x, int index) {
    const uint32_t u = __float_as_uint(x + 0.0f), k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return (uint64_t)(x == x ? k : 0u) << 32 | (uint32_t)~index;
}

__device__ __forceinline__ int drafts_of(const VerifyParams& prm, int b) {
    const int n = prm.n_drafts ? prm.n_drafts[b] : prm.q_len - 1;
    return n < 0 ? 0 : n < prm.q_len ? n : prm.q_len - 1;
}

// ---------------------------------------------------------------------------------- read
// grid.x = rows, those of the target, then those of the draft; grid.y = parts.
template <typename T>
__global__ __launch_bounds__(kVerifyThreads) void verify_read_kernel(VerifyParams prm, VerifyCut cut) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, part = blockIdx.y;
    const int target_rows = prm.batch * prm.q_len, row = blockIdx.x;
    const bool is_draft = row >= target_rows;
    const int r = is_draft ? row - target_rows : row, per = is_draft ? prm.q_len - 1 : prm.q_len;
    const int b = r / per, t = r - b * per, n = drafts_of(prm, b);
    if (t >= n + (is_draft ? 0 : 1)) return;      // a row that no token is drawn from or judged by
    const T* const p = static_cast<const T*>(is_draft ? prm.draft : prm.target) + (int64_t)r * (is_draft ? prm.draft_stride : prm.target_stride);
    const float c = (float)((double)(is_draft ? prm.draft_scale : prm.scale) * kLog2e);
    const int first = part * cut.size, end = first + cut.size < prm.vocab ? first + cut.size : prm.vocab;
    float m = kNegInf, ref = 0.0f, sum = 0.0f;
    uint64_t best = 0;
    for (int i = first + 8 * tid; i < end; i += kVerifyStep) {
        float x[8];
        load_logits(p + i, end - i, x);
        float top = x[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
        if (top > m) {
            const float to = top * c;
            sum *= fast_exp2(m == kNegInf ? 0.0f : ref - to);
            m = top;
            ref = to;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sum += fast_exp2(__builtin_fmaf(x[j], c, -ref));
            if (prm.greedy) {
                const uint64_t key = i + j < end ? token_key(x[j], i + j) : 0;
                best = key > best ? key : best;
            }
        }
    }
    __shared__ float refs[kWaves], sums[kWaves];
    __shared__ uint64_t keys[kWaves];
    const float mine = m == kNegInf ? kNegInf : ref, top = wave_max(mine);
    // a lane of nothing but -inf has 0, one with a NaN NaN
    const float s = wave_sum(sum * (mine == kNegInf ? (sum == sum ? 0.0f : sum) : fast_exp2(mine - top)));
    if (prm.greedy) {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint64_t other = __shfl_xor(best, d, 64);
            best = other > best ? other : best;
        }
    }
    if (lane == 0) {
        refs[wave] = top;
        sums[wave] = s;
        keys[wave] = best;
    }
    __syncthreads();
    if (tid > 0) return;
    float all = refs[0];
    for (int w = 1; w < kWaves; ++w) all = fmaxf(all, refs[w]);
    float total = 0.0f;
    for (int w = 0; w < kWaves; ++w) {
        total += refs[w] == kNegInf ? sums[w] : sums[w] * fast_exp2(refs[w] - all);
        best = keys[w] > best ? keys[w] : best;
    }
    prm.stats[(int64_t)row * cut.parts + part] = make_float2(all, total);
    if (prm.greedy) prm.best[(int64_t)row * cut.parts + part] = best;
}

// ---------------------------------------------------------------------------------- weigh
// log2 of a row's sum of exponentials, and the largest exponent; NaN where the row has no probabilities.  By one wave.
struct RowSum {
    double log2_sum, top;
};
__device__ __forceinline__ RowSum row_sum(const float2* stats, int parts, int lane) {
    const float2 mine = lane < parts ? stats[lane] : make_float2(kNegInf, 0.0f);
    const double top = wave_max_d((double)mine.x);
    const double s = wave_sum_d(mine.x == kNegInf ? (double)mine.y : (double)mine.y * exp2((double)mine.x - top));
    return RowSum{log2(s) + top, top};
}
template <typename T>
__device__ __forceinline__ double logit_at(const void* rows, int64_t stride, int64_t row, int token) { return (double)to_float(static_cast<const T*>(rows)[row * stride + token]); }

// Sequence b's drafts, by all waves; the outputs that are known.
template <typename T>
__device__ __forceinline__ Decision decide(const VerifyParams& prm, const VerifyCut& cut, int b, int tid, bool writes) {
    __shared__ double lses[16], tops[16], draft_tops[16], lps[16];
    __shared__ int stands[16], tokens[16];
    const int lane = tid & 63, wave = tid >> 6, n = drafts_of(prm, b);
    const double c = (double)(float)((double)prm.scale * kLog2e), dc = (double)(float)((double)prm.draft_scale * kLog2e);
    for (int t = wave; t <= n; t += kWaves) {
        const int64_t row = (int64_t)b * prm.q_len + t, draft_row = (int64_t)b * (prm.q_len - 1) + t;
        const RowSum p = row_sum(prm.stats + row * cut.parts, cut.parts, lane);
        int best = -1;
        if (prm.greedy) {
            uint64_t key = lane < cut.parts ? prm.best[row * cut.parts + lane] : 0;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const uint64_t other = __shfl_xor(key, d, 64);
                key = other > key ? other : key;
            }
            best = (int)~(uint32_t)key;
        }
        bool fine = false;
        double lp = 0.0, draft_top = 0.0;
        int x = -1;
        if (t < n) {
            double lq = 0.0, draft_log2_sum = 0.0;
            if (prm.draft && !prm.greedy) {
                const RowSum q = row_sum(prm.stats + ((int64_t)prm.batch * prm.q_len + draft_row) * cut.parts, cut.parts, lane);
                draft_log2_sum = q.log2_sum;
                draft_top = q.log2_sum - q.log2_sum == 0.0 ? q.top : __builtin_nan("");
            }
            x = prm.draft_tokens[draft_row];
            if (x >= 0 && x < prm.vocab) {
                lp = logit_at<T>(prm.target, prm.target_stride, row, x) * c - p.log2_sum;
                if (prm.greedy) {
                    fine = x == best && lp == lp;
                } else {
                    if (prm.draft) lq = logit_at<T>(prm.draft, prm.draft_stride, draft_row, x) * dc - draft_log2_sum;
                    fine = draft_top == draft_top && (double)prm.uniforms[(int64_t)b * prm.q_len + t] * exp2(lq) < exp2(lp);
                }
            }
        }
        if (lane == 0) {
            lses[t] = p.log2_sum;
            tops[t] = p.top;
            draft_tops[t] = draft_top;
            lps[t] = lp;
            stands[t] = fine;
            tokens[t] = prm.greedy && (t == n || !fine) ? best : x;
        }
    }
    __syncthreads();
    Decision d;
    d.accepted = 0;
    while (d.accepted < n && stands[d.accepted]) ++d.accepted;
    const int at = d.accepted;
    d.top = tops[at];
    d.draft_top = draft_tops[at];
    d.row = lses[at] - lses[at] == 0.0 ? at : -1;
    d.mode = prm.greedy || at == n || !(d.draft_top == d.draft_top) ? kPlain : prm.draft ? kRest : kWithout;
    d.without = d.mode == kWithout && tokens[at] < prm.vocab ? tokens[at] : -1;
    if (writes) {
        if (tid < prm.q_len) {
            int token = tid < at ? tokens[tid] : -1;
            float lp = tid < at ? (float)(lps[tid] / kLog2e) : 0.0f;
            if (prm.greedy && tid == at) {
                token = d.row >= 0 ? tokens[at] : -1;
                lp = d.row >= 0 ? (float)((logit_at<T>(prm.target, prm.target_stride, (int64_t)b * prm.q_len + at, token) * c - lses[at]) / kLog2e) : __builtin_nanf("");
            }
            prm.tokens[(int64_t)b * prm.q_len + tid] = token;
            if (prm.token_lp) prm.token_lp[(int64_t)b * prm.q_len + tid] = lp;
        }
        if (tid == 0) {
            prm.accepted[b] = at;
            static_cast<Decision*>(prm.decisions)[b] = d;
        }
    }
    return d;
}

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
    s.c = (double)prm.scale * kLog2e;
    s.dc = (double)prm.draft_scale * kLog2e;
    return s;
}
// Unnormalised weights of eight tokens.
__device__ __forceinline__ void weights(const float (&x)[8], double c, double top, double (&w)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = x[j] == kNegInf ? 0.0 : exp2_d((double)x[j] * c - top);
}

__device__ __forceinline__ double block_sum_d(double x, int tid, double* space) {
    x = wave_sum_d(x);
    if ((tid & 63) == 0) space[tid >> 6] = x;
    __syncthreads();
    double all = space[0];
    for (int w = 1; w < kWaves; ++w) all += space[w];
    return all;
}

// grid.x = parts, grid.y = sequences.  The first part's workgroup leaves the decision for the passes behind.
template <typename T>
__global__ __launch_bounds__(kVerifyThreads) void verify_weigh_kernel(VerifyParams prm, VerifyCut read, VerifyCut cut) {
    __shared__ double space[2][kWaves];
    const int tid = threadIdx.x, part = blockIdx.x, b = blockIdx.y;
    const Decision d = decide<T>(prm, read, b, tid, part == 0);
    if (d.row < 0 || prm.greedy) return;
    const Source<T> s = source_of<T>(prm, b, d);
    const int first = part * cut.size, end = first + cut.size < prm.vocab ? first + cut.size : prm.vocab;
    double sum = 0.0, draft_sum = 0.0;
    for (int i = first + 8 * tid; i < end; i += kVerifyStep) {
        float x[8];
        double w[8];
        load_logits(s.p + i, end - i, x);
        weights(x, s.c, d.top, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += i + j == d.without ? 0.0 : w[j];
        if (s.q) {
            load_logits(s.q + i, end - i, x);
            weights(x, s.dc, d.draft_top, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) draft_sum += w[j];
        }
    }
    sum = block_sum_d(sum, tid, space[0]);
    draft_sum = block_sum_d(draft_sum, tid, space[1]);
    if (tid == 0) {
        prm.sums[(int64_t)b * cut.parts + part] = sum;
        prm.sums[((int64_t)prm.batch + b) * cut.parts + part] = draft_sum;
    }
}

// ---------------------------------------------------------------------------------- rest and pick
// What 1 / sum p and 1 / sum q are, from the parts' sums: by every wave.
struct Norms {
    double p, q;
};
__device__ __forceinline__ Norms norms_of(const VerifyParams& prm, const VerifyCut& cut, int b, int lane) {
    const double p = wave_sum_d(lane < cut.parts ? prm.sums[(int64_t)b * cut.parts + lane] : 0.0);
    const double q = wave_sum_d(lane < cut.parts ? prm.sums[((int64_t)prm.batch + b) * cut.parts + lane] : 0.0);
    return Norms{1.0 / p, 1.0 / q};
}
// max(0, p - q) of eight tokens.
template <typename T>
__device__ __forceinline__ void rest_of(const Source<T>& s, const Decision& d, const Norms& norm, int i, int end, double (&w)[8]) {
    float x[8];
    double v[8];
    load_logits(s.p + i, end - i, x);
    weights(x, s.c, d.top, w);
    load_logits(s.q + i, end - i, x);
    weights(x, s.dc, d.draft_top, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = fmax(w[j] * norm.p - v[j] * norm.q, 0.0);
}

template <typename T>
__global__ __launch_bounds__(kVerifyThreads) void verify_rest_kernel(VerifyParams prm, VerifyCut cut) {
    __shared__ double space[kWaves];
    const int tid = threadIdx.x, part = blockIdx.x, b = blockIdx.y;
    const Decision d = static_cast<const Decision*>(prm.decisions)[b];
    if (d.row < 0 || d.mode != kRest) return;
    const Source<T> s = source_of<T>(prm, b, d);
    const Norms norm = norms_of(prm, cut, b, tid & 63);
    const int first = part * cut.size, end = first + cut.size < prm.vocab ? first + cut.size : prm.vocab;
    double sum = 0.0;
    for (int i = first + 8 * tid; i < end; i += kVerifyStep) {
        double w[8];
        rest_of(s, d, norm, i, end, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += w[j];
    }
    sum = block_sum_d(sum, tid, space);
    if (tid == 0) prm.sums[((int64_t)2 * prm.batch + b) * cut.parts + part] = sum;
}

__device__ __forceinline__ double wave_scan_d(double x, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double other = __shfl_up(x, d, 64);
        x += lane >= d ? other : 0.0;
    }
    return x;
}

// A workgroup per sequence: the part that holds the random number's share of the sum, then step by step the logits of that part.
template <typename T>
__global__ __launch_bounds__(kVerifyThreads) void verify_pick_kernel(VerifyParams prm, VerifyCut read, VerifyCut cut) {
    __shared__ double totals[kWaves];
    __shared__ int found, last;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x;
    const Decision d = static_cast<const Decision*>(prm.decisions)[b];
    const int64_t out = (int64_t)b * prm.q_len + d.accepted;
    auto nothing = [&] {
        if (tid == 0) {
            prm.tokens[out] = -1;
            if (prm.token_lp) prm.token_lp[out] = __builtin_nanf("");
        }
    };
    if (d.row < 0) {
        nothing();
        return;
    }
    const Source<T> s = source_of<T>(prm, b, d);
    const Norms norm = norms_of(prm, cut, b, lane);
    bool rest = d.mode == kRest;
    double mine = lane < cut.parts ? prm.sums[((int64_t)(rest ? 2 : 0) * prm.batch + b) * cut.parts + lane] : 0.0;
    double upto = wave_scan_d(mine, lane), all = __shfl(upto, 63, 64);
    if (rest && !(all > 0.0)) {      // p is nowhere above q: nothing could have fallen but by rounding
        rest = false;
        mine = lane < cut.parts ? prm.sums[(int64_t)b * cut.parts + lane] : 0.0;
        upto = wave_scan_d(mine, lane);
        all = __shfl(upto, 63, 64);
    }
    if (!(all > 0.0) && d.mode == kWithout) {      // the token left out has all of p: rounding alone let it fall
        if (tid == 0) {
            prm.tokens[out] = d.without;
            if (prm.token_lp) prm.token_lp[out] = 0.0f;
        }
        return;
    }
    if (!(all > 0.0) || !(all < __builtin_inf())) {
        nothing();
        return;
    }
    const double u = (double)prm.uniforms[(int64_t)b * prm.q_len + prm.q_len - 1], goal = u * all;
    const unsigned long long hit = __ballot(lane < cut.parts && upto > goal), some = __ballot(mine > 0.0);
    const int part = hit ? __builtin_ctzll(hit) : 63 - __builtin_clzll(some);
    double before = __shfl(upto - mine, part, 64);
    const int first = part * cut.size, end = first + cut.size < prm.vocab ? first + cut.size : prm.vocab;
    if (tid == 0) {
        found = 0x7fffffff;
        last = -1;
    }
    for (int step = first; step < end; step += kVerifyStep) {
        const int i = step + 8 * tid;
        double w[8] = {};
        if (i < end) {
            if (rest) {
                rest_of(s, d, norm, i, end, w);
            } else {
                float x[8];
                load_logits(s.p + i, end - i, x);
                weights(x, s.c, d.top, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = i + j == d.without ? 0.0 : w[j];
            }
        }
        double sum = 0.0;
        int top = -1;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sum += w[j];
            top = w[j] > 0.0 ? i + j : top;
        }
        const double scan = wave_scan_d(sum, lane);
        __syncthreads();
        if (lane == 63) totals[wave] = scan;
        if (top >= 0) atomicMax(&last, top);
        __syncthreads();
        double at = before + (scan - sum);
        for (int q = 0; q < kWaves; ++q) {
            at += q < wave ? totals[q] : 0.0;
            before += totals[q];
        }
        int here = 0x7fffffff;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            at += w[j];
            if (at > goal && w[j] > 0.0 && here == 0x7fffffff) here = i + j;
        }
        if (here != 0x7fffffff) atomicMin(&found, here);
        __syncthreads();
        if (found != 0x7fffffff) break;
    }
    if (tid == 0) {
        const int token = found != 0x7fffffff ? found : last;      // the last of the part where rounding leaves the goal just behind it
        prm.tokens[out] = token;
        if (prm.token_lp) {
            double z = 0.0;
            for (int q = 0; q < cut.parts; ++q) z += prm.sums[(int64_t)b * cut.parts + q];
            if (d.mode == kWithout) {      // the sums lack the token left out
                const double less = d.without < 0 ? (double)kNegInf : (double)to_float(s.p[d.without]);
                if (less > kNegInf) z += exp2_d(less * s.c - d.top);
            }
            prm.token_lp[out] = (float)(((double)to_float(s.p[token]) * s.c - d.top - log2(z)) / kLog2e);
        }
    }
}

template <typename T>
hipError_t launch_type(const VerifyParams& prm, const VerifyLayout& w, hipStream_t stream) {
    const long rows = (long)prm.batch * (prm.draft && !prm.greedy ? 2 * prm.q_len - 1 : prm.q_len);
    hipError_t e = launch(verify_read_kernel<T>, dim3((unsigned)rows, (unsigned)w.read.parts), kVerifyThreads, stream, prm, w.read);
    if (e != hipSuccess) return e;
    const dim3 grid(prm.greedy ? 1u : (unsigned)w.pick.parts, (unsigned)prm.batch);
    e = launch(verify_weigh_kernel<T>, grid, kVerifyThreads, stream, prm, w.read, w.pick);
    if (e != hipSuccess || prm.greedy) return e;
    if (prm.draft && (e = launch(verify_rest_kernel<T>, grid, kVerifyThreads, stream, prm, w.pick)) != hipSuccess) return e;
    return launch(verify_pick_kernel<T>, dim3((unsigned)prm.batch), kVerifyThreads, stream, prm, w.read, w.pick);
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
