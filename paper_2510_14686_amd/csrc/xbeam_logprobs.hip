// Log-probabilities of given tokens, entropy and the top alternatives of rows of logits (xbeam_logprobs), in one pass.
//
//   x = scale * logit;  s = sum exp(x - m), t = sum (x - m) exp(x - m);  lse = m + ln s;  lp = x - lse;  H = ln s - t / s
//
// Bound by memory: a row is read once.  Every lane keeps m (its own maximum), s and t of its values, moved on when m moves, and the
// lanes' are put together at the end.
//
// Alternatives: a lane's maximum is there anyway, and if in each of the 8 waves ceil(k / 8) lanes have a maximum of tau or
// more, so have k values of the row: what is below tau is none of the k.  So values are only compared with tau, eight at
// a time, by their maximum; those that pass go to the wave's list in LDS, with their index.  tau rises as the row is read, and of
// random rows a few times k values pass.  A list that is full (a row that ascends, or whose values are all equal) is cut to its k
// best.  Order everywhere: value descending, then index ascending, as one 64-bit number.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "../../include/xbeam.h"
#include "xattn_device.h"
#include "xattn_launch.h"
#include "xbeam_logprobs.h"

namespace xattn {
namespace {

constexpr int kRowWaves = 8;
constexpr int kRowThreads = 64 * kRowWaves;
constexpr int kVec = 8;                          // values per lane and load
constexpr int kStep = 64 * kVec;                 // values per wave and load
constexpr int kLoads = 2;                        // loads of a wave in a row
constexpr int kLeastPart = kRowWaves * kStep;    // values
constexpr int kMostMerged = 8192;                // candidates that the merge of a row's parts holds
constexpr float kFar = 1e30f;                    // logits beyond are summed up in a second pass, whose differences do not overflow

// Bits that order as the values do; NaN below everything (0), -0 as 0.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    const uint32_t k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return x == x ? k : 0u;
}
constexpr uint32_t kLowKey = 0x007fffffu;        // of -inf; lesser ones are no value's
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k ^ (k & 0x80000000u ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ uint64_t candidate(uint32_t key, int index) { return (uint64_t)key << 32 | (uint32_t)~index; }

struct Bf16 {
    uint16_t bits;
};
__device__ __forceinline__ float to_float(Bf16 x) { return __uint_as_float((uint32_t)x.bits << 16); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(float x) { return x; }

// Eight values as they lie in memory; rows begin where they like.
template <typename T> struct Raw;
typedef uint32_t u32x4_un __attribute__((ext_vector_type(4), aligned(2)));
template <> struct Raw<Bf16> {
    u32x4_t x;
    __device__ __forceinline__ void load(const Bf16* p) { x = *reinterpret_cast<const u32x4_un*>(p); }
    __device__ __forceinline__ float get(int i) const { return i & 1 ? bf16_hi(x[i >> 1]) : bf16_lo(x[i >> 1]); }
};
template <> struct Raw<__half> {
    u32x4_t x;
    __device__ __forceinline__ void load(const __half* p) { x = *reinterpret_cast<const u32x4_un*>(p); }
    __device__ __forceinline__ float get(int i) const {
        const uint32_t w = x[i >> 1];
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? w >> 16 : w));
    }
};
typedef uint32_t u32x4_un4 __attribute__((ext_vector_type(4), aligned(4)));
template <> struct Raw<float> {
    u32x4_t x[2];
    __device__ __forceinline__ void load(const float* p) {
        x[0] = *reinterpret_cast<const u32x4_un4*>(p);
        x[1] = *reinterpret_cast<const u32x4_un4*>(p + 4);
    }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(x[i >> 2][i & 3]); }
};

// m, s and t of some values; m is finite.
struct Sums {
    float m, s, t;
};
__device__ __forceinline__ void move_to(Sums& a, float m, float c) {
    const float d = fmaxf((a.m - m) * c, -1e30f), f = fast_exp2(d);
    a.t = f * (a.t + d * a.s);
    a.s *= f;
    a.m = m;
}
__device__ __forceinline__ void add(Sums& a, float y) {      // y = (x - m) * c
    const float e = fast_exp2(y);
    a.s += e;
    a.t = __builtin_fmaf(e, fmaxf(y, -1000.0f), a.t);        // e is 0 from -150 on, and -inf times that no number
}

// The k best of the `count` candidates of a wave's list, which it leaves at the list's start; returns the least of them.
template <int kCap>
__device__ __forceinline__ uint64_t cut_list(uint64_t* list, int count, int k, int lane) {
    uint64_t c[kCap / 64];
#pragma unroll
    for (int i = 0; i < kCap / 64; ++i) c[i] = 64 * i + lane < count ? list[64 * i + lane] : 0;
    uint64_t least = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t trial = least | 1ull << bit;
        int n = 0;
#pragma unroll
        for (int i = 0; i < kCap / 64; ++i) n += __builtin_popcountll(__ballot(c[i] >= trial));
        if (n >= k) least = trial;
        if (n == k) break;
    }
    __builtin_amdgcn_wave_barrier();
    int at = 0;
#pragma unroll
    for (int i = 0; i < kCap / 64; ++i) {
        const unsigned long long keep = __ballot(c[i] >= least);
        if (c[i] >= least) list[at + __builtin_popcountll(keep & ((1ull << lane) - 1))] = c[i];
        at += __builtin_popcountll(keep);
    }
    __builtin_amdgcn_wave_barrier();
    return least;
}

// The r-th largest of the lanes' keys, or a little less (16 bits of it).
__device__ __forceinline__ uint32_t nth_key(uint32_t key, int r) {
    uint32_t at = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t trial = at | 1u << bit;
        if (__builtin_popcountll(__ballot(key >= trial)) >= r) at = trial;
    }
    return at;
}

// Puts n candidates (at most `room`, a power of two) of the workgroup into order.  Called by all threads; LDS is ready before and after.
template <int kThreads>
__device__ __forceinline__ void sort_candidates(uint64_t* list, int n, int room, int tid) {
    if (n <= 128) {
        const uint64_t mine = tid < n ? list[tid] : 0;
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += list[j] > mine;
        __syncthreads();
        if (tid < n) list[rank] = mine;
        __syncthreads();
        return;
    }
    int size = 256;
    while (size < n) size <<= 1;
    if (size > room) size = room;
    for (int i = n + tid; i < size; i += kThreads) list[i] = 0;
    __syncthreads();
    for (int k = 2; k <= size; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            for (int p = tid; p < size / 2; p += kThreads) {
                const int i = 2 * p - (p & (j - 1)), other = i + j;
                const uint64_t a = list[i], b = list[other];
                if ((a < b) == ((i & k) == 0)) {
                    list[i] = b;
                    list[other] = a;
                }
            }
            __syncthreads();
        }
}

template <typename T>
__device__ __forceinline__ void write_sums(const LogprobsParams& prm, int row, const Sums& a, float log_s, int tid) {
    if (tid != 0) return;
    if (prm.lse) prm.lse[row] = a.m * prm.scale + log_s;
    if (prm.entropy) prm.entropy[row] = log_s - a.t / a.s * kLn2;
    if (prm.tokens) {
        const int token = prm.tokens[row];
        float lp = 0.0f;
        if (token >= 0) {
            const float x = token < prm.vocab ? to_float(static_cast<const T*>(prm.logits)[row * prm.row_stride + token]) : __builtin_nanf("");
            lp = (x - a.m) * prm.scale - log_s;
        }
        prm.token_lp[row] = lp;
    }
}
__device__ __forceinline__ void write_top(const LogprobsParams& prm, int row, const uint64_t* list, int n, float m, float log_s, int tid, int threads) {
    for (int i = tid; i < prm.top_k; i += threads) {
        const uint64_t c = i < n ? list[i] : 0;
        const int64_t at = (int64_t)row * prm.top_k + i;
        prm.top_tok[at] = c ? (int)~(uint32_t)c : -1;
        prm.top_lp[at] = c ? (key_value((uint32_t)(c >> 32)) - m) * prm.scale - log_s : __builtin_nanf("");
    }
}

// What a part of a row leaves in the workspace: its sums, and its candidates in order (0: none).
struct PartSpace {
    float* sums;               // [rows * parts, 4]
    uint64_t* candidates;      // [rows * parts, top_k]
};
__device__ __host__ __forceinline__ PartSpace part_space(char* ws, int rows, int parts) {
    return PartSpace{reinterpret_cast<float*>(ws), reinterpret_cast<uint64_t*>(ws + (size_t)rows * parts * 16)};
}

// A row, or one of its parts, per workgroup.  kCap: candidates that a wave's list holds; 0 without alternatives.
template <typename T, int kCap>
__global__ __launch_bounds__(kRowThreads) void logprobs_kernel(LogprobsParams prm, int parts, int part_size) {
    __shared__ uint64_t lists[kCap ? kRowWaves * kCap : 1];
    __shared__ volatile uint32_t taus[kRowWaves];
    __shared__ int counts[kRowWaves];
    __shared__ float tops[kRowWaves];
    __shared__ Sums partial[kRowWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int row = blockIdx.x / (unsigned)parts, part = blockIdx.x - row * parts;
    const int begin = part * part_size, end = prm.vocab - begin < part_size ? prm.vocab : begin + part_size;
    const T* const logits = static_cast<const T*>(prm.logits) + row * prm.row_stride;
    const float c = prm.scale_log2;
    const int k = prm.top_k, per_wave = (k + kRowWaves - 1) / kRowWaves;
    uint64_t* const list = lists + wave * kCap;

    Sums a = {-kFar, 0.0f, 0.0f};
    float top = kNegInf;             // the lane's maximum
    uint32_t tau = 1, own = 1;       // least key to take: by all waves' maxima, by the own list
    int count = 0, round = 0;
    if (tid < kRowWaves) taus[tid] = 0;
    __syncthreads();

    // Largest keys so far -> tau.  The waves do not wait for each other: an older tau is a lower one.
    auto raise = [&]() {
        const uint32_t mine = nth_key(order_key(top), per_wave);
        if (lane == 0) taus[wave] = mine;
    };
    auto look = [&]() {
        uint32_t all = ~0u;
#pragma unroll
        for (int i = 0; i < kRowWaves; ++i) {
            const uint32_t x = taus[i];
            all = x < all ? x : all;
        }
        all = (uint32_t)uniform((int)all);
        tau = all > tau ? all : tau;
    };
    const int stride = kRowWaves * kLoads * kStep, rounds = (end - begin + stride - 1) / stride;
    for (; round < rounds; ++round) {
        const int base = begin + round * stride + wave * (kLoads * kStep);
        Raw<T> raw[kLoads];
        float x[kLoads][kVec], most[kLoads];
        if (base + kLoads * kStep <= end) {
#pragma unroll
            for (int u = 0; u < kLoads; ++u) raw[u].load(logits + base + u * kStep + lane * kVec);
#pragma unroll
            for (int u = 0; u < kLoads; ++u)
#pragma unroll
                for (int i = 0; i < kVec; ++i) x[u][i] = raw[u].get(i);
        } else {
#pragma unroll
            for (int u = 0; u < kLoads; ++u)
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const int at = base + u * kStep + lane * kVec + i;
                    x[u][i] = at < end ? to_float(logits[at]) : kNegInf;
                }
        }
        float new_top = top;
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            most[u] = x[u][0];
#pragma unroll
            for (int i = 1; i < kVec; ++i) most[u] = fmaxf(most[u], x[u][i]);
            new_top = fmaxf(new_top, most[u]);
        }
        if (__ballot(new_top > top) != 0) {
            top = new_top;
            move_to(a, fmaxf(top, -kFar), c);
        }
        const float mc = a.m * c;
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
#pragma unroll
            for (int i = 0; i < kVec; ++i) add(a, __builtin_fmaf(x[u][i], c, -mc));
        if constexpr (kCap > 0) {
            if ((round & (round - 1)) == 0) {      // rounds 0, 1, 2, 4, 8, ...
                raise();
                if (round == 0) __syncthreads();
                look();
            }
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                const uint32_t low = tau > own ? tau : own;
                if (low > kLowKey && __ballot(most[u] >= key_value(low)) == 0) continue;
                const int first = base + u * kStep + lane * kVec;
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const uint32_t key = order_key(x[u][i]);
                    const bool take = key >= low && first + i < end;
                    const unsigned long long takes = __ballot(take);
                    if (takes == 0) continue;
                    if (count + 64 > kCap) {
                        // The list's k best come before any later value that equals the least of them; not before the rest
                        // of these 512, whose indices are not in order, hence `low`.
                        const uint32_t least = (uint32_t)(cut_list<kCap>(list, count, k, lane) >> 32);
                        own = least + 1;
                        count = k;
                    }
                    if (take) list[count + __builtin_popcountll(takes & ((1ull << lane) - 1))] = candidate(key, first + i);
                    count += __builtin_popcountll(takes);
                }
            }
        }
    }

    // The lanes' sums, then the waves'.
    if constexpr (kCap > 0) raise();
    const float wave_top = wave_max(top);
    {
        const float m = fmaxf(wave_top, -kFar);
        move_to(a, m, c);
        a.s = wave_sum(a.s);
        a.t = wave_sum(a.t);
    }
    if (lane == 0) {
        tops[wave] = wave_top;
        partial[wave] = a;
    }
    __syncthreads();
    float row_top = tops[0];
#pragma unroll
    for (int i = 1; i < kRowWaves; ++i) row_top = fmaxf(row_top, tops[i]);
    Sums r = {fmaxf(row_top, -kFar), 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kRowWaves; ++i) {
        Sums x = partial[i];
        move_to(x, r.m, c);
        r.s += x.s;
        r.t += x.t;
    }
    if (__builtin_fabsf(row_top) >= kFar && __builtin_fabsf(row_top) < __builtin_inff()) {
        __syncthreads();
        a = Sums{row_top, 0.0f, 0.0f};
        for (int i = begin + tid; i < end; i += kRowThreads) add(a, (to_float(logits[i]) - row_top) * c);
        a.s = wave_sum(a.s);
        a.t = wave_sum(a.t);
        if (lane == 0) partial[wave] = a;
        __syncthreads();
        r = Sums{row_top, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < kRowWaves; ++i) {
            r.s += partial[i].s;
            r.t += partial[i].t;
        }
    }

    int n = 0;
    if constexpr (kCap > 0) {
        look();
        // All candidates from tau on, one behind the other.
        uint64_t mine[kCap / 64];
        int kept = 0;
#pragma unroll
        for (int i = 0; i < kCap / 64; ++i) {
            mine[i] = 64 * i + lane < count ? list[64 * i + lane] : 0;
            if ((uint32_t)(mine[i] >> 32) < tau) mine[i] = 0;
            kept += __builtin_popcountll(__ballot(mine[i] != 0));
        }
        if (lane == 0) counts[wave] = kept;
        __syncthreads();
        int at = 0;
#pragma unroll
        for (int i = 0; i < kRowWaves; ++i) {
            at += i < wave ? counts[i] : 0;
            n += counts[i];
        }
        at = uniform(at);
#pragma unroll
        for (int i = 0; i < kCap / 64; ++i) {
            const unsigned long long here = __ballot(mine[i] != 0);
            if (mine[i] != 0) lists[at + __builtin_popcountll(here & ((1ull << lane) - 1))] = mine[i];
            at += __builtin_popcountll(here);
        }
        __syncthreads();
        sort_candidates<kRowThreads>(lists, n, kRowWaves * kCap, tid);
    }
    if (parts > 1) {
        const PartSpace ws = part_space(prm.workspace, prm.rows, parts);
        if (tid == 0) *reinterpret_cast<f32x4_t*>(ws.sums + 4 * (int64_t)blockIdx.x) = f32x4_t{row_top, r.s, r.t, 0.0f};
        if constexpr (kCap > 0)
            for (int i = tid; i < k; i += kRowThreads) ws.candidates[(int64_t)blockIdx.x * k + i] = i < n ? lists[i] : 0;
        return;
    }
    const float log_s = __builtin_amdgcn_logf(r.s) * kLn2;
    write_sums<T>(prm, row, r, log_s, tid);
    if constexpr (kCap > 0) write_top(prm, row, lists, n, r.m, log_s, tid, kRowThreads);
}

// A row's parts put together, a workgroup per row.
template <typename T>
__global__ __launch_bounds__(kRowThreads) void logprobs_merge_kernel(LogprobsParams prm, int parts) {
    __shared__ uint64_t list[kMostMerged];
    __shared__ int total;
    const int tid = threadIdx.x, row = blockIdx.x, k = prm.top_k;
    const PartSpace ws = part_space(prm.workspace, prm.rows, parts);
    const float* const sums = ws.sums + (int64_t)row * parts * 4;
    const uint64_t* const from = ws.candidates + (int64_t)row * parts * k;
    Sums r = {kNegInf, 0.0f, 0.0f};
    uint64_t least = 1;              // k candidates of one part are that good
    for (int p = 0; p < parts; ++p) {
        r.m = fmaxf(r.m, sums[4 * p]);
        if (k > 0) {
            const uint64_t last = from[(int64_t)p * k + k - 1];
            least = last > least ? last : least;
        }
    }
    for (int p = 0; p < parts; ++p) {
        Sums x = {sums[4 * p], sums[4 * p + 1], sums[4 * p + 2]};
        move_to(x, r.m, prm.scale_log2);
        r.s += x.s;
        r.t += x.t;
    }
    const float log_s = __builtin_amdgcn_logf(r.s) * kLn2;
    write_sums<T>(prm, row, r, log_s, tid);
    if (k == 0) return;
    if (tid == 0) total = 0;
    __syncthreads();
    for (int i = tid; i < parts * k; i += kRowThreads) {
        const uint64_t c = from[i];
        if (c >= least) list[atomicAdd(&total, 1)] = c;
    }
    __syncthreads();
    const int n = total;
    sort_candidates<kRowThreads>(list, n, kMostMerged, tid);
    write_top(prm, row, list, n, r.m, log_s, tid, kRowThreads);
}

template <typename T>
hipError_t launch_type(const LogprobsParams& prm, const LogprobsCut& cut, hipStream_t stream) {
    const dim3 grid((unsigned)((int64_t)prm.rows * cut.parts));
    hipError_t e;
    if (prm.top_k == 0) e = launch(logprobs_kernel<T, 0>, grid, kRowThreads, stream, prm, cut.parts, cut.part_size);
    else if (prm.top_k <= 64) e = launch(logprobs_kernel<T, 256>, grid, kRowThreads, stream, prm, cut.parts, cut.part_size);
    else e = launch(logprobs_kernel<T, 1024>, grid, kRowThreads, stream, prm, cut.parts, cut.part_size);
    if (e != hipSuccess || cut.parts == 1) return e;
    return launch(logprobs_merge_kernel<T>, dim3((unsigned)prm.rows), kRowThreads, stream, prm, cut.parts);
}

}  // namespace

LogprobsCut logprobs_cut(int rows, int vocab, int top_k) {
    int parts = 512 / rows;
    if (parts > vocab / kLeastPart) parts = vocab / kLeastPart;
    if (top_k > 0 && parts > kMostMerged / top_k) parts = kMostMerged / top_k;
    if (parts <= 1) return LogprobsCut{1, vocab, 0};
    const int steps = (vocab + kStep - 1) / kStep, size = (steps + parts - 1) / parts * kStep;
    parts = (vocab + size - 1) / size;
    return LogprobsCut{parts, size, parts > 1 ? (size_t)rows * parts * (16 + 8 * (size_t)top_k) : 0};
}

hipError_t launch_logprobs(const LogprobsParams& prm, const LogprobsCut& cut, hipStream_t stream) {
    switch (prm.dtype) {
        case XBEAM_BF16: return launch_type<Bf16>(prm, cut, stream);
        case XBEAM_FP16: return launch_type<__half>(prm, cut, stream);
        default: return launch_type<float>(prm, cut, stream);
    }
}

}  // namespace xattn
