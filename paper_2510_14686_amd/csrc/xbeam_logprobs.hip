// Log-probabilities of given tokens, entropy and the top alternatives of rows of logits (xbeam_logprobs), in one pass.
//
//   x = scale * logit;  s = sum exp(x - m), t = sum (x - m) exp(x - m);  lse = m + ln s;  lp = x - lse;  H = ln s - t / s
//
// A row is read once.  Every lane keeps m (its own maximum), s and t of its values, moved on when m moves, and the lanes' are put together at
// the end.  Long rows are bound by the instructions beside the reading, eleven per value: 4096 rows of 131072 bf16 logits, 5 alternatives, 191
// us, 5.6 TB/s, the vector units busy 99 % of the time.  Short rows with many alternatives are bound by picking and ordering them: 1024 rows of
// 8192 fp32 logits, 512 alternatives, 25 us, of which the sums take 9, marking what may be one of the best 6, picking 6 and ordering 4.
//
// Alternatives: a lane's maximum is there anyway, and if in each of some waves ceil(k / 8) lanes have a maximum of tau or more, and
// those are k in all, so have k values of the row: what is below tau is none of the k.  So of every chunk of 16 bytes only the maximum
// is compared with tau; a chunk that passes goes to its wave's list in LDS, by (maximum, place).  tau rises as the row is read, and
// of random rows a few times k chunks pass.  A list that is full (a row that ascends, or whose values are all equal) is cut to its k best
// chunks.  The k best values are in the k best chunks: a chunk behind k others has k values ahead of all of its own.  These are read
// again at the end, and their values put into order.  Order everywhere: value descending, then index ascending, as one 64-bit number.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/xbeam.h"
#include "xattn_device.h"
#include "xattn_launch.h"
#include "xbeam_logprobs.h"

namespace xattn {
namespace {

constexpr int kVals = kLoads * kStep / 64;       // a lane's values in a round
constexpr int kAtOnce = -1;
// Rows whose maximum, in log2 units, is this far from 0 are summed up in a second pass, of differences of logits: a reference is off by half of its
// last digit, which is up to 2^-1 here.
constexpr float kFar = 16777216.0f;

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

// Sixteen bytes of a row, which may begin anywhere.
typedef uint32_t words_at_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t words_at_4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T> struct Chunk {
    static constexpr int kCount = 16 / (int)sizeof(T);
    u32x4_t x;
    __device__ __forceinline__ void load(const T* p) {
        using words = typename std::conditional<sizeof(T) == 4, words_at_4, words_at_2>::type;
        x = __builtin_nontemporal_load(reinterpret_cast<const words*>(p));
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(x[i]);
        else if constexpr (std::is_same<T, Bf16>::value) return i & 1 ? bf16_hi(x[i >> 1]) : bf16_lo(x[i >> 1]);
        else return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? x[i >> 1] >> 16 : x[i >> 1]));
    }
};

// s and t of some values, and what they are relative to.  While a row is read that is the reference r = m * c as rounded: y = x * c - r is one
// operation per value, whose terms belong to r itself, so that the sums of lanes and waves meet at the differences of their r, whatever
// m * c lost in rounding.  (Taken for m * c, r is off by 2^-24 of it: logits 10^5 from 0 had log-probabilities 5e-3 off.)  A whole row's sums are
// relative to its maximum m.
struct Sums {
    float m, s, t;
};
__device__ __forceinline__ void move_by(Sums& a, float m, float d) {      // d: from there to m in log2 units
    d = fmaxf(d, -1e30f);
    const float f = fast_exp2(d);
    a.t = f * (a.t + d * a.s);
    a.s *= f;
    a.m = m;
}
__device__ __forceinline__ void move_reference(Sums& a, float r) { move_by(a, r, a.m - r); }
__device__ __forceinline__ void move_to(Sums& a, float m, float c) { move_by(a, m, (a.m - m) * c); }
// From the reference of m to m itself.  Divided by the weight that m has, the sum is 1 at least, and exactly 1 where nothing is beside m.
__device__ __forceinline__ void settle(Sums& a, float m, float c) {
    const float d = __builtin_fmaf(m, c, -a.m), w = fast_exp2(d);
    a.t = (a.t - d * a.s) / w;
    a.s /= w;
    a.m = m;
}
__device__ __forceinline__ void add(Sums& a, float y) {      // y = x * c - r
    const float e = fast_exp2(y);
    a.s += e;
    a.t = __builtin_fmaf(e, fmaxf(y, -1000.0f), a.t);        // e is 0 from -150 on, and -inf times that no number
}

// How many of the lanes in `lanes` are below this one.
__device__ __forceinline__ int before(unsigned long long lanes) {
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0u));
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
        if (c[i] >= least) list[at + before(keep)] = c[i];
        at += __builtin_popcountll(keep);
    }
    __builtin_amdgcn_wave_barrier();
    return least;
}

// The r-th largest of the lanes' keys, of which each has two, or a little less (16 bits of it).
__device__ __forceinline__ uint32_t nth_of_two(uint32_t one, uint32_t other, int r) {
    uint32_t at = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t trial = at | 1u << bit;
        if (__builtin_popcountll(__ballot(one >= trial)) + __builtin_popcountll(__ballot(other >= trial)) >= r) at = trial;
    }
    return at;
}
// The key of the r-th largest of the lanes' values, or a little less.
__device__ __forceinline__ uint32_t nth_key(float x, int r) {
    if (r <= 4) {      // a few times the largest of those left; lanes that share it count together
        float best = wave_max(x);
        for (int left = r - __builtin_popcountll(__ballot(x == best)); left > 0; left -= __builtin_popcountll(__ballot(x == best))) {
            x = x == best ? kNegInf : x;
            if (__ballot(x > kNegInf) == 0) return 0u;
            best = wave_max(x);
        }
        return order_key(best);
    }
    return nth_of_two(order_key(x), 0u, r);
}

// A thread's candidates: a bit of `on` for each that counts.
template <int kRegs> struct Candidates {
    static constexpr int kCount = kRegs;
    uint64_t c[kRegs];
    uint32_t on;
    __device__ __forceinline__ uint32_t key(int i) const { return (uint32_t)(c[i] >> 32); }
    __device__ __forceinline__ uint32_t place(int i) const { return (uint32_t)c[i]; }
};
// The same of values whose places follow from where their chunks are: half the registers.
template <int kRegs, int kChunk> struct Values {
    static constexpr int kCount = kRegs;
    uint32_t keys[kRegs];
    int from[kRegs / kChunk];
    uint32_t on;
    __device__ __forceinline__ uint32_t key(int i) const { return keys[i]; }
    __device__ __forceinline__ uint32_t place(int i) const { return ~(uint32_t)(from[i / kChunk] + i % kChunk); }
};
template <typename Set> __device__ __forceinline__ uint64_t get(const Set& set, int i) { return (uint64_t)set.key(i) << 32 | set.place(i); }

// What the workgroup's threads need of LDS to pick and order candidates.
struct PickSpace {
    uint32_t bins[3][256];       // one counts, one is clear for the next round, one may still be read
    int counts[kMostWaves];
    uint64_t list[kMaxTopK + 8];
};

// Leaves the k best of the threads' candidates (more than k of them) on, and no others: their keys eight bits at a time
// from the top, each round counting the candidates that agree with the k-th so far by their next eight bits; then, where several share the
// k-th's key, their places likewise.  low: a key that none is below; bits: of the largest difference from it.  Returns the least that is left.
// Called by all threads.
template <int kWaves, typename Set>
__device__ __forceinline__ uint64_t keep_best(Set& mine, int k, uint32_t low, int bits, PickSpace& ws, int tid) {
    const int lane = tid & 63;
    int need = k, round = 0;
    for (int i = tid; i < 256; i += 64 * kWaves) ws.bins[0][i] = 0;
    __syncthreads();
    // The k-th of digits(i), whose `shift` lowest bits are open where that is enough to tell the k best.
    auto find = [&](auto digits, auto counts, int& shift) {
        uint32_t prefix = 0;
        for (;; ++round) {
            const int width = shift < 8 ? shift : 8;
            shift -= width;
            uint32_t* const bins = ws.bins[round % 3];
#pragma unroll
            for (int i = 0; i < Set::kCount; ++i) {
                const uint32_t d = digits(i) >> shift;
                if (counts(i) && d >> width == prefix) atomicAdd(bins + (d & ((1u << width) - 1)), 1u);
            }
            for (int i = tid; i < 256; i += 64 * kWaves) ws.bins[(round + 1) % 3][i] = 0;
            __syncthreads();
            // Lane l has the bins 255 - 4 l and the three below: the scan counts from the top.
            const int first = 252 - 4 * lane;
            int n[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                n[i] = (int)bins[first + 3 - i];
                sum += n[i];
            }
            const int higher = wave_incl_scan_i(sum) - sum;
            const unsigned long long hit = __ballot(higher < need && higher + sum >= need);
            const int at = __builtin_ctzll(hit | 1ull << 63);
            int above = higher, digit = first + 3, count = n[0];
#pragma unroll
            for (int i = 1; i < 4; ++i)
                if (above + count < need) {
                    above += count;
                    count = n[i];
                    digit = first + 3 - i;
                }
            need -= __builtin_amdgcn_readlane(above, at);
            count = __builtin_amdgcn_readlane(count, at);
            prefix = prefix << width | (uint32_t)__builtin_amdgcn_readlane(digit, at);
            if (count == need || shift == 0) {
                ++round;
                if (count == need) need = 0;
                return prefix << shift;
            }
        }
    };
    int shift = bits;
    const uint32_t key = low + find([&](int i) { return mine.key(i) - low; }, [&](int i) { return (mine.on >> i & 1) != 0; }, shift);
    uint64_t least = (uint64_t)key << 32;
    if (need > 0) {
        shift = 32;
        least |= find([&](int i) { return mine.place(i); }, [&](int i) { return (mine.on >> i & 1) != 0 && mine.key(i) == key; }, shift);
    }
#pragma unroll
    for (int i = 0; i < Set::kCount; ++i) mine.on &= get(mine, i) >= least ? ~0u : ~(1u << i);
    __syncthreads();
    return least;
}

// How many candidates are ranked by counting the better ones, a thread each; of more a bitonic network is faster.
template <int kWaves>
constexpr int kRanked = kWaves >= kRowWaves ? 256 : 128;
// How many candidates are kept where k are asked for.
template <int kWaves>
__device__ __forceinline__ int most_kept(int k) { return k <= kRanked<kWaves> ? kRanked<kWaves> : kMaxTopK; }

// How many of the list's n candidates are better; it goes on with up to 7 zeros.
__device__ __forceinline__ int rank_of(uint64_t c, const uint64_t* list, int n) {
    int rank = 0;
    for (int j = 0; j < n; j += 8) {
        uint64_t y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = list[j + i];
#pragma unroll
        for (int i = 0; i < 8; ++i) rank += y[i] > c;
    }
    return rank;
}

// Puts the threads' candidates, or the k best where they are more than most_kept(k), into ws.list, in no order, and returns how many
// there are.  least: none is below, raised to the least of the k best; bits: of the largest difference of a key from that one's.  Called
// by all threads, which find the list ready.
template <int kWaves, typename Set>
__device__ __forceinline__ int gather_best(Set& mine, int k, uint64_t& least, int bits, PickSpace& ws, int tid) {
    const int lane = tid & 63, wave = uniform(tid >> 6);
    int n = 0, at = 0;
    for (bool again = true;; again = false) {
        const int own = __builtin_popcount(mine.on), upto = wave_incl_scan_i(own);
        if (lane == 63) ws.counts[wave] = upto;
        __syncthreads();
        n = 0;
        at = upto - own;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            at += i < wave ? ws.counts[i] : 0;
            n += ws.counts[i];
        }
        n = uniform(n);
        if (!again || n <= most_kept<kWaves>(k)) break;
        least = keep_best<kWaves>(mine, k, (uint32_t)(least >> 32), bits, ws, tid);
    }
#pragma unroll
    for (int i = 0; i < Set::kCount; ++i)
        if (mine.on >> i & 1) ws.list[at++] = get(mine, i);
    if (n <= kRanked<kWaves> && tid < 8) ws.list[n + tid] = 0;      // ranks are counted eight at a time
    __syncthreads();
    return n;
}

// The value of lane `this one ^ kJ`.
template <int kJ>
__device__ __forceinline__ uint32_t other_lane(uint32_t x, int lane) {
    if constexpr (kJ == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true);         // quad_perm [1,0,3,2]
    else if constexpr (kJ == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true);    // quad_perm [2,3,0,1]
    else if constexpr (kJ == 4) return (uint32_t)__builtin_amdgcn_ds_swizzle((int)x, 4 << 10 | 0x1f);
    else if constexpr (kJ == 8) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, true);   // row_ror:8
    else {
        const u32x2_t t = kJ == 16 ? __builtin_amdgcn_permlane16_swap(x, x, false, false) : __builtin_amdgcn_permlane32_swap(x, x, false, false);
        const uint32_t t0 = t.x, t1 = t.y;
        return lane & kJ ? t0 : t1;
    }
}
// The last steps of a bitonic merge of runs of kSize lanes; descending where `down`.
template <int kSize>
__device__ __forceinline__ void sort_step(uint64_t& x, int lane, bool down) {
    if constexpr (kSize > 1) {
        constexpr int kJ = kSize / 2;
        const uint64_t y = (uint64_t)other_lane<kJ>((uint32_t)(x >> 32), lane) << 32 | other_lane<kJ>((uint32_t)x, lane);
        x = (x > y) == (down == ((lane & kJ) == 0)) ? x : y;
        sort_step<kJ>(x, lane, down);
    }
}

// Calls put(rank, candidate) for every one of the threads' candidates, or for the best of them, k at least; returns how many
// it was called for.  Called by all threads, which are done with ws.list.
template <int kWaves, typename Set, typename Put>
__device__ __forceinline__ int rank_candidates(Set& mine, int k, uint64_t least, int bits, PickSpace& ws, int tid, Put put) {
    const int lane = tid & 63, wave = uniform(tid >> 6);
    const int n = gather_best<kWaves>(mine, k, least, bits, ws, tid);
    if (n <= kRanked<kWaves>) {
        if (wave * 64 < n) {
            const uint64_t x = tid < n ? ws.list[tid] : 0;
            const int rank = rank_of(x, ws.list, n);
            if (tid < n) put(rank, x);
        }
        return n;
    }
    // A bitonic network, a candidate per thread: steps within a wave by lane exchanges, the six others through LDS.
    if constexpr (kWaves >= kRowWaves) {
        uint64_t x = tid < n ? ws.list[tid] : 0;
        sort_step<2>(x, lane, (tid & 2) == 0);
        sort_step<4>(x, lane, (tid & 4) == 0);
        sort_step<8>(x, lane, (tid & 8) == 0);
        sort_step<16>(x, lane, (tid & 16) == 0);
        sort_step<32>(x, lane, (tid & 32) == 0);
        sort_step<64>(x, lane, (tid & 64) == 0);
        for (int size = 128; size <= kMaxTopK; size <<= 1) {
            for (int j = size >> 1; j >= 64; j >>= 1) {
                __syncthreads();
                if (kWaves == kRowWaves || tid < kMaxTopK) ws.list[tid] = x;
                __syncthreads();
                const uint64_t y = ws.list[(tid ^ j) & (kMaxTopK - 1)];
                x = (x > y) == (((tid & size) == 0) == ((tid & j) == 0)) ? x : y;
            }
            sort_step<64>(x, lane, (tid & size) == 0);
        }
        if (tid < n) put(tid, x);
    }
    return n;
}

// The row's token and its logit, fetched ahead by the thread that writes what becomes of them.
struct Token {
    int id;
    float x;
};
template <typename T>
__device__ __forceinline__ Token fetch_token(const LogprobsParams& prm, int row, int tid) {
    Token t = {-1, __builtin_nanf("")};
    if (tid == 0 && prm.tokens) {
        t.id = prm.tokens[row];
        if (t.id >= 0 && t.id < prm.vocab) t.x = to_float(static_cast<const T*>(prm.logits)[row * prm.row_stride + t.id]);
    }
    return t;
}
__device__ __forceinline__ void write_sums(const LogprobsParams& prm, int row, const Sums& a, float log_s, const Token& token, int tid) {
    if (tid != 0) return;
    if (prm.lse) prm.lse[row] = a.m * prm.scale + log_s;
    if (prm.entropy) prm.entropy[row] = log_s - a.t / a.s * kLn2;
    if (prm.token_lp) prm.token_lp[row] = token.id < 0 ? 0.0f : (token.x - a.m) * prm.scale - log_s;
}
__device__ __forceinline__ void write_candidate(const LogprobsParams& prm, int row, int rank, uint64_t c, float m, float log_s) {
    if (rank >= prm.top_k) return;
    const int64_t at = (int64_t)row * prm.top_k + rank;
    prm.top_tok[at] = c ? (int)~(uint32_t)c : -1;
    prm.top_lp[at] = c ? (key_value((uint32_t)(c >> 32)) - m) * prm.scale - log_s : __builtin_nanf("");
}

// What a part of a row leaves in the workspace: its sums, and its candidates in order (0: none).
struct PartSpace {
    float* sums;               // [rows * parts, 4]
    uint64_t* candidates;      // [rows * parts, top_k]
};
__device__ __host__ __forceinline__ PartSpace part_space(char* ws, int rows, int parts) {
    return PartSpace{reinterpret_cast<float*>(ws), reinterpret_cast<uint64_t*>(ws + (size_t)rows * parts * 16)};
}

// A row, or one of its parts, per workgroup.  kCap: chunks that a wave's list holds; 0 without alternatives, kAtOnce for alternatives of
// rows (or parts) of one round, whose values stay in registers.  There eight waves share a SIMD at the price of a few spilled registers: 1024
// rows of 8192, 512 alternatives 26.4 -> 25.2 us, 4096 rows, 20 alternatives 47.1 -> 44.1.
template <typename T, int kCap, int kWaves>
__global__ __launch_bounds__(64 * kWaves, kCap == kAtOnce ? 8 : 4) void logprobs_kernel(LogprobsParams prm, int parts, int part_size) {
    constexpr bool kTop = kCap != 0, kList = kCap > 0;
    __shared__ uint64_t lists[kList ? kWaves * kCap : 1];
    __shared__ uint32_t taus[kWaves];
    __shared__ typename std::conditional<kTop, PickSpace, int>::type ws;
    __shared__ float tops[kWaves];
    __shared__ Sums partial[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int row = blockIdx.x / (unsigned)parts, part = blockIdx.x - row * parts;
    const int begin = part * part_size, end = prm.vocab - begin < part_size ? prm.vocab : begin + part_size;
    const T* const logits = static_cast<const T*>(prm.logits) + row * prm.row_stride;
    const float c = prm.scale_log2;
    const int k = prm.top_k;
    const Token token = parts == 1 ? fetch_token<T>(prm, row, tid) : Token{};
    // per_wave values of each of `enough` waves are k values: tau is what the enough-th best of the waves has per_wave of.
    const int with_values = (end - begin + kStep - 1) / kStep < kWaves ? (end - begin + kStep - 1) / kStep : kWaves;
    const int per_wave = (k + with_values - 1) / with_values, enough = per_wave > 0 ? (k + per_wave - 1) / per_wave : 0;
    uint64_t* const list = lists + (kList ? wave * kCap : 0);

    Sums a = {-kFar, 0.0f, 0.0f};
    float top = kNegInf;             // the lane's maximum
    uint32_t tau = 1, own = 1;       // least key to take: by all waves' maxima, by the own list
    int count = 0;
    // Largest keys so far -> tau.  The waves do not wait for each other: an older tau is a lower one.
    auto raise = [&]() {
        const uint32_t mine = wave < with_values ? nth_key(top, per_wave) : 0u;
        if (lane == 0) __hip_atomic_store(taus + wave, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    };
    auto look = [&]() {
        // (The last bits, made the wave's, keep them apart.)
        const uint32_t mine = lane < kWaves ? (__hip_atomic_load(taus + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) & ~(kWaves - 1u)) | (uint32_t)lane : 0u;
        int better = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) better += (uint32_t)__builtin_amdgcn_readlane((int)mine, i) > mine;
        const unsigned long long at = __ballot(lane < kWaves && better == enough - 1);
        const uint32_t all = (uint32_t)__builtin_amdgcn_readlane((int)mine, __builtin_ctzll(at | 1ull << 63)) & ~(kWaves - 1u);
        tau = all > tau ? all : tau;
    };
    // A round: kLoads steps per wave, the waves side by side in each, so that a short row has values for all, and a wave's rounds come in
    // order of their indices.  A chunk that would pass the row's end is read at the end, and its values that belong to the chunk
    // before it (`skip` of them, all if it lies behind the end) are left out.
    constexpr int kRound = kWaves * kLoads * kStep, kChunk = Chunk<T>::kCount, kChunks = kVals / kChunk, kPerStep = kStep / 64 / kChunk;
    const int rounds = (end - begin + kRound - 1) / kRound;
    auto nominal = [&](int round, int q) {
        return begin + round * kRound + ((q / kPerStep) * kWaves + wave) * kStep + (q % kPerStep) * (64 * kChunk) + lane * kChunk;
    };
    const bool tiny = prm.vocab < kChunk;      // no chunk fits: the first thread takes the values one by one
    const int last = begin + (rounds - 1) * kRound < end - kChunk ? begin + (rounds - 1) * kRound : end - kChunk;      // where the last round reads from
    Chunk<T> next[kChunks];
    uint32_t ahead[kChunks];                   // of a round's chunks, in bytes
#pragma unroll
    for (int q = 0; q < kChunks; ++q) ahead[q] = (uint32_t)(nominal(0, q) - begin) * (uint32_t)sizeof(T);
    auto fetch = [&](int round) {
        int from = begin + round * kRound;
        if (round == rounds - 1) {
            from = last;
#pragma unroll
            for (int q = 0; q < kChunks; ++q) {
                const int at = nominal(round, q) < end - kChunk ? nominal(round, q) : end - kChunk;
                ahead[q] = (uint32_t)(at - last) * (uint32_t)sizeof(T);
            }
        }
        const char* const base = reinterpret_cast<const char*>(logits + from);
#pragma unroll
        for (int q = 0; q < kChunks; ++q) next[q].load(reinterpret_cast<const T*>(base + ahead[q]));
    };
    float x[kVals];
    for (int round = 0; round < rounds; ++round) {
        if (tiny) {
#pragma unroll
            for (int i = 0; i < kVals; ++i) x[i] = tid == 0 && i < end ? to_float(logits[i]) : kNegInf;
        } else {
            fetch(round);
#pragma unroll
            for (int i = 0; i < kVals; ++i) x[i] = next[i / kChunk].get(i % kChunk);
            if (round + 1 == rounds) {
#pragma unroll
                for (int q = 0; q < kChunks; ++q) {
                    const int skip = nominal(round, q) - (last + (int)(ahead[q] / (uint32_t)sizeof(T)));
#pragma unroll
                    for (int i = 0; i < kChunk; ++i) x[q * kChunk + i] = i < skip ? kNegInf : x[q * kChunk + i];
                }
            }
        }
        float most[kChunks], all = kNegInf;
#pragma unroll
        for (int q = 0; q < kChunks; ++q) {
            most[q] = x[q * kChunk];
#pragma unroll
            for (int i = 1; i < kChunk; ++i) most[q] = fmaxf(most[q], x[q * kChunk + i]);
            all = fmaxf(all, most[q]);
        }
        if (__ballot(all > top) != 0) {
            top = fmaxf(top, all);
            move_reference(a, fmaxf(top * c, -kFar));
        }
#pragma unroll
        for (int i = 0; i < kVals; ++i) add(a, __builtin_fmaf(x[i], c, -a.m));
        if constexpr (kList) {
            if ((round & (round - 1)) == 0 && (round & 0x2aaaaaaa) == 0) {      // rounds 0, 1, 4, 16, ...
                raise();
                if (round == 0) __syncthreads();
                look();
            }
            const uint32_t low = tau > own ? tau : own;
            const float low_value = key_value(low);
            const bool any = low <= kLowKey;       // -inf counts, and what is left out has to be told from it
            if (!any && __ballot(all >= low_value) == 0) continue;
#pragma unroll
            for (int q = 0; q < kChunks; ++q) {
                const unsigned long long takes =
                    any ? __ballot(order_key(most[q]) >= low && nominal(round, q) < end) : __ballot(most[q] >= low_value);
                if (takes == 0) continue;
                if (count + 64 > kCap) {
                    // The k best chunks come before any of a later round whose maximum equals the least of them; not before the rest of
                    // this one, which are not in order: `low` stays.
                    own = (uint32_t)(cut_list<kCap>(list, count, k, lane) >> 32) + 1;
                    count = k;
                }
                if (takes >> lane & 1) list[count + before(takes)] = candidate(order_key(most[q]), nominal(round, q));
                count += __builtin_popcountll(takes);
            }
        }
    }

    // The lanes' sums, then the waves'.
    if constexpr (kList) raise();
    if constexpr (kCap == kAtOnce) {
        // All values are here: twice as many maxima, each of half of a lane's, put tau nearer to the k-th value.
        float one = x[0], other = x[kVals / 2];
#pragma unroll
        for (int i = 1; i < kVals / 2; ++i) {
            one = fmaxf(one, x[i]);
            other = fmaxf(other, x[kVals / 2 + i]);
        }
        const uint32_t mine = wave >= with_values ? 0u : per_wave <= 4 ? nth_key(top, per_wave) : nth_of_two(order_key(one), order_key(other), per_wave);
        if (lane == 0) taus[wave] = mine;
    }
    const float wave_top = wave_max(top);
    {
        move_reference(a, fmaxf(wave_top * c, -kFar));
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
    for (int i = 1; i < kWaves; ++i) row_top = fmaxf(row_top, tops[i]);
    Sums r = {fmaxf(row_top * c, -kFar), 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        Sums x = partial[i];
        move_reference(x, r.m);
        r.s += x.s;
        r.t += x.t;
    }
    if (__builtin_fabsf(row_top * c) < kFar) settle(r, row_top, c);
    else if (__builtin_fabsf(row_top) < __builtin_inff()) {
        __syncthreads();
        a = Sums{row_top, 0.0f, 0.0f};
        for (int i = begin + tid; i < end; i += 64 * kWaves) add(a, (to_float(logits[i]) - row_top) * c);
        a.s = wave_sum(a.s);
        a.t = wave_sum(a.t);
        if (lane == 0) partial[wave] = a;
        __syncthreads();
        r = Sums{row_top, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            r.s += partial[i].s;
            r.t += partial[i].t;
        }
    }

    const float log_s = __builtin_amdgcn_logf(r.s) * kLn2;
    const PartSpace to = part_space(prm.workspace, prm.rows, parts);
    if (parts == 1) write_sums(prm, row, r, log_s, token, tid);
    else if (tid == 0) *reinterpret_cast<f32x4_t*>(to.sums + 4 * (int64_t)blockIdx.x) = f32x4_t{row_top, r.s, r.t, 0.0f};
    if constexpr (kTop) {
        look();
        uint64_t least = (uint64_t)tau << 32;
        const int bits = 32 - __builtin_clz((order_key(row_top) - tau) | 1);
        auto put = [&](int rank, uint64_t c) {
            if (parts == 1) write_candidate(prm, row, rank, c, r.m, log_s);
            else if (rank < k) to.candidates[(int64_t)blockIdx.x * k + rank] = c;
        };
        if constexpr (!kList) {
            Values<kVals, kChunk> value;
            value.on = 0;
#pragma unroll
            for (int q = 0; q < kChunks; ++q) {
                const int from = tiny ? 0 : last + (int)(ahead[q] / (uint32_t)sizeof(T)), skip = nominal(0, q) - from, count = tiny ? end : kChunk;
                value.from[q] = from;
                uint32_t on = 0;
#pragma unroll
                for (int i = 0; i < kChunk; ++i) {
                    value.keys[q * kChunk + i] = order_key(x[q * kChunk + i]);
                    on |= value.keys[q * kChunk + i] >= tau ? 1u << i : 0u;
                }
                // (Values from `first` on count, and of a tiny row those that there are.)
                on &= skip < count ? (1u << count) - (1u << skip) : 0u;
                value.on |= on << (q * kChunk);
            }
            const int n = rank_candidates<kWaves>(value, k, least, bits, ws, tid, put);
            for (int i = n + tid; i < k; i += 64 * kWaves) put(i, 0);
            return;
        } else {
            Candidates<kCap / 64> mine;
            mine.on = 0;
#pragma unroll
            for (int i = 0; i < kCap / 64; ++i) {
                mine.c[i] = 64 * i + lane < count ? list[64 * i + lane] : 0;
                if (64 * i + lane < count && mine.key(i) >= tau) mine.on |= 1u << i;
            }
            const int chunks = gather_best<kWaves>(mine, k, least, bits, ws, tid);
            least &= ~0xffffffffull;      // places of chunks are not places of values
            // The chunks' values, a chunk per thread.
            static_assert(64 * kRowWaves >= kMaxTopK, "a thread for every chunk");
            const int first = tid < chunks ? (int)~(uint32_t)ws.list[tid] : end, from = first < end - kChunk ? first : end - kChunk;
            Chunk<T> chunk;
            chunk.load(logits + from);
            Values<kChunk, kChunk> value;
            value.from[0] = from;
            value.on = 0;
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                value.keys[i] = order_key(chunk.get(i));
                if (from + i >= first && from + i < end && value.keys[i] >= (uint32_t)(least >> 32) && value.keys[i] != 0) value.on |= 1u << i;
            }
            const int n = rank_candidates<kWaves>(value, k, least, bits, ws, tid, put);
            for (int i = n + tid; i < k; i += 64 * kWaves) put(i, 0);
        }
    }
}

// A row's parts put together, a workgroup per row.
template <typename T>
__global__ __launch_bounds__(64 * kRowWaves) void logprobs_merge_kernel(LogprobsParams prm, int parts) {
    __shared__ PickSpace ws;
    const int tid = threadIdx.x, lane = tid & 63, row = blockIdx.x, k = prm.top_k;
    const PartSpace from = part_space(prm.workspace, prm.rows, parts);
    const Token token = fetch_token<T>(prm, row, tid);
    const float* const sums = from.sums + (int64_t)row * parts * 4;
    const uint64_t* const candidates = from.candidates + (int64_t)row * parts * k;
    constexpr int kRegs = kMostMerged / (64 * kRowWaves);
    Candidates<kRegs> mine;
#pragma unroll
    for (int i = 0; i < kRegs; ++i) mine.c[i] = i * 64 * kRowWaves + tid < parts * k ? candidates[i * 64 * kRowWaves + tid] : 0;
    // Every wave by itself, a part per lane.
    float top = kNegInf;
    uint64_t least = 1, best = 0;    // k candidates of one part are that good; the best one
    for (int p = lane; p < parts; p += 64) {
        top = fmaxf(top, sums[4 * p]);
        if (k > 0) {
            const uint64_t first = candidates[(int64_t)p * k], last = candidates[(int64_t)p * k + k - 1];
            least = last > least ? last : least;
            best = first > best ? first : best;
        }
    }
    Sums r = {wave_max(top), 0.0f, 0.0f};
    for (int p = lane; p < parts; p += 64) {
        Sums x = {sums[4 * p], sums[4 * p + 1], sums[4 * p + 2]};
        move_to(x, r.m, prm.scale_log2);
        r.s += x.s;
        r.t += x.t;
    }
    r.s = wave_sum(r.s);
    r.t = wave_sum(r.t);
    const float log_s = __builtin_amdgcn_logf(r.s) * kLn2;
    write_sums(prm, row, r, log_s, token, tid);
    if (k == 0) return;
#pragma unroll
    for (int j = 32; j > 0; j >>= 1) {
        const uint64_t l = __shfl_xor(least, j, 64), b = __shfl_xor(best, j, 64);
        least = l > least ? l : least;
        best = b > best ? b : best;
    }
    mine.on = 0;
#pragma unroll
    for (int i = 0; i < kRegs; ++i)
        if (mine.c[i] >= least) mine.on |= 1u << i;
    auto put = [&](int rank, uint64_t x) { write_candidate(prm, row, rank, x, r.m, log_s); };
    const int n = rank_candidates<kRowWaves>(mine, k, least, 32 - __builtin_clz((uint32_t)(best >> 32) - (uint32_t)(least >> 32) | 1), ws, tid, put);
    for (int i = n + tid; i < k; i += 64 * kRowWaves) put(i, 0);
}

template <typename T>
hipError_t launch_type(const LogprobsParams& prm, const LogprobsCut& cut, hipStream_t stream) {
    const dim3 grid((unsigned)((int64_t)prm.rows * cut.parts));
    auto with = [&](auto cap, auto waves) {
        constexpr int kCap = decltype(cap)::value, kWaves = decltype(waves)::value;
        return launch(logprobs_kernel<T, kCap, kWaves>, grid, 64 * kWaves, stream, prm, cut.parts, cut.part_size);
    };
    const std::integral_constant<int, kRowWaves> many;
    const std::integral_constant<int, kFewWaves> few;
    const std::integral_constant<int, kMostWaves> most;
    const bool is_short = cut.parts == 1 && prm.vocab <= kFewWaves * kLoads * kStep, at_once = cut.part_size <= kAtOnceSize;
    const bool wide = grid.x <= kParts && cut.part_size > kManyRounds * kAtOnceSize;
    hipError_t e;
    const std::integral_constant<int, 0> none;
    if (prm.top_k == 0) e = is_short ? with(none, few) : wide ? with(none, most) : with(none, many);
    else if (is_short && prm.top_k <= 128) e = with(std::integral_constant<int, kAtOnce>(), few);
    else if (at_once) e = with(std::integral_constant<int, kAtOnce>(), many);
    else if (prm.top_k <= 64) e = wide ? with(std::integral_constant<int, 256>(), most) : with(std::integral_constant<int, 256>(), many);
    else e = wide ? with(std::integral_constant<int, 640>(), most) : with(std::integral_constant<int, 640>(), many);
    if (e != hipSuccess || cut.parts == 1) return e;
    return launch(logprobs_merge_kernel<T>, dim3((unsigned)prm.rows), 64 * kRowWaves, stream, prm, cut.parts);
}

}  // namespace

hipError_t launch_logprobs(const LogprobsParams& prm, const LogprobsCut& cut, hipStream_t stream) {
    switch (prm.dtype) {
        case XBEAM_BF16: return launch_type<Bf16>(prm, cut, stream);
        case XBEAM_FP16: return launch_type<__half>(prm, cut, stream);
        default: return launch_type<float>(prm, cut, stream);
    }
}

}  // namespace xattn
