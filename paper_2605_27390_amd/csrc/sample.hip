// Sampling: one token for each row of logits by temperature, top-k, top-p and min-p, from a given random number.
//
// All four filters keep a front part of the row's tokens in the order (larger logit, smaller id), which is that of the
// 64-bit keys of common.hpp; a filter is therefore a smallest key, and so is the drawn token: the key at which the
// cumulative weight of the kept ones passes u times their sum.  Such keys are found digit by digit from a histogram of the
// keys that agree so far, of numbers (top-k) or of weights (top-p, the draw).  Weights w = exp((z - z_max) / T) are computed
// in 64 bits and kept as whole multiples of 2^-43: their sums do not depend on an order, so that a histogram may be filled by
// atomics, and 2^20 of them fit 64 bits.  (They are off by 2^-44 each, and by a table to 2^-39 of themselves: sums to V 2^-44, and to as much
// again where slices' bins are joined.)  Measured on rows of 151,936: one in 19 us, 60 with top-k in 27, 960 of bf16 with top-p in 222.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "decode.hpp"

namespace evospec {
namespace {

constexpr int kThreads = 1024;
constexpr double kOne = 8796093022208.0;          // 2^43: a weight of 1

// exp(x ln 2) for x <= 0 by the series of exp around the nearest whole power of two: |f ln 2| <= 0.3466, whose 12th power
// over 12! is 6e-15
__device__ __forceinline__ double exp2_series(double x) {
    const double n = rint(x), g = (x - n) * 0.69314718055994530942;
    double p = 1.0 / 39916800.0;
    p = fma(p, g, 1.0 / 3628800.0);
    p = fma(p, g, 1.0 / 362880.0);
    p = fma(p, g, 1.0 / 40320.0);
    p = fma(p, g, 1.0 / 5040.0);
    p = fma(p, g, 1.0 / 720.0);
    p = fma(p, g, 1.0 / 120.0);
    p = fma(p, g, 1.0 / 24.0);
    p = fma(p, g, 1.0 / 6.0);
    p = fma(p, g, 0.5);
    p = fma(p, g, 1.0);
    p = fma(p, g, 1.0);
    return ldexp(p, (int)n);
}
// log2(e) / T, from the reciprocal by two steps of Newton's (a division is four times as many instructions, and every thread of a
// slice needs it for 20 logits)
__device__ __forceinline__ double log2e_over(float T) {
    const double t = (double)T;
    double r = __builtin_amdgcn_rcp(t);
    r = fma(r, fma(-t, r, 1.0), r);
    r = fma(r, fma(-t, r, 1.0), r);
    return 1.4426950408889634074 * r;
}
// the weight of a logit; c = log2(e) / T
__device__ __forceinline__ double weight(float z, float z_max, double c) {
    if (z == z_max) return 1.0;
    const double x = ((double)z - (double)z_max) * c;
    return x > -45.0 ? exp2_series(x) : 0.0;
}
__device__ __forceinline__ u64 fixed(double w) { return (u64)(w * kOne + 0.5); }

// Products of a sum of weights with a fraction, exact: a float is a whole number of 24 bits over a power of two.
// floor(f x), f in [0, 1)
__device__ __forceinline__ u64 share(float f, u64 x, bool up) {
    const uint32_t bits = __float_as_uint(f), e = bits >> 23, man = e ? (bits & 0x7fffffu) | 0x800000u : bits & 0x7fffffu;
    const int down = 150 - (int)(e ? e : 1);                     // f = man / 2^down, down >= 24
    const unsigned __int128 y = (unsigned __int128)man * x;
    if (down >= 127) return up && y != 0 ? 1 : 0;
    const u64 q = (u64)(y >> down);
    return q + (up && ((unsigned __int128)q << down) != y ? 1 : 0);
}
// the least whole number >= f x, at least 1 and at most x (f < 1)
__device__ __forceinline__ u64 share_up(float f, u64 x) {
    const u64 s = f > 0.f ? share(f, x, true) : 0;
    return s < 1 ? 1 : s;
}
// the least whole number > f x, at most x (which NaN does not pass either)
__device__ __forceinline__ u64 share_past(float f, u64 x) {
    if (!(f < 1.f)) return x;
    return f > 0.f ? share(f, x, false) + 1 : 1;
}

template <int TYPE>
__device__ __forceinline__ float logit(const void* row, int i) {
    if constexpr (TYPE == EVOSPEC_FP32) return static_cast<const float*>(row)[i];
    else if constexpr (TYPE == EVOSPEC_FP16) return (float)static_cast<const _Float16*>(row)[i];
    else return (float)static_cast<const __bf16*>(row)[i];
}

__device__ __forceinline__ u64 shfl_xor64(u64 x, int s) {
    return (u64)(uint32_t)__shfl_xor((int)(uint32_t)x, s) | (u64)(uint32_t)__shfl_xor((int)(uint32_t)(x >> 32), s) << 32;
}
__device__ __forceinline__ u64 sum_eight(u64 x, int lane) {
    x += (u64)xor_lane<1>((uint32_t)(x >> 32), lane) << 32 | xor_lane<1>((uint32_t)x, lane);
    x += (u64)xor_lane<2>((uint32_t)(x >> 32), lane) << 32 | xor_lane<2>((uint32_t)x, lane);
    x += (u64)xor_lane<4>((uint32_t)(x >> 32), lane) << 32 | xor_lane<4>((uint32_t)x, lane);
    return x;
}
__device__ __forceinline__ u64 first_lane(u64 x) {
    return (u64)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x) | (u64)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(x >> 32)) << 32;
}
template <class F>
__device__ __forceinline__ u64 reduce_all(u64 x, u64* s_part, F f) {
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) x = f(x, shfl_xor64(x, s));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = x;
    __syncthreads();
    x = s_part[0];
    for (int w = 1; w < kThreads / 64; ++w) x = f(x, s_part[w]);
    return x;
}

__device__ __forceinline__ u64 shfl_up64(u64 x, int s) {
    return (u64)(uint32_t)__shfl_up((int)(uint32_t)x, s) | (u64)(uint32_t)__shfl_up((int)(uint32_t)(x >> 32), s) << 32;
}

// The key of the row at which the cumulative measure of the keys from the largest down reaches `target` (>= 1; no more than
// the measure of all keys >= low), 11 bits of it at a time.  each(f) calls f(key, logit) for every key of the row; measure(logit)
// is asked for those alone that agree with what is known.
constexpr int kDigit = 11, kDigits2 = 1 << kDigit;
template <class EachKey, class Measure>
__device__ __forceinline__ u64 find_key(u64 low, u64 target, u64* s_hist, u64* s_part, u64* s_pick, EachKey each, Measure measure) {
    const int tid = threadIdx.x, lane = tid & 63;
    u64 prefix = 0, mask = 0;
    for (int top = 64; top > 0; top -= kDigit) {
        const int shift = top > kDigit ? top - kDigit : 0, width = top - shift;
        for (int i = tid; i < kDigits2; i += kThreads) s_hist[i] = 0;
        __syncthreads();
        each([&](u64 key, float z) {
            if (key >= low && (key & mask) == prefix) {
                const u64 w = measure(z);
                if (w) atomicAdd(&s_hist[(key >> shift) & ((1u << width) - 1)], w);
            }
        });
        __syncthreads();
        // two digits a thread, the largest first
        const int d = kDigits2 - 1 - 2 * tid;
        const u64 a = s_hist[d], b = s_hist[d - 1];
        u64 run = a + b;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const u64 x = shfl_up64(run, s);
            if (lane >= s) run += x;
        }
        if (lane == 63) s_part[tid >> 6] = run;
        __syncthreads();
        run -= a + b;
        for (int w = 0; w < tid >> 6; ++w) run += s_part[w];
        if (run < target && run + a + b >= target) {
            const bool first = run + a >= target;
            s_pick[0] = (u64)(first ? d : d - 1);
            s_pick[1] = target - run - (first ? 0 : a);
        }
        __syncthreads();
        prefix |= s_pick[0] << shift;
        target = s_pick[1];
        mask |= (u64)((1u << width) - 1) << shift;
        __syncthreads();
    }
    return prefix;
}
static_assert(2 * kThreads == kDigits2, "two digits a thread");

// A row by one workgroup, read again for every digit of a key: for rows whose tokens the bins below do not separate.
template <int TYPE>
__device__ __forceinline__ void sample_by_digits(const SampleArgs& A, int m, u64* s_hist, u64* s_part, u64* s_pick) {
    const char* row = static_cast<const char*>(A.logits) + (long long)m * A.stride * (TYPE == EVOSPEC_FP32 ? 4 : 2);
    const float T = A.temperature ? A.temperature[m] : 1.f;
    auto each = [&](auto f) {
        // (eight loads at a time: one after the other a pass over 151,936 logits took 56 us)
        for (int first = threadIdx.x; first < A.V; first += 8 * kThreads) {
            float z[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = first + j * kThreads < A.V ? logit<TYPE>(row, first + j * kThreads) : -__builtin_inff();
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
                const float v = z[0];
#pragma unroll
                for (int e = 0; e < 7; ++e) z[e] = z[e + 1];     // (a loop, not eight copies of what is called)
                const int i = first + j * kThreads;
                if (v > -__builtin_inff()) f(make_key(v, A.ids ? A.ids[i] : i), v);
            }
        }
    };
    u64 top = 0, n = 0;
    each([&](u64 key, float) { top = key > top ? key : top; ++n; });
    top = reduce_all(top, s_part, [](u64 a, u64 b) { return a > b ? a : b; });
    n = reduce_all(n, s_part, [](u64 a, u64 b) { return a + b; });
    if (top == 0) {
        if (threadIdx.x == 0) {
            A.out_ids[m] = -1;
            if (A.out_logprob) A.out_logprob[m] = __uint_as_float(0x7fc00000u);
        }
        return;
    }
    const float z_max = key_value(top);
    if (!(T > 0.f)) {
        if (threadIdx.x == 0) {
            A.out_ids[m] = key_id(top);
            if (A.out_logprob) A.out_logprob[m] = 0.f;
        }
        return;
    }
    const double c = 1.4426950408889634074 / (double)T;          // (any temperature: rows that are not regular come here)
    auto mass = [&](float z) { return fixed(weight(z, z_max, c)); };
    auto mass_from = [&](u64 low) {
        u64 sum = 0;
        each([&](u64 key, float z) { if (key >= low) sum += mass(z); });
        return reduce_all(sum, s_part, [](u64 a, u64 b) { return a + b; });
    };
    u64 low = 0;
    const int k = A.top_k ? A.top_k[m] : 0;
    if (k > 0 && (u64)k < n) low = find_key(low, (u64)k, s_hist, s_part, s_pick, each, [](float) { return (u64)1; });
    const float p = A.top_p ? A.top_p[m] : 1.f;
    if (p < 1.f) {
        const u64 all = mass_from(low);
        low = find_key(low, share_up(p, all), s_hist, s_part, s_pick, each, mass);
    }
    const float least = A.min_p ? A.min_p[m] : 0.f;
    if (least > 0.f) {
        u64 first = top;
        each([&](u64 key, float z) { if (key >= low && key < first && weight(z, z_max, c) >= (double)least) first = key; });
        low = reduce_all(first, s_part, [](u64 a, u64 b) { return a < b ? a : b; });
    }
    const u64 total = mass_from(low);
    const u64 key = find_key(low, share_past(A.u[m], total), s_hist, s_part, s_pick, each, mass);
    if (threadIdx.x == 0) {
        A.out_ids[m] = key_id(key);
        if (A.out_logprob) {
            const double x = key_value(key) == z_max ? 0.0 : ((double)key_value(key) - (double)z_max) / (double)T;
            A.out_logprob[m] = (float)(x - log((double)total / kOne));
        }
    }
}


// ---------------------------------------------------------------------------------------
// The fast way, four launches or two.
//
// 1. sample_bins_kernel, a workgroup for each slice of a row (kSlice logits at most, which stay in registers): the slice's
//    largest logit, and the weights of its tokens, summed in bins of 1 / kBins of a power of two below e = the next power of two
//    above that logit.  References are whole powers of two, so that slices' bins lie on one grid and their sums are joined by shifts.
// 2. sample_row_kernel, a workgroup for each row: the bins of all slices, joined (eight slices' loads at a time); in which bins top-k, top-p and min-p cut, and in which
//    the draw falls (a range of them where one depends on a cut inside a bin).  Greedy rows end here.
// 3. sample_pick_kernel, a workgroup for each part of a row again: tokens of those bins are put on the row's list.
// 4. sample_finish_kernel, a workgroup for each row: sorts the list, and goes through the filters with the list's tokens and the bins'
//    sums.
// Rows of a top-k up to kMostK need no weights but those of their k largest tokens: 1. lists the tokens that can be among them, and 2.
// ends the row.  Lists that are full (thousands of tokens within 1 / kBins of a power of two) leave the row to sample_by_digits.
constexpr int kBins = 32;                         // to a factor of 2
constexpr int kRange = 44;                        // factors of 2 that are kept,
constexpr int kFine = kBins * 28;                 // those behind the 28th have a bin each, which slices' references move as they move the
constexpr int kAll = kFine + kRange - 28;         // fine ones: what is in a bin of the row is what has weight there
constexpr int kPlaces = kRange * kBins;           // all of them fine
constexpr int kGroups = 5;                        // of 4 logits of a thread
constexpr int kSlice = kThreads * 4 * kGroups;
constexpr int kMostSlices = ((1 << 20) + kSlice - 1) / kSlice;
constexpr int kAtOnce = 8;                        // slices whose bins are joined side by side
constexpr int kList = 4096;                       // tokens of a row that are looked at one by one
constexpr int kStage = 1024;                      // of a slice that go to that list at once
constexpr int kMostK = 256;                       // top-k up to this goes by lists alone
constexpr int kSteps = 32;                        // to a factor of 2 in the table of powers: each has its own banks of LDS

struct RowState {
    double ref;                                   // exponent of the row's reference
    float z_max;
    int state;                                    // kOpen, kDone, kDigits
    int lo[3], hi[3];                             // bins lo[i] .. hi[i] are on the list
    int end_bin;                                  // the last bin in which the kept tokens can end
    int least_bin;                                // the last bin that can hold a weight of min-p
    int k_bin, k_left;                            // the bin that top-k cuts, and how many of it are kept; -1: none
};
enum { kOpen = 0, kDone = 1, kDigits = 2 };

struct SliceState {
    double ref;                                   // exponent of its reference; with lists the bound that they reach (see `missing`)
    u64 top;                                      // its largest logit as a key, greedy rows with its id; 0: no number there
    uint32_t n, pad;                              // tokens on its list
};

// A row's part of the workspace.
struct RowSpace {
    u64* mass;                                    // [slices][kAll]
    uint32_t* count;                              // [slices][kAll], where top-k asks for it
    SliceState* slice;                            // [slices]
    u64* before;                                  // [kAll + 1]: what the bins in front weigh
    RowState* row;
    uint32_t* ticket;                             // tokens on the list
    u64* list;                                    // [kList], in any order
};
__host__ __device__ inline size_t row_bytes(int slices) {
    const size_t n = (size_t)slices * (kAll * 12 + sizeof(SliceState)) + (kAll + 1) * 8 + sizeof(RowState) + 8 + kList * 8;
    return (n + 255) / 256 * 256;
}
__device__ __forceinline__ RowSpace row_space(char* ws, int m, int slices) {
    char* p = ws + (size_t)m * row_bytes(slices);
    RowSpace r;
    r.mass = reinterpret_cast<u64*>(p);           p += (size_t)slices * kAll * 8;
    r.slice = reinterpret_cast<SliceState*>(p);   p += (size_t)slices * sizeof(SliceState);
    r.before = reinterpret_cast<u64*>(p);         p += (kAll + 1) * 8;
    r.list = reinterpret_cast<u64*>(p);           p += kList * 8;
    r.row = reinterpret_cast<RowState*>(p);       p += sizeof(RowState);
    r.ticket = reinterpret_cast<uint32_t*>(p);    p += 8;
    r.count = reinterpret_cast<uint32_t*>(p);
    return r;
}

// Weights by table: with y = z log2(e) / T = k / kSteps + r, |r| <= 1 / (2 kSteps), and `ref` a whole power of two above the row's or
// slice's largest, w = 2^(y - ref) = 2^(-m / kSteps) 2^r, m = kSteps ref - k >= 0.  2^r by its series to the fourth power is off by
// 2^-39.  What bounds the bins is LDS, an addition to a bin for each logit: 151 us for 146 million logits of bf16 (183 when the tail had one
// bin for all, and 191 then with a table of 128 steps, whose reads meet in its banks).
struct Steps {
    int m;
    double r;
};
// x y + c with c in scalar registers (the compiler's choice copies c to vector registers first, 2 more instructions of 3)
__device__ __forceinline__ double fma_to(double x, double y, double c) {
    double d;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(d) : "v"(x), "v"(y), "s"(c));
    return d;
}
__device__ __forceinline__ Steps locate(float z, double c, int ref_steps) {
    const double magic = 6755399441055744.0 / kSteps;            // 1.5 * 2^52 / kSteps: k in the low bits
    const double zd = (double)z, t = fma_to(zd, c, magic);
    Steps s;
    s.r = fma(zd, c, -(t - magic));
    s.m = ref_steps - (int)(uint32_t)__double_as_longlong(t);
    return s;
}
__device__ __forceinline__ void fill_table(double* table) {
    if (threadIdx.x < kSteps) table[threadIdx.x] = kOne * exp2_series(-(double)threadIdx.x / kSteps);
}
// m < kRange kSteps
__device__ __forceinline__ u64 weight_of(Steps s, const double* table) {
    double first = 0.0096181291076284772;                        // ln(2)^k / k!
    asm("" : "+v"(first));                                       // (one vector register pair for all calls)
    double p = fma_to(s.r, first, 0.055504108664821580);
    p = fma_to(p, s.r, 0.24022650695910071);
    p = fma_to(p, s.r, 0.69314718055994531);
    p = fma(p, s.r, 1.0);
    const long long power = __double_as_longlong(table[s.m & (kSteps - 1)]);
    const uint32_t hi = (uint32_t)(power >> 32) - ((uint32_t)s.m / kSteps << 20);
    const double d = fma_to(__longlong_as_double((long long)((u64)hi << 32 | (uint32_t)power)), p, 4503599627370496.0);
    return (u64)__double_as_longlong(d) & 0xfffffffffffffull;    // 2^52 + the weight, rounded to a whole number
}
static_assert(kSteps == kBins, "a step is a bin");
// (the second is the smaller one from kFine on; kAll for what has no weight)
__device__ __forceinline__ int bin_of(int m) { return min(m, kFine - kFine / kBins + (int)((uint32_t)m / kBins)); }
// the least m of a bin
__device__ __forceinline__ int first_of(int bin) { return bin < kFine ? bin : (bin - (kFine - kFine / kBins)) * kBins; }
// logits below this have no weight; a little lower, as it is rounded to 32 bits: `m` decides
__device__ __forceinline__ float cut_of(double ref, float T) {
    const double z = (ref - kRange) * ((double)T * 0.69314718055994530942);
    return (float)(z - fabs(z) * 0x1p-22);
}
__device__ __forceinline__ bool has_weight(float z, float cut, Steps s) { return z >= cut && (uint32_t)s.m < (uint32_t)(kRange * kSteps); }

struct Slice {
    int first, last;
    // the logit that is the thread's e-th of group g: 4 in a row, the next group kThreads * 4 further on; short slices are dealt
    // out one by one, so that all wavefronts have a share of them
    __device__ __forceinline__ bool small() const { return last - first <= 4 * kThreads; }
    __device__ __forceinline__ int at(int g, int e) const {
        return small() ? first + (4 * g + e) * kThreads + (int)threadIdx.x : first + (g * kThreads + (int)threadIdx.x) * 4 + e;
    }
};
__device__ __forceinline__ Slice slice_of(int V, int slices, int j) {
    const int per = ((V + slices - 1) / slices + 3) / 4 * 4;     // (<= kSlice)
    return Slice{min(V, j * per), min(V, (j + 1) * per)};
}
// A thread's logits as they come: 16-bit types two to a word.
template <int TYPE>
struct RawSlice {
    static constexpr int kWords = TYPE == EVOSPEC_FP32 ? 4 : 2;
    uint32_t w[kGroups][kWords];
    __device__ __forceinline__ void load(const char* row, Slice S) {
        constexpr int kBytes = TYPE == EVOSPEC_FP32 ? 4 : 2;
        constexpr uint32_t kInf = TYPE == EVOSPEC_FP32 ? 0xff800000u : TYPE == EVOSPEC_FP16 ? 0xfc00u : 0xff80u;       // -inf
        const bool whole = (reinterpret_cast<uintptr_t>(row) & (4 * kBytes - 1)) == 0 && !S.small();
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int i = S.at(g, 0);
            if (whole && i + 4 <= S.last) {
                if constexpr (TYPE == EVOSPEC_FP32) {
                    const uint4 v = *reinterpret_cast<const uint4*>(row + (size_t)i * 4);
                    w[g][0] = v.x; w[g][1] = v.y; w[g][2] = v.z; w[g][3] = v.w;
                } else {
                    const uint2 v = *reinterpret_cast<const uint2*>(row + (size_t)i * 2);
                    w[g][0] = v.x; w[g][1] = v.y;
                }
            } else {
                uint32_t x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = kInf;
                    if (S.at(g, e) < S.last) {
                        if constexpr (TYPE == EVOSPEC_FP32) x[e] = reinterpret_cast<const uint32_t*>(row)[S.at(g, e)];
                        else x[e] = reinterpret_cast<const uint16_t*>(row)[S.at(g, e)];
                    }
                }
#pragma unroll
                for (int e = 0; e < kWords; ++e) w[g][e] = TYPE == EVOSPEC_FP32 ? x[e] : x[2 * e & 3] | x[(2 * e + 1) & 3] << 16;
            }
        }
    }
    __device__ __forceinline__ void give(float (&z)[kGroups][4]) const {
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (TYPE == EVOSPEC_FP32) {
                    z[g][e] = __uint_as_float(w[g][e]);
                } else {
                    const uint32_t x = w[g][e >> 1];
                    if constexpr (TYPE == EVOSPEC_BF16) z[g][e] = __uint_as_float(e & 1 ? x & 0xffff0000u : x << 16);
                    else z[g][e] = (float)__builtin_bit_cast(_Float16, (uint16_t)(x >> (16 * (e & 1))));
                }
            }
    }
};
template <int TYPE>
__device__ __forceinline__ void load_slice(const char* row, Slice S, float (&z)[kGroups][4]) {
    RawSlice<TYPE> raw;
    raw.load(row, S);
    raw.give(z);
}

// What bins can take: rows by their largest logit, the others go by digits.  Slices of such rows may lie a little past that (kRange factors of
// 2 are 31 temperatures), and are taken to twice as far.
__device__ __forceinline__ bool regular(float T, float z_max, float most = 0x1p22f) {
    return T < 0x1p60f && T > 0x1p-60f && fabsf(z_max) < T * most;
}
__device__ __forceinline__ bool regular_slice(float T, float top) { return regular(T, top, 0x1p23f); }

// A bound of a list that lacks tokens which equal it: a little larger, and the same in 32 bits.
__device__ __forceinline__ double missing(float bound) { return (double)bound + fabs((double)bound) * 0x1p-30 + 1e-300; }
// Rows of a small top-k: tokens of the slice that can be among the row's k largest, as keys in the place of its bins, and a
// bound that k of them reach.  Of every wavefront's 64 largest logits of a lane the q-th largest is taken, q times the wavefronts >= k, and
// the least of these: k logits reach it.  (k = 50 of 19,000: some 150 tokens pass.)  Where that is no bound, because a mask leaves some
// wavefronts nothing, or too many reach it, the slice's k-th largest logit is looked for bit by bit; what has no weight beside the slice's
// largest is not listed then either, nor what equals the k-th if that is too many (masked tokens that are all the same low value).
template <int TYPE>
__device__ __forceinline__ void list_largest(const SampleArgs& A, const float (&z)[kGroups][4], Slice S, int k, float top, float T,
                                             const char* row, const RowSpace& R, int j, u64* s_key, float* s_bound) {
    __shared__ uint32_t s_n;
    const int tid = threadIdx.x;
    float mine = -__builtin_inff();
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) mine = fmaxf(mine, z[g][e]);
    // (short slices have none for some wavefronts)
    const int waves = min(kThreads, S.last - S.first) / 64, q = waves > 0 ? (k + waves - 1) / waves : 65;
    const float b = q <= 64 ? ordered_to_f32(wave_kth_largest(f32_to_ordered(mine), q)) : -__builtin_inff();
    __syncthreads();                                             // (s_bound held the maxima)
    if ((tid & 63) == 0) s_bound[tid >> 6] = b;
    if (tid == 0) s_n = 0;
    __syncthreads();
    float bound = s_bound[0];
    for (int w = 1; w < waves; ++w) bound = fminf(bound, s_bound[w]);
    if (top > -__builtin_inff()) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (z[g][e] >= bound && z[g][e] > -__builtin_inff()) {
                    const uint32_t at = atomicAdd(&s_n, 1u);
                    const int i = S.at(g, e);
                    if (at < kAll) s_key[at] = make_key(z[g][e], A.ids ? A.ids[i] : i);
                }
    }
    __syncthreads();
    uint32_t n = s_n, full = 0;
    // (uniform; lists without a bound may be too many for the row's, if each is short enough)
    if (n > (uint32_t)(bound > -__builtin_inff() ? kAll : k)) {
        __shared__ uint32_t s_reach[32];
        if (tid < 32) s_reach[tid] = 0;
        __syncthreads();
        if (tid == 0) s_n = 0;
        // f(logit, column) for all of the slice's, from memory again, four loads at a time: kept in registers for this, they cost all
        // lists 30 that spill
        auto each = [&](auto f) {
#pragma unroll 1
            for (int first = S.first; first < S.last; first += 4 * kThreads) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = first + e * kThreads + tid;
                    v[e] = i < S.last ? logit<TYPE>(row, i) : -__builtin_inff();
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) f(v[e], first + e * kThreads + tid);
            }
        };
        uint32_t kth = 0;                                        // the largest that k logits reach: n > k are numbers
#pragma unroll 1
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t x = kth | 1u << bit;
            uint32_t reach = 0;
            each([&](float v, int) { reach += __popcll(__ballot(v == v && f32_to_ordered(v) >= x)); });
            if ((tid & 63) == 0) atomicAdd(&s_reach[bit], reach);
            __syncthreads();
            if (s_reach[bit] >= (uint32_t)k) kth = x;
        }
        bound = ordered_to_f32(kth);
        if (regular_slice(T, top)) bound = fmaxf(bound, cut_of(ceil((double)top * log2e_over(T)), T));
        for (;; full = 1) {                                      // (fewer than k are larger than the k-th)
            each([&](float v, int i) {
                if ((full ? v > bound : v >= bound) && v > -__builtin_inff()) {
                    const uint32_t at = atomicAdd(&s_n, 1u);
                    if (at < kAll) s_key[at] = make_key(v, A.ids ? A.ids[i] : i);
                }
            });
            __syncthreads();
            n = s_n;
            if (n <= (uint32_t)kAll) break;                      // (uniform)
            __syncthreads();
            if (tid == 0) s_n = 0;
            __syncthreads();
        }
    }
    for (int i = tid; i < (int)n; i += kThreads) R.mass[(size_t)j * kAll + i] = s_key[i];
    if (tid == 0) {
        R.slice[j] = SliceState{full ? missing(bound) : (double)bound, top > -__builtin_inff() ? make_key(top, 0) : 0, n, 0};
    }
}

// bf16 has 128 values to a factor of 2: a slice's logits between 2^-12 and 2^6, of either sign, are counted by value, and each value is
// weighed once, times its number (whole numbers: the sums are the same).  960 rows of 151,936 151 us one by one, 134 so, 64 rows 13.9 and
// 12.7.
constexpr int kLeastByValue = 8192;               // logits of a slice (8 rows of 50,000 in slices of 6,252 8.6 us by value, 6.8 one by one)
constexpr int kLowCode = 0x3980, kCodes = 0x4280 - kLowCode;    // upper halves of 2^-12 and 2^6

template <int TYPE, bool BY_VALUE>
__global__ __launch_bounds__(kThreads, 8) void sample_bins_kernel(SampleArgs A, char* ws, int slices) {
    __shared__ u64 s_mass[kAll];
    __shared__ uint32_t s_count[kAll];
    static_assert(!BY_VALUE || TYPE == EVOSPEC_BF16, "");
    __shared__ uint32_t s_num[BY_VALUE ? 2 * kCodes : 1];
    __shared__ double s_table[kSteps];
    __shared__ float s_max[kThreads / 64];
    __shared__ u64 s_part[kThreads / 64];
    const int m = blockIdx.x / slices, j = blockIdx.x % slices, tid = threadIdx.x, lane = tid & 63;
    const char* row = static_cast<const char*>(A.logits) + (long long)m * A.stride * (TYPE == EVOSPEC_FP32 ? 4 : 2);
    const Slice S = slice_of(A.V, slices, j);
    const RowSpace R = row_space(ws, m, slices);
    float z[kGroups][4];
    load_slice<TYPE>(row, S, z);
    const float T = A.temperature ? A.temperature[m] : 1.f;
    const bool counts = A.top_k && A.top_k[m] > 0;
    fill_table(s_table);
    for (int b = tid; b < kAll; b += kThreads) {
        s_mass[b] = 0;
        s_count[b] = 0;
    }
    if constexpr (BY_VALUE)
        for (int i = tid; i < 2 * kCodes; i += kThreads) s_num[i] = 0;
    if (j == 0 && tid == 0) *R.ticket = 0;
    float top = -__builtin_inff();
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, z[g][e]);
    top = wave_max(top, lane);
    if (lane == 0) s_max[tid >> 6] = top;
    __syncthreads();
    top = s_max[lane & (kThreads / 64 - 1)];
    top = wave_max(top, lane);
    if (!(T > 0.f)) {                                            // greedy: the largest key
        u64 best = 0;
        if (top > -__builtin_inff()) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (z[g][e] == top) {
                        const int i = S.at(g, e);
                        const u64 key = make_key(top, A.ids ? A.ids[i] : i);
                        best = key > best ? key : best;
                    }
        }
        best = reduce_all(best, s_part, [](u64 a, u64 b) { return a > b ? a : b; });
        if (tid == 0) R.slice[j] = SliceState{0.0, best, 0, 0};
        return;
    }
    if (counts && A.top_k[m] <= kMostK) {                        // (uniform)
        list_largest<TYPE>(A, z, S, A.top_k[m], top, T, row, R, j, s_mass, s_max);
        return;
    }
    const double c = log2e_over(T);
    const bool ok = top > -__builtin_inff() && regular_slice(T, top);
    const double ref = ok ? ceil((double)top * c) : 0.0;
    if (tid == 0) R.slice[j] = SliceState{ref, top > -__builtin_inff() ? make_key(top, 0) : 0, 0, 0};
    if (!ok) return;                                             // (uniform) nothing here, or a row for the digits
    const float cut = cut_of(ref, T);
    const int ref_steps = (int)ref * kSteps;
    auto add = [&](float x, uint32_t n) {
        if (x >= cut) {                                          // (not NaN)
            const Steps s = locate(x, c, ref_steps);
            if ((uint32_t)s.m >= (uint32_t)(kRange * kSteps)) return;
            const int b = bin_of(s.m);
            atomicAdd(&s_mass[b], n * weight_of(s, s_table));
            if (counts) atomicAdd(&s_count[b], n);
        }
    };
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (BY_VALUE) {
                const uint32_t u = __float_as_uint(z[g][e]), code = ((u >> 16) & 0x7fffu) - kLowCode;
                if (code < (uint32_t)kCodes) {
                    atomicAdd(&s_num[code + (u >> 31) * kCodes], 1u);
                    continue;
                }
            }
            add(z[g][e], 1);
        }
    if constexpr (BY_VALUE) {
        __syncthreads();
        for (int i = tid; i < 2 * kCodes; i += kThreads) {
            const uint32_t n = s_num[i], code = (uint32_t)(i < kCodes ? i : i - kCodes) + kLowCode;
            if (n) add(__uint_as_float((code | (i < kCodes ? 0u : 0x8000u)) << 16), n);
        }
    }
    __syncthreads();
    for (int b = tid; b < kAll; b += kThreads) {
        R.mass[(size_t)j * kAll + b] = s_mass[b];
        if (counts) R.count[(size_t)j * kAll + b] = s_count[b];
    }
}

// The same by value for many rows of bf16 without a top-k: a slice is `parts` times as long, taken in parts with the next one under way,
// and its values are weighed once.  The window goes down to 2^-22, and what lies outside of it is read again at the end, when the
// slice's largest logit is known.  960 rows of 151,936 in slices of 75,968: 134 and 92 us; 128 rows 22 and 19.
constexpr int kWideLow = 0x3480, kWideCodes = 0x4280 - kWideLow;
__global__ __launch_bounds__(kThreads, 8) void sample_wide_bins_kernel(SampleArgs A, char* ws, int slices, int parts) {
    __shared__ u64 s_mass[kAll];
    __shared__ uint32_t s_num[2 * kWideCodes];
    __shared__ double s_table[kSteps];
    __shared__ float s_max[kThreads / 64];
    __shared__ u64 s_part[kThreads / 64];
    __shared__ uint32_t s_outside;
    const int m = blockIdx.x / slices, j = blockIdx.x % slices, tid = threadIdx.x, lane = tid & 63;
    const char* row = static_cast<const char*>(A.logits) + (long long)m * A.stride * 2;
    const Slice S = slice_of(A.V, slices, j);
    const int per = ((S.last - S.first + parts - 1) / parts + 3) / 4 * 4;      // (<= kSlice)
    auto part = [&](int p) { return Slice{min(S.last, S.first + p * per), min(S.last, S.first + (p + 1) * per)}; };
    // f(logit, where it is: part, group, element) for all of the slice's
    auto each = [&](auto f) {
        RawSlice<EVOSPEC_BF16> raw;
        raw.load(row, part(0));
        for (int p = 0; p < parts; ++p) {
            float z[kGroups][4];
            raw.give(z);
            if (p + 1 < parts) raw.load(row, part(p + 1));
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) f(z[g][e], p, g, e);
        }
    };
    auto code_of = [](float z) { return ((__float_as_uint(z) >> 16) & 0x7fffu) - kWideLow; };
    const RowSpace R = row_space(ws, m, slices);
    const float T = A.temperature ? A.temperature[m] : 1.f;
    fill_table(s_table);
    for (int b = tid; b < kAll; b += kThreads) s_mass[b] = 0;
    for (int i = tid; i < 2 * kWideCodes; i += kThreads) s_num[i] = 0;
    if (tid == 0) s_outside = 0;
    if (j == 0 && tid == 0) *R.ticket = 0;
    __syncthreads();
    float top = -__builtin_inff();
    bool outside = false;
    each([&](float z, int, int, int) {
        top = fmaxf(top, z);
        const uint32_t code = code_of(z);
        if (code < (uint32_t)kWideCodes) atomicAdd(&s_num[code + (__float_as_uint(z) >> 31) * kWideCodes], 1u);
        else outside |= z > -__builtin_inff();
    });
    top = wave_max(top, lane);
    if (lane == 0) s_max[tid >> 6] = top;
    if (__ballot(outside) && lane == 0) s_outside = 1;
    __syncthreads();
    top = s_max[lane & (kThreads / 64 - 1)];
    top = wave_max(top, lane);
    if (!(T > 0.f)) {                                            // greedy: the largest key
        u64 best = 0;
        if (top > -__builtin_inff())
            each([&](float z, int p, int g, int e) {
                if (z == top) {
                    const int i = part(p).at(g, e);
                    const u64 key = make_key(top, A.ids ? A.ids[i] : i);
                    best = key > best ? key : best;
                }
            });
        best = reduce_all(best, s_part, [](u64 a, u64 b) { return a > b ? a : b; });
        if (tid == 0) R.slice[j] = SliceState{0.0, best, 0, 0};
        return;
    }
    const double c = log2e_over(T);
    const bool ok = top > -__builtin_inff() && regular_slice(T, top);
    const double ref = ok ? ceil((double)top * c) : 0.0;
    if (tid == 0) R.slice[j] = SliceState{ref, top > -__builtin_inff() ? make_key(top, 0) : 0, 0, 0};
    if (!ok) return;                                             // (uniform) nothing here, or a row for the digits
    const float cut = cut_of(ref, T);
    const int ref_steps = (int)ref * kSteps;
    auto add = [&](float x, uint32_t n) {
        if (x >= cut) {                                          // (not NaN)
            const Steps s = locate(x, c, ref_steps);
            if ((uint32_t)s.m < (uint32_t)(kRange * kSteps)) atomicAdd(&s_mass[bin_of(s.m)], n * weight_of(s, s_table));
        }
    };
    for (int i = tid; i < 2 * kWideCodes; i += kThreads) {
        const uint32_t n = s_num[i], code = (uint32_t)(i < kWideCodes ? i : i - kWideCodes) + kWideLow;
        if (n) add(__uint_as_float((code | (i < kWideCodes ? 0u : 0x8000u)) << 16), n);
    }
    if (s_outside)
        each([&](float z, int, int, int) {
            if (code_of(z) >= (uint32_t)kWideCodes) add(z, 1);
        });
    __syncthreads();
    for (int b = tid; b < kAll; b += kThreads) R.mass[(size_t)j * kAll + b] = s_mass[b];
}

// One step of a bitonic sort within a wavefront: the larger of lane and lane ^ D goes to the one that is to have it.
template <int D>
__device__ __forceinline__ void exchange(u64& v, bool descending, int lane) {
    const u64 y = (u64)xor_lane<D>((uint32_t)(v >> 32), lane) << 32 | xor_lane<D>((uint32_t)v, lane);
    const bool larger = ((lane & D) == 0) == descending;
    v = (y > v) == larger ? y : v;
}
template <int D>
__device__ __forceinline__ void exchange_from(u64& v, bool descending, int lane) {
    exchange<D>(v, descending, lane);
    if constexpr (D > 1) exchange_from<D / 2>(v, descending, lane);
}
// Sorts s_key[0, n), descending; places up to the next power of two are there.  Exchanges of up to 32 places are made in the
// registers of a wavefront that holds 64 keys in a row, the others (10 of the 55 steps of 1,024 keys) in LDS.
template <int THREADS>
__device__ __forceinline__ void sort_keys(u64* s_key, int n) {
    const int tid = threadIdx.x, lane = tid & 63;
    int size = 64;
    while (size < n) size *= 2;
    for (int i = tid; i < size; i += THREADS) {
        u64 v = i < n ? s_key[i] : 0;
        exchange_from<1>(v, (lane & 2) == 0, lane);
        exchange_from<2>(v, (lane & 4) == 0, lane);
        exchange_from<4>(v, (lane & 8) == 0, lane);
        exchange_from<8>(v, (lane & 16) == 0, lane);
        exchange_from<16>(v, (lane & 32) == 0, lane);
        exchange_from<32>(v, (i & 64) == 0, lane);
        s_key[i] = v;
    }
    __syncthreads();
    for (int w = 128; w <= size; w *= 2) {
        for (int d = w / 2; d >= 64; d /= 2) {
            for (int i = tid; i < size / 2; i += THREADS) {
                const int a = (i & ~(d - 1)) * 2 + (i & (d - 1)), b = a + d;
                const u64 x = s_key[a], y = s_key[b];
                if ((x < y) == ((a & w) == 0)) {
                    s_key[a] = y;
                    s_key[b] = x;
                }
            }
            __syncthreads();
        }
        for (int i = tid; i < size; i += THREADS) {
            u64 v = s_key[i];
            exchange_from<32>(v, (i & w) == 0, lane);
            s_key[i] = v;
        }
        __syncthreads();
    }
}
// s_sum[i] = sum of the weights of s_key[0, i]; `each` places in a row to a thread, each * THREADS >= n.
template <int THREADS, int EACH>
__device__ __forceinline__ void sum_weights(const u64* s_key, u64* s_sum, int n, float T, double ref, const double* table, u64* s_part) {
    const double c = log2e_over(T);
    const float cut = cut_of(ref, T);
    const int tid = threadIdx.x, lane = tid & 63;
    u64 w[EACH], sum = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int at = tid * EACH + i;
        w[i] = 0;
        if (at < n) {
            const float z = key_value(s_key[at]);
            const Steps s = locate(z, c, (int)ref * kSteps);
            w[i] = has_weight(z, cut, s) ? weight_of(s, table) : 0;
        }
        sum += w[i];
    }
    u64 run = sum;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const u64 x = shfl_up64(run, s);
        if (lane >= s) run += x;
    }
    if (lane == 63) s_part[tid >> 6] = run;
    __syncthreads();
    run -= sum;
    for (int v = 0; v < tid >> 6; ++v) run += s_part[v];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        run += w[i];
        if (tid * EACH + i < n) s_sum[tid * EACH + i] = run;
    }
    __syncthreads();
}
// The first of [lo, hi) for which f holds (and holds from there on), hi if there is none; a wavefront tries 64 at a time.
template <class F>
__device__ __forceinline__ int search(int lo, int hi, int lane, F f) {
    while (lo < hi) {
        const int step = (hi - lo + 63) / 64, i = lo + lane * step;
        const u64 yes = __ballot(i >= hi || f(i < hi ? i : hi - 1));
        const int first = yes ? __ffsll((long long)yes) - 1 : 64;
        if (first == 0) return lo;
        hi = min(hi, lo + first * step);
        lo += (first - 1) * step + 1;
    }
    return hi;
}
// Whether min-p leaves out the i-th of a sorted list, logit z.  Above 1 only the row's first token stays, which is on the list then, and
// not those that tie with it.
__device__ __forceinline__ bool too_light(int i, float z, float z_max, double c, float least) {
    return least > 1.f ? i > 0 : z != z_max && weight(z, z_max, c) < (double)least;
}
__device__ __forceinline__ void give(const SampleArgs& A, int m, u64 key, u64 kept, double c, double ref) {
    A.out_ids[m] = key_id(key);
    if (A.out_logprob)
        A.out_logprob[m] = (float)((fma((double)key_value(key), c, -ref) - log2((double)kept / kOne)) * 0.69314718055994530942);
}

constexpr int kRowThreads = kThreads;
constexpr int kRowList = 2048;

// Of n keys in LDS, logits in [bound, top], those that can be among the k largest, k <= n: by their numbers in kRowThreads even steps
// of the range.  Gives how many are left, by a counter of its own: the caller's, from which n came, may still be read by wavefronts that
// left the last barrier late.
__device__ int keep_front(u64* s_key, int n, int k, float bound, float top) {
    __shared__ uint32_t s_num[kRowThreads + 1], s_wave[kRowThreads / 64], s_left;
    __shared__ int s_cut;
    const int tid = threadIdx.x, lane = tid & 63;
    const float per = (float)kRowThreads / fmaxf(top - bound, 1e-30f);
    auto step_of = [&](u64 key) { return min(max((int)((top - key_value(key)) * per), 0), kRowThreads - 1); };
    s_num[tid] = 0;
    if (tid == 0) s_left = 0;
    __syncthreads();
    u64 mine[kRowList / kRowThreads];
#pragma unroll
    for (int r = 0; r < kRowList / kRowThreads; ++r) {
        mine[r] = r * kRowThreads + tid < n ? s_key[r * kRowThreads + tid] : 0;
        if (mine[r]) atomicAdd(&s_num[step_of(mine[r])], 1u);
    }
    __syncthreads();
    const uint32_t num = s_num[tid];
    uint32_t run = num;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const uint32_t x = (uint32_t)__shfl_up((int)run, s);
        if (lane >= s) run += x;
    }
    if (lane == 63) s_wave[tid >> 6] = run;
    __syncthreads();
    for (int w = 0; w < tid >> 6; ++w) run += s_wave[w];
    if (run >= (uint32_t)k && run - num < (uint32_t)k) s_cut = tid;
    __syncthreads();
    const int cut = s_cut;
#pragma unroll
    for (int r = 0; r < kRowList / kRowThreads; ++r)
        if (mine[r] && step_of(mine[r]) <= cut) s_key[atomicAdd(&s_left, 1u)] = mine[r];
    __syncthreads();
    return (int)s_left;
}

// A row of a small top-k, from its slices' lists; `most` is the largest of their bounds, which is one for the row.  False if they do not
// hold what is needed.
__device__ bool finish_largest(const SampleArgs& A, int m, int k, const RowSpace& R, const SliceState* s_slice, int slices, double most, double c, double ref,
                               float z_max, u64* s_key, u64* s_sum, double* s_table, u64* s_part, uint32_t* s_n) {
    const int tid = threadIdx.x, lane = tid & 63;
    const float bound = (float)most;
    fill_table(s_table);
    if (tid == 0) *s_n = 0;
    if (most != (double)bound) return false;                     // (uniform) tokens are missing at that bound
    __syncthreads();
    for (int j = tid >> 6; j < slices; j += kRowThreads / 64) {
        const int n = (int)s_slice[j].n;
        for (int i = lane; i < n; i += 64) {
            const u64 key = R.mass[(size_t)j * kAll + i];
            if (key_value(key) >= bound) {
                const uint32_t at = atomicAdd(s_n, 1u);
                if (at < kRowList) s_key[at] = key;
            }
        }
    }
    __syncthreads();
    int n = (int)*s_n;
    if (n > kRowList) return false;
    if (n > 2 * k) n = keep_front(s_key, n, k, bound, z_max);
    sort_keys<kRowThreads>(s_key, n);
    n = min(n, k);
    sum_weights<kRowThreads, 1>(s_key, s_sum, n, A.temperature ? A.temperature[m] : 1.f, ref, s_table, s_part);     // (n <= k <= kMostK)
    if (tid >= 64) return true;
    int last = n - 1;
    const float p = A.top_p ? A.top_p[m] : 1.f;
    if (p < 1.f) {
        const u64 target = share_up(p, s_sum[last]);
        last = min(last, search(0, n, lane, [&](int i) { return s_sum[i] >= target; }));
    }
    const float least = A.min_p ? A.min_p[m] : 0.f;
    if (least > 0.f) {
        const int first = search(0, n, lane, [&](int i) {
            return too_light(i, key_value(s_key[i]), z_max, c, least);
        });
        last = max(min(last, first - 1), 0);
    }
    const u64 kept = s_sum[last], target = share_past(A.u[m], kept);
    const int at = min(search(0, n, lane, [&](int i) { return s_sum[i] >= target; }), last);
    if (tid == 0) give(A, m, s_key[at], kept, c, ref);
    return true;
}
static_assert(kMostK <= kRowThreads, "one token a thread");

template <int TYPE>
__device__ __forceinline__ const char* row_of(const SampleArgs& A, int m) {
    return static_cast<const char*>(A.logits) + (long long)m * A.stride * (TYPE == EVOSPEC_FP32 ? 4 : 2);
}
// Calls put(key) for the slice's tokens whose bins are to be on the list.
template <class Put>
__device__ __forceinline__ void pick_tokens(const SampleArgs& A, Slice S, const float (&z)[kGroups][4], const RowState& st, float T,
                                            Put put) {
    const double c = log2e_over(T);
    const int b_max = max(st.hi[0], max(st.hi[1], st.hi[2]));
    // logits that can be in those bins, a little generously: bin b ends where x = -(b + 1) / kBins, to half a step
    const double far = (st.ref - (double)(b_max + 2) * (1.0 / kBins)) * ((double)T * 0.69314718055994530942);
    const float cut = cut_of(st.ref, T), least = b_max >= kFine ? cut : fmaxf(cut, (float)(far - fabs(far) * 0x1p-20));
    const int ref_steps = (int)st.ref * kSteps;
    int from[3], to[3];                                          // of m, the bins' (to: none has weight behind the last)
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        from[i] = first_of(st.lo[i]);
        to[i] = first_of(st.hi[i] + 1);
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (z[g][e] >= least) {
                const int m = locate(z[g][e], c, ref_steps).m;
                if ((m >= from[0] && m < to[0]) || (m >= from[1] && m < to[1]) || (m >= from[2] && m < to[2])) {
                    const int i = S.at(g, e);
                    put(make_key(z[g][e], A.ids ? A.ids[i] : i));
                }
            }
}

// Goes through the filters with a row's list (n tokens in LDS, in any order) and the sums of its bins.
__device__ void finish_row(const SampleArgs& A, int m, const RowState& st, u64* s_key, int n, u64* s_sum, const u64* s_before,
                           const double* s_table, u64* s_part) {
    const int tid = threadIdx.x, lane = tid & 63;
    const double c = log2e_over(A.temperature ? A.temperature[m] : 1.f);
    sort_keys<kThreads>(s_key, n);
    sum_weights<kThreads, kList / kThreads>(s_key, s_sum, n, A.temperature ? A.temperature[m] : 1.f, st.ref, s_table, s_part);
    if (tid >= 64) return;
    // One wavefront goes through the filters.  Every place is an index into the sorted list.
    auto m_at = [&](int i) { return locate(key_value(s_key[i]), c, (int)st.ref * kSteps).m; };
    auto bin_at = [&](int i) { return bin_of(m_at(i)); };
    // the first place of the list in bin b or behind
    auto place_of = [&](int b) { return search(0, n, lane, [&](int i) { return m_at(i) >= first_of(b); }); };
    auto sum_to = [&](int i) { return i > 0 ? s_sum[i - 1] : 0ull; };
    // the weight of the row's tokens in front of the list's place i
    auto before = [&](int i) {
        const int b = bin_at(i);
        return s_before[b] + sum_to(i) - sum_to(place_of(b));
    };
    auto upto = [&](int i) { return before(i) + s_sum[i] - sum_to(i); };
    // the place where that reaches target: its bin from the row's sums, then within the bin
    auto place_at = [&](u64 target) {
        const int bin = min(search(0, kAll, lane, [&](int b) { return s_before[b + 1] >= target; }), kAll - 1);
        const int first = place_of(bin), end = place_of(bin + 1);
        const u64 rest = target - s_before[bin] + sum_to(first);
        const int i = search(first, end, lane, [&](int i) { return s_sum[i] >= rest; });
        return max(min(i, min(end, n) - 1), 0);                  // (the last of the bin if rounding leaves it short)
    };
    int last = n;                                                // the place of the last token that is kept; n: all of the row are
    u64 kept = s_before[kAll];
    if (st.k_bin >= 0) {
        last = min(place_of(st.k_bin) + st.k_left, n) - 1;
        kept = upto(last);
    }
    const float p = A.top_p ? A.top_p[m] : 1.f;
    if (p < 1.f) {
        kept = share_up(p, kept);
        if (s_before[st.end_bin + 1] >= kept) {                  // (otherwise min-p cuts in front of that)
            last = min(last, place_at(kept));
            kept = upto(last);
        }
    }
    const float least = A.min_p ? A.min_p[m] : 0.f;
    if (least > 0.f) {
        // the first place whose weight is too small; if that is not on the list, the last bin that may hold larger ones ends there
        const int first = search(0, n, lane, [&](int i) {
            return too_light(i, key_value(s_key[i]), st.z_max, c, least);
        });
        const bool on = first < n && bin_at(min(first, n - 1)) <= st.least_bin;
        const u64 mass = on ? before(first) : s_before[st.least_bin + 1];
        if (mass < kept) {
            kept = mass;
            last = max((on ? first : place_of(st.least_bin + 1)) - 1, 0);
        }
    }
    int at = place_at(share_past(A.u[m], kept));
    if (last < n) at = min(at, last);
    if (tid == 0) give(A, m, s_key[at], kept, c, st.ref);
}

// Joins the bins of a row's slices (s_before[b] = what lies in front of bin b) and says which bins have to be looked at.
__device__ __forceinline__ RowState plan_row(const SampleArgs& A, int m, const RowSpace& R, const SliceState* s_slice, int slices, int k, float T,
                                             double c, double ref, float z_max, u64* s_before, u64* s_place, uint32_t* s_first, u64* s_part,
                                             uint32_t* s_num, int* s_found) {
    const int tid = threadIdx.x, lane = tid & 63;
    // the slices' bins, joined: those of a slice whose reference is `shift` factors of 2 lower go as many factors further
    static_assert(kAll < kRowThreads, "a bin a thread");
    __shared__ int s_shift[kMostSlices];
    if (tid < slices) {
        const SliceState s = s_slice[tid];
        const double gap = s.top != 0 && regular_slice(T, key_value(s.top)) ? ref - s.ref : kRange;      // (a whole number >= 0)
        s_shift[tid] = gap < kRange ? (int)gap : -1;
    }
    // (a row's bins behind kFine are 32 places each until all slices are there: lanes that add to one place of LDS go one by one)
    for (int i = tid; i < kPlaces; i += kRowThreads) {
        s_place[i] = 0;
        if (k > 0) s_first[i] = 0;
    }
    __syncthreads();
    const int mine = tid < kFine ? tid : kFine + (tid - kFine) * kBins;
    for (int first = 0; first < slices; first += kAtOnce) {
        u64 w[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) w[i] = R.mass[(size_t)min(first + i, slices - 1) * kAll + min(tid, kAll - 1)];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int j = first + i, shift = __builtin_amdgcn_readfirstlane(j < slices ? s_shift[j] : -1), to = mine + shift * kBins;
            if (shift < 0) continue;                             // (uniform)
            if (tid < kAll && to < kPlaces) {
                atomicAdd(&s_place[to], shift ? (w[i] + (1ull << (shift - 1))) >> shift : w[i]);
                if (k > 0) atomicAdd(&s_first[to], R.count[(size_t)j * kAll + tid]);
            }
        }
    }
    __syncthreads();
    // A bin a thread; of those behind kFine every eighth, which the eight sum up, 4 places each.
    static_assert(kFine % 64 == 0 && kBins == 32 && kPlaces - kFine == 4 * (kRowThreads - kFine), "whole wavefronts");
    u64 mass = 0;
    uint32_t count = 0;
    int bin = tid;
    if (tid < kFine) {                                           // (uniform)
        mass = s_place[tid];
        if (k > 0) count = s_first[tid];
    } else {
        const int at = kFine + 4 * (tid - kFine);
        mass = s_place[at] + s_place[at + 1] + s_place[at + 2] + s_place[at + 3];
        mass = sum_eight(mass, lane);
        if (k > 0) count = (uint32_t)sum_eight((u64)s_first[at] + s_first[at + 1] + s_first[at + 2] + s_first[at + 3], lane);
        bin = kFine + (tid - kFine) / 8;
        if (lane & 7) {
            mass = count = 0;
            bin = tid == kRowThreads - 1 ? kAll : -1;
        }
    }
    // what lies in front of each bin
    u64 run = mass;
    uint32_t runs = count;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const u64 x = shfl_up64(run, s);
        const uint32_t y = (uint32_t)__shfl_up((int)runs, s);
        if (lane >= s) {
            run += x;
            runs += y;
        }
    }
    if (lane == 63) {
        s_part[tid >> 6] = run;
        s_num[tid >> 6] = runs;
    }
    __syncthreads();
    run -= mass;
    runs -= count;
    for (int w = 0; w < tid >> 6; ++w) {
        run += s_part[w];
        runs += s_num[w];
    }
    if (bin >= 0) {
        s_before[bin] = run;
        s_first[bin] = runs;
    }
    __syncthreads();
    const u64 total = s_before[kAll];
    // the bin at which the sum over the bins reaches target (1 <= target <= total)
    auto bin_at = [&](u64 target, int slot) {
        target = target < 1 ? 1 : target > total ? total : target;
        for (int b = tid; b < kAll; b += kRowThreads)
            if (s_before[b] < target && s_before[b + 1] >= target) s_found[slot] = b;
        __syncthreads();
        return s_found[slot];
    };
    int k_bin = -1, k_left = 0;
    u64 lo = total, hi = total;                                  // bounds of what is kept
    int end_lo = kAll, end_hi = kAll;                            // and of the bin where that ends (kAll: all are kept)
    if (k > 0 && (uint32_t)k < s_first[kAll]) {
        for (int b = tid; b < kAll; b += kRowThreads)
            if (s_first[b] < (uint32_t)k && s_first[b + 1] >= (uint32_t)k) s_found[0] = b;
        __syncthreads();
        k_bin = s_found[0];
        k_left = k - (int)s_first[k_bin];
        lo = s_before[k_bin];
        hi = s_before[k_bin + 1];
        end_lo = end_hi = k_bin;
    }
    const float p = A.top_p ? A.top_p[m] : 1.f;
    if (p < 1.f) {
        end_lo = bin_at(share_up(p, lo), 1);
        end_hi = bin_at(share_up(p, hi), 2);
    }
    const float least = A.min_p ? A.min_p[m] : 0.f;
    int least_bin = kAll - 1;
    if (least > 0.f) {
        // the bin of w = least, give or take two
        const double x = fma((double)z_max, c, -ref) + (least < 1.f ? (double)__log2f(least) : 0.0);
        const int b = (int)fmin(-x * kBins, (double)(kRange + 2) * kBins), near = bin_of(max(b - 2, 0)), far = bin_of(b + 2);
        if (near < end_lo) end_lo = near;
        if (far < end_hi) end_hi = far;
        least_bin = min(far, kAll - 1);
    }
    int n = 0;
    int bins[3][2];
    if (end_hi < kAll) {
        lo = s_before[end_lo];
        hi = s_before[end_hi + 1];
        bins[n][0] = end_lo;
        bins[n++][1] = end_hi;
    } else if (end_lo < kAll) {                                  // min-p cuts among the last bins, or behind them
        lo = s_before[end_lo];
        hi = total;
        bins[n][0] = end_lo;
        bins[n++][1] = end_hi = kAll - 1;
    }
    const float u = A.u[m];
    const int draw_lo = bin_at(share_past(u, lo), 3), draw_hi = bin_at(share_past(u, hi), 4);
    bins[n][0] = draw_lo;
    bins[n++][1] = draw_hi;
    if (k_bin >= 0) {
        bins[n][0] = k_bin;
        bins[n++][1] = k_bin;
    }
    RowState st;
    st.ref = ref;
    st.z_max = z_max;
    st.state = kOpen;
    for (int i = 0; i < 3; ++i) {
        st.lo[i] = i < n ? bins[i][0] : kAll;
        st.hi[i] = i < n ? bins[i][1] : -1;
    }
    st.end_bin = min(end_hi, kAll - 1);
    st.least_bin = least_bin;
    st.k_bin = k_bin;
    st.k_left = k_left;
    return st;
}

// REST: the row is ended here, where a workgroup for each row is what there is to do, or most rows end early.  TOP_K: there may be one (calls
// without have a kernel of their own, whose registers the lists do not crowd: 960 rows of bf16 222 us, and 235 to 250 together).
template <int TYPE, bool REST, bool TOP_K>
__global__ __launch_bounds__(kRowThreads, 8) void sample_row_kernel(SampleArgs A, char* ws, int slices) {
    __shared__ u64 s_before[kAll + 1];
    __shared__ uint32_t s_counts[REST ? 1 : kAll + 1];
    __shared__ u64 s_part[kRowThreads / 64], s_pick[2];
    __shared__ uint32_t s_num[kRowThreads / 64];
    __shared__ u64 s_key[REST ? kList : 1], s_sum[REST ? kList : 1];
    __shared__ u64 s_places[REST ? 1 : kPlaces];
    // (numbers of tokens are done with before the list's sums are there, and places before the list; two of these workgroups fit a
    // compute unit)
    uint32_t* s_first = REST ? reinterpret_cast<uint32_t*>(s_sum) : s_counts;
    u64* s_place = REST ? s_key : s_places;
    __shared__ double s_table[kSteps];
    __shared__ uint32_t s_n;
    __shared__ int s_found[8];
    __shared__ SliceState s_slice[kMostSlices];
    const int m = blockIdx.x, tid = threadIdx.x;
    const RowSpace R = row_space(ws, m, slices);
    const float T = A.temperature ? A.temperature[m] : 1.f;
    static_assert(kMostSlices <= 64, "a slice a lane");
    const SliceState of_lane = R.slice[min(tid & 63, slices - 1)];
    if (tid < slices) s_slice[tid] = of_lane;
    u64 top = of_lane.top;
    double bound = of_lane.ref;                                  // (of lists: k logits of one slice reach its bound)
    for (int s = 32; s >= 1; s >>= 1) {
        if (s >= slices) continue;                               // (uniform; lanes from there on repeat the last slice)
        const u64 x = shfl_xor64(top, s);
        top = x > top ? x : top;
        if (TOP_K) bound = fmax(bound, __longlong_as_double((long long)shfl_xor64((u64)__double_as_longlong(bound), s)));
    }
    if (slices > 1) {
        top = first_lane(top);
        if (TOP_K) bound = __longlong_as_double((long long)first_lane((u64)__double_as_longlong(bound)));
    }
    __syncthreads();
    const float z_max = key_value(top);
    static_assert(REST || !TOP_K, "with a top-k rows are ended here");
    const int k = TOP_K ? A.top_k[m] : 0;
    if (top == 0 || !(T > 0.f)) {
        if (tid == 0) {
            A.out_ids[m] = top == 0 ? -1 : key_id(top);
            if (A.out_logprob) A.out_logprob[m] = top == 0 ? __uint_as_float(0x7fc00000u) : 0.f;
            if (!REST) R.row->state = kDone;
        }
        return;
    }
    bool digits = !regular(T, z_max);                            // (uniform)
    if (digits && !REST) {
        if (tid == 0) R.row->state = kDigits;
        return;
    }
    const double c = log2e_over(T);
    const double ref = ceil((double)z_max * c);
    if constexpr (TOP_K)
        if (!digits && k > 0 && k <= kMostK) {
            if (finish_largest(A, m, k, R, s_slice, slices, bound, c, ref, z_max, s_key, s_sum, s_table, s_part, &s_n)) return;
            digits = true;
        }
    if constexpr (REST) {
        if (!digits) {
            const RowState st = plan_row(A, m, R, s_slice, slices, k, T, c, ref, z_max, s_before, s_place, s_first, s_part, s_num, s_found);
            fill_table(s_table);
            if (tid == 0) s_n = 0;
            __syncthreads();
            const char* row = row_of<TYPE>(A, m);
            const int parts = (A.V + kSlice - 1) / kSlice;       // (few and large, whatever the slices of the bins were)
            RawSlice<TYPE> raw;                                  // (16-bit types: the next part is under way meanwhile)
            if (TYPE != EVOSPEC_FP32) raw.load(row, slice_of(A.V, parts, 0));
            for (int j = 0; j < parts; ++j) {
                const Slice S = slice_of(A.V, parts, j);
                float z[kGroups][4];
                if (TYPE == EVOSPEC_FP32) raw.load(row, S);
                raw.give(z);
                if (TYPE != EVOSPEC_FP32 && j + 1 < parts) raw.load(row, slice_of(A.V, parts, j + 1));
                pick_tokens(A, S, z, st, T, [&](u64 key) {
                    const uint32_t at = atomicAdd(&s_n, 1u);
                    if (at < kList) s_key[at] = key;
                });
            }
            __syncthreads();
            if (s_n <= (uint32_t)kList) {                        // (uniform)
                finish_row(A, m, st, s_key, (int)s_n, s_sum, s_before, s_table, s_part);
                return;
            }
        }
        __syncthreads();
        sample_by_digits<TYPE>(A, m, s_key, s_part, s_pick);
        return;
    }
    if constexpr (!REST) {
        const RowState st = plan_row(A, m, R, s_slice, slices, k, T, c, ref, z_max, s_before, s_place, s_first, s_part, s_num, s_found);
        for (int b = tid; b <= kAll; b += kRowThreads) R.before[b] = s_before[b];
        if (tid == 0) *R.row = st;
    }
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void sample_pick_kernel(SampleArgs A, char* ws, int slices, int parts) {
    __shared__ u64 s_key[kStage];
    __shared__ uint32_t s_n, s_at;
    const int m = blockIdx.x / parts, j = blockIdx.x % parts, tid = threadIdx.x;
    const RowSpace R = row_space(ws, m, slices);
    const Slice S = slice_of(A.V, parts, j);
    float z[kGroups][4];
    load_slice<TYPE>(row_of<TYPE>(A, m), S, z);                  // (under way while the row's state is looked at)
    const RowState st = *R.row;
    if (st.state != kOpen) return;
    const float T = A.temperature ? A.temperature[m] : 1.f;
    if (tid == 0) s_n = 0;
    __syncthreads();
    pick_tokens(A, S, z, st, T, [&](u64 key) {
        const uint32_t at = atomicAdd(&s_n, 1u);
        if (at < kStage) {
            s_key[at] = key;
        } else {                                                 // (rare: places of the row's list one by one)
            const uint32_t far = atomicAdd(R.ticket, 1u);
            if (far < kList) R.list[far] = key;
        }
    });
    __syncthreads();
    const uint32_t n = min(s_n, (uint32_t)kStage);
    if (tid == 0) s_at = atomicAdd(R.ticket, n);
    __syncthreads();
    for (uint32_t i = tid; i < n; i += kThreads)
        if (s_at + i < kList) R.list[s_at + i] = s_key[i];
}

// What the bins leave open, a workgroup for each row.
template <int TYPE>
__global__ __launch_bounds__(kThreads, 8) void sample_finish_kernel(SampleArgs A, char* ws, int slices) {
    __shared__ u64 s_key[kList], s_sum[kList], s_before[kAll + 1];
    __shared__ double s_table[kSteps];
    __shared__ u64 s_part[kThreads / 64], s_pick[2];
    const int m = blockIdx.x, tid = threadIdx.x;
    const RowSpace R = row_space(ws, m, slices);
    const RowState st = *R.row;
    if (st.state == kDone) return;
    const int n = (int)*R.ticket;
    if (st.state == kDigits || n > kList) {
        sample_by_digits<TYPE>(A, m, s_key, s_part, s_pick);
        return;
    }
    fill_table(s_table);
    for (int b = tid; b <= kAll; b += kThreads) s_before[b] = R.before[b];
    for (int i = tid; i < n; i += kThreads) s_key[i] = R.list[i];
    __syncthreads();
    finish_row(A, m, st, s_key, n, s_sum, s_before, s_table, s_part);
}

}  // namespace

constexpr int kManyRows = 512;

// Slices of a row: as few as there can be, or, where no row asks for a top-k, as many as give each compute unit one, of kLeastSlice
// logits at least and no more than are joined at once (lists of a top-k get longer with more slices).  Top-p of fp32, in as few slices, in
// up to 8 and in up to 52: one row of 50,000 28.2, 26.9 and 28.6 us, of 151,936 32.7, 32.6 and 36.4; 30 rows of 40,000 33.1, 30.3 and 35.1.
constexpr int kLeastSlice = 4096, kUnits = 256;
static int whole_slices(int V) { return (V + kSlice - 1) / kSlice; }
static int many_slices(int M, int V) {
    const int most = std::min(std::max(V / kLeastSlice, 1), kAtOnce);
    return std::max(whole_slices(V), std::min((kUnits + M - 1) / M, most));
}
int sample_slices(int V) { return whole_slices(V); }

// What any M' <= M rows take: M' many_slices(M') is M' whole_slices at most, or less than kUnits + M'.
size_t sample_workspace(int M, int V) {
    if (M == 0) return 0;
    const size_t n = whole_slices(V), most = (size_t)M * std::max((size_t)many_slices(1, V), n);
    const size_t slices = std::max((size_t)M * n, std::min((size_t)kUnits + M, most));
    return slices * (row_bytes(2) - row_bytes(1) + 256) + (size_t)M * row_bytes(1);
}

template <int TYPE>
static hipError_t sample_as(const SampleArgs& a, char* ws, hipStream_t stream) {
    // Who ends the rows: a workgroup for each, with less to launch and to pass on, where top-k leaves little, rows would fit one
    // slice, or there are enough of them; otherwise its slices side by side.  By itself against side by side (top-p, fp32): one row of 151,936
    // 42 and 32 us, 256 rows 122 and 116, 384 155 and 155, 512 175 and 191; 30 rows of 60,000 38 and 33; 60 rows of 20,000 28 and 29.  A call
    // with a top-k has its rows ended by a workgroup each whatever their own says: one row without 55 us there, 60 rows 64 and 48.
    const bool rest = a.top_k || whole_slices(a.V) == 1 || a.M >= kManyRows;
    const int parts = a.top_k ? whole_slices(a.V) : many_slices(a.M, a.V);
    // (longer slices where two workgroups for each compute unit are left)
    const int wide = TYPE != EVOSPEC_BF16 || a.top_k ? 1 : std::min((int)std::min((long long)a.M * parts / (2 * kUnits), 4ll), parts);
    const int slices = wide > 1 ? (parts + wide - 1) / wide : parts;
    const dim3 grid((unsigned)(a.M * slices));
    if (wide > 1) sample_wide_bins_kernel<<<grid, kThreads, 0, stream>>>(a, ws, slices, wide);
    else if (TYPE == EVOSPEC_BF16 && a.V / slices >= kLeastByValue) sample_bins_kernel<TYPE, TYPE == EVOSPEC_BF16><<<grid, kThreads, 0, stream>>>(a, ws, slices);
    else sample_bins_kernel<TYPE, false><<<grid, kThreads, 0, stream>>>(a, ws, slices);
    if (a.top_k) {
        sample_row_kernel<TYPE, true, true><<<dim3((unsigned)a.M), kRowThreads, 0, stream>>>(a, ws, slices);
    } else if (rest) {
        sample_row_kernel<TYPE, true, false><<<dim3((unsigned)a.M), kRowThreads, 0, stream>>>(a, ws, slices);
    } else {
        sample_row_kernel<TYPE, false, false><<<dim3((unsigned)a.M), kRowThreads, 0, stream>>>(a, ws, slices);
        sample_pick_kernel<TYPE><<<dim3((unsigned)(a.M * parts)), kThreads, 0, stream>>>(a, ws, slices, parts);
        sample_finish_kernel<TYPE><<<dim3((unsigned)a.M), kThreads, 0, stream>>>(a, ws, slices);
    }
    return hipGetLastError();
}

hipError_t launch_sample(const SampleArgs& a, int type, void* workspace, hipStream_t stream) {
    char* ws = static_cast<char*>(workspace);
    return type == EVOSPEC_FP32 ? sample_as<EVOSPEC_FP32>(a, ws, stream)
                                : type == EVOSPEC_FP16 ? sample_as<EVOSPEC_FP16>(a, ws, stream) : sample_as<EVOSPEC_BF16>(a, ws, stream);
}

}  // namespace evospec
