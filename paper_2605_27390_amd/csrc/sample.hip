// Sampling: one token for each row of logits by temperature, top-k, top-p and min-p, from a given random number.
//
// All four filters keep a front part of the row's tokens in the order (larger logit, smaller id), which is that of the
// 64-bit keys of common.hpp; a filter is therefore a smallest key, and so is the drawn token: the key at which the
// cumulative weight of the kept ones passes u times their sum.  Such keys are found digit by digit from a histogram of the
// keys that agree so far, of numbers (top-k) or of weights (top-p, the draw).  Weights w = exp((z - z_max) / T) are computed
// in 64 bits and kept as whole multiples of 2^-43: their sums do not depend on an order, so that a histogram may be filled by
// atomics, and 2^20 of them fit 64 bits.
#include <hip/hip_runtime.h>

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
// the weight of a logit; c = log2(e) / T
__device__ __forceinline__ double weight(float z, float z_max, double c) {
    if (z == z_max) return 1.0;
    const double x = ((double)z - (double)z_max) * c;
    return x > -45.0 ? exp2_series(x) : 0.0;
}
__device__ __forceinline__ u64 fixed(double w) { return (u64)(w * kOne + 0.5); }

template <int TYPE>
__device__ __forceinline__ float logit(const void* row, int i) {
    if constexpr (TYPE == EVOSPEC_FP32) return static_cast<const float*>(row)[i];
    else if constexpr (TYPE == EVOSPEC_FP16) return (float)static_cast<const _Float16*>(row)[i];
    else return (float)static_cast<const __bf16*>(row)[i];
}

__device__ __forceinline__ u64 shfl_xor64(u64 x, int s) {
    return (u64)(uint32_t)__shfl_xor((int)(uint32_t)x, s) | (u64)(uint32_t)__shfl_xor((int)(uint32_t)(x >> 32), s) << 32;
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

// The key of the row at which the cumulative measure of the keys from the largest down reaches `target` (>= 1; no more than
// the measure of all keys >= low): f(key index) calls back with (key, measure) of every key.
template <class EachKey>
__device__ u64 find_key(u64 low, u64 target, u64* s_hist, u64* s_pick, EachKey each) {
    u64 prefix = 0, mask = 0;
    for (int shift = 56; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += kThreads) s_hist[i] = 0;
        __syncthreads();
        each([&](u64 key, u64 measure) {
            if (key >= low && (key & mask) == prefix && measure) atomicAdd(&s_hist[(key >> shift) & 255], measure);
        });
        __syncthreads();
        if (threadIdx.x == 0) {
            u64 sum = 0;
            int d = 255;
            for (; d > 0; --d) {
                if (sum + s_hist[d] >= target) break;
                sum += s_hist[d];
            }
            s_pick[0] = (u64)d;
            s_pick[1] = target - sum;
        }
        __syncthreads();
        prefix |= s_pick[0] << shift;
        target = s_pick[1];
        mask |= 255ull << shift;
        __syncthreads();
    }
    return prefix;
}

// One workgroup a row; the row is read again for every digit.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void sample_row_kernel(SampleArgs A) {
    __shared__ u64 s_hist[256], s_part[kThreads / 64], s_pick[2];
    const int m = blockIdx.x;
    const char* row = static_cast<const char*>(A.logits) + (long long)m * A.stride * (TYPE == EVOSPEC_FP32 ? 4 : 2);
    const float T = A.temperature ? A.temperature[m] : 1.f;
    auto each = [&](auto f) {
        for (int i = threadIdx.x; i < A.V; i += kThreads) {
            const float z = logit<TYPE>(row, i);
            if (z > -__builtin_inff()) f(make_key(z, A.ids ? A.ids[i] : i), z);
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
    const double c = 1.4426950408889634074 / (double)T;
    auto masses = [&](auto f) { each([&](u64 key, float z) { f(key, fixed(weight(z, z_max, c))); }); };
    auto mass_from = [&](u64 low) {
        u64 sum = 0;
        masses([&](u64 key, u64 w) { sum += key >= low ? w : 0; });
        return reduce_all(sum, s_part, [](u64 a, u64 b) { return a + b; });
    };
    u64 low = 0;
    const int k = A.top_k ? A.top_k[m] : 0;
    if (k > 0 && (u64)k < n) low = find_key(low, (u64)k, s_hist, s_pick, [&](auto f) { each([&](u64 key, float) { f(key, 1); }); });
    const float p = A.top_p ? A.top_p[m] : 1.f;
    if (p < 1.f) {
        const u64 all = mass_from(low);
        const double t = ceil((double)p * (double)all);
        const u64 target = t >= 1.0 ? (u64)t : 1;
        low = find_key(low, target < all ? target : all, s_hist, s_pick, masses);
    }
    const float least = A.min_p ? A.min_p[m] : 0.f;
    if (least > 0.f) {
        u64 first = top;
        each([&](u64 key, float z) { if (key >= low && key < first && weight(z, z_max, c) >= (double)least) first = key; });
        low = reduce_all(first, s_part, [](u64 a, u64 b) { return a < b ? a : b; });
    }
    const u64 total = mass_from(low);
    const float u = A.u[m];
    const double t = floor((double)u * (double)total);
    const u64 target = t >= 0.0 ? (t < (double)total ? (u64)t + 1 : total) : 1;
    const u64 key = find_key(low, target < total ? target : total, s_hist, s_pick, masses);
    if (threadIdx.x == 0) {
        A.out_ids[m] = key_id(key);
        if (A.out_logprob) {
            const double x = key_value(key) == z_max ? 0.0 : ((double)key_value(key) - (double)z_max) / (double)T;
            A.out_logprob[m] = (float)(x - log((double)total / kOne));
        }
    }
}

}  // namespace

size_t sample_workspace(int M, int V) { return 0; }

hipError_t launch_sample(const SampleArgs& a, int type, void* workspace, int num_cu, hipStream_t stream) {
    const dim3 grid((unsigned)a.M);
    if (type == EVOSPEC_FP32) sample_row_kernel<EVOSPEC_FP32><<<grid, kThreads, 0, stream>>>(a);
    else if (type == EVOSPEC_FP16) sample_row_kernel<EVOSPEC_FP16><<<grid, kThreads, 0, stream>>>(a);
    else sample_row_kernel<EVOSPEC_BF16><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace evospec
