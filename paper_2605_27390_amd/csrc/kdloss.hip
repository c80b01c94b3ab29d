// The distillation loss on the retained support and its gradient (EvoSpec paper, Eq. 5): for an event with hidden state h and
// support rows W_j, z_j = h . W_j, q = softmax(z / T), p = softmax(target / T),
//   loss = w T^2 sum p (log p - log q)        dh = w T (sum q_j W_j - sum p_j W_j).
// The gradient is attention of one query whose keys and values are the same rows: a row of W_lm is read once, gives its logit, and
// joins two sums, sum exp((z_j - max) / T) W_j under a running maximum and sum p_j W_j, whose weights the targets alone give.  Bound by
// the rows' bytes (K d 2 of an event); an element costs four vector instructions.
// A workgroup has an event, or a part of its rows; a thread has every 256th piece of 8 elements of the rows, of h and of both sums, in
// registers.  The loss is taken from the K logits in 64 bits at the end: near its minimum it is a small difference of large terms.
#include <hip/hip_runtime.h>

#include "adapt.hpp"
#include "common.hpp"

namespace evospec {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMost = EVOSPEC_KD_K_MAX;

// Sum over the workgroup in a fixed order; every thread has it.
template <typename T>
__device__ __forceinline__ T block_sum(T x, T* buf /*LDS [kWaves]*/) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = x;
    __syncthreads();
    T s = buf[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) s += buf[i];
    return s;
}
// The largest, leaving NaN out.
__device__ __forceinline__ float block_max(float x, float* buf) {
    x = wave_max(x, threadIdx.x & 63);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = x;
    __syncthreads();
    float s = buf[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) s = fmaxf(s, buf[i]);
    return s;
}

// weight T^2 KL(p || q) of an event in 64 bits, by all threads; draft: its logits.
__device__ __forceinline__ void event_loss(const KdArgs& a, int e, const float* draft, double* buf, float* fbuf) {
    const int32_t* ids = a.support + (long long)e * a.K;
    const float* target = a.target + (long long)e * a.K;
    float mt = -__builtin_inff(), mz = mt;
    for (int j = threadIdx.x; j < a.K; j += kThreads)
        if ((unsigned)ids[j] < (unsigned)a.V) {
            mt = fmaxf(mt, target[j]);
            mz = fmaxf(mz, draft[j]);
        }
    mt = block_max(mt, fbuf);
    mz = block_max(mz, fbuf);
    const double inv = 1.0 / (double)a.T;
    double st = 0.0, sz = 0.0;
    bool any_nan = false;
    for (int j = threadIdx.x; j < a.K; j += kThreads)
        if ((unsigned)ids[j] < (unsigned)a.V) {
            any_nan |= target[j] != target[j];
            st += exp(((double)target[j] - mt) * inv);
            sz += exp(((double)draft[j] - mz) * inv);
        }
    any_nan = __syncthreads_or(any_nan);
    st = block_sum(st, buf);
    sz = block_sum(sz, buf);
    const double lt = log(st), lz = log(sz);
    double kl = 0.0;
    for (int j = threadIdx.x; j < a.K; j += kThreads)
        if ((unsigned)ids[j] < (unsigned)a.V) {
            const double lp = ((double)target[j] - mt) * inv - lt, lq = ((double)draft[j] - mz) * inv - lz, p = exp(lp);
            if (!(p == 0.0)) kl += p * (lp - lq);
        }
    kl = block_sum(kl, buf);
    if (threadIdx.x == 0) {
        const bool none = mt == -__builtin_inff() && !any_nan;   // no entry, or no target mass
        a.loss[e] = none ? 0.f : (float)((double)(a.weight ? a.weight[e] : 1.f) * a.T * a.T * kl);
    }
}

template <int TYPE>
__device__ __forceinline__ void store8(void* out, long long at, const float* x) {
    if constexpr (TYPE == EVOSPEC_FP32) {
        reinterpret_cast<float4*>((float*)out + at)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>((float*)out + at)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        bf16x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
        *reinterpret_cast<bf16x8*>((__bf16*)out + at) = v;
    }
}

// NC pieces of 8 elements to a thread, RB rows at a time.
template <int NC, int RB, int TYPE>
__global__ __launch_bounds__(kThreads) void kd_rows_kernel(KdArgs a) {
    __shared__ float dots[2][kWaves][RB];
    __shared__ float p[kMost];                                   // of this workgroup's entries
    __shared__ float z[kMost];
    __shared__ int32_t ids[kMost];
    __shared__ double dbuf[kWaves];
    __shared__ float fbuf[kWaves];
    const int e = blockIdx.x, part = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int j0 = (int)((long long)a.K * part / a.splits), j1 = (int)((long long)a.K * (part + 1) / a.splits);
    const float inv = 1.f / a.T;
    bool in[NC];
    u32x4 h[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        in[c] = 8 * (c * kThreads + tid) < a.d;
        h[c] = in[c] ? *(gvec_ptr)((const uint16_t*)a.h + (long long)e * a.d + 8 * (c * kThreads + tid)) : u32x4{0, 0, 0, 0};
    }
    // p, from all entries of the event
    float mt = -__builtin_inff();
    for (int j = tid; j < a.K; j += kThreads)
        if ((unsigned)a.support[(long long)e * a.K + j] < (unsigned)a.V) mt = fmaxf(mt, a.target[(long long)e * a.K + j]);
    mt = block_max(mt, fbuf);
    float sum = 0.f;
    bool nan = false;
    for (int j = tid; j < a.K; j += kThreads) {
        const int32_t id = a.support[(long long)e * a.K + j];
        const float t = a.target[(long long)e * a.K + j];
        const bool mine = (unsigned)id < (unsigned)a.V;
        const float x = mine ? expf((t - mt) * inv) : 0.f;
        sum += x;
        nan |= mine && t != t;
        if (j >= j0 && j < j1) {
            p[j - j0] = x;
            ids[j - j0] = mine ? id : -1;
        }
    }
    nan = __syncthreads_or(nan);
    const float total = block_sum(sum, fbuf);
    const bool none = mt == -__builtin_inff() && !nan;
    const float per = none ? 0.f : 1.f / total;
    __syncthreads();

    float o1[NC][8] = {}, o2[NC][8] = {};
    float m = -__builtin_inff(), l = 0.f;
    u32x4 row[RB][NC];
    const int n = j1 - j0;
    auto load = [&](int at) {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int id = at + r < n ? ids[at + r] : -1;        // (uniform)
            const uint16_t* w = (const uint16_t*)a.W + (long long)(id < 0 ? 0 : id) * a.d;
#pragma unroll
            for (int c = 0; c < NC; ++c)
                row[r][c] = in[c] && id >= 0 ? *(gvec_ptr)(w + 8 * (c * kThreads + tid)) : u32x4{0, 0, 0, 0};
        }
    };
    for (int at = 0, turn = 0; at < n; at += RB, turn ^= 1) {
        load(at);
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            float dot = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    dot = fmaf(__uint_as_float(row[r][c][q] << 16), __uint_as_float(h[c][q] << 16), dot);
                    dot = fmaf(__uint_as_float(row[r][c][q] & 0xffff0000u), __uint_as_float(h[c][q] & 0xffff0000u), dot);
                }
            dot = wave_sum(dot, lane);
            if (lane == 0) dots[turn][wave][r] = dot;
        }
        __syncthreads();
        float x[RB], top = m;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            x[r] = dots[turn][0][r];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) x[r] += dots[turn][w][r];
            const bool mine = at + r < n && ids[at + r] >= 0;
            if (tid == 0 && at + r < n) z[at + r] = mine ? x[r] : __builtin_nanf("");
            if (!mine) x[r] = -__builtin_inff();
            else x[r] *= inv;
            top = fmaxf(top, x[r]);
        }
        const float back = top == m ? 1.f : expf(m - top);       // (uniform)
        if (back != 1.f) {
            l *= back;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) o1[c][i] *= back;
        }
        m = top;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            if (at + r >= n || ids[at + r] < 0) continue;
            const float q = expf(x[r] - m), w = p[at + r] * per;
            l += q;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float v = i & 1 ? __uint_as_float(row[r][c][i / 2] & 0xffff0000u) : __uint_as_float(row[r][c][i / 2] << 16);
                    o1[c][i] = fmaf(q, v, o1[c][i]);
                    o2[c][i] = fmaf(w, v, o2[c][i]);
                }
        }
    }
    __syncthreads();
    for (int j = tid; j < n; j += kThreads) a.draft[(long long)e * a.K + j0 + j] = z[j];
    if (a.splits == 1) {
        const float factor = (a.weight ? a.weight[e] : 1.f) * a.T, li = 1.f / l;
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (in[c]) {
                float g[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = none ? 0.f : factor * (o1[c][i] * li - o2[c][i]);
                store8<TYPE>(a.dh, (long long)e * a.d + 8 * (c * kThreads + tid), g);
            }
        event_loss(a, e, z, dbuf, fbuf);
    } else {
        float* out = a.part + ((long long)e * a.splits + part) * 2 * a.d;
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (in[c]) {
                store8<EVOSPEC_FP32>(out, 8 * (c * kThreads + tid), o1[c]);
                store8<EVOSPEC_FP32>(out, a.d + 8 * (c * kThreads + tid), o2[c]);
            }
        if (tid == 0) a.part_ml[(long long)e * a.splits + part] = make_float2(m, none ? -1.f : l);
    }
}

// Joins the parts of an event's rows: 2,048 elements of its gradient to a workgroup, the first of which takes the loss as well.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void kd_join_kernel(KdArgs a) {
    __shared__ double dbuf[kWaves];
    __shared__ float fbuf[kWaves];
    const int e = blockIdx.x, at = 8 * (blockIdx.y * kThreads + threadIdx.x);
    const float2* ml = a.part_ml + (long long)e * a.splits;
    float m = -__builtin_inff();
    for (int s = 0; s < a.splits; ++s) m = fmaxf(m, ml[s].x);
    float l = 0.f, o[8] = {}, o2[8] = {};
    bool none = false;
    for (int s = 0; s < a.splits; ++s) {
        const float2 x = ml[s];
        none |= x.y == -1.f;
        const bool empty = x.y == 0.f && x.x == -__builtin_inff();           // a part without entries (its sums are zeros)
        const float f = empty ? 0.f : expf(x.x - m);
        l += x.y * f;
        if (at < a.d && !empty) {
            const float4* p = reinterpret_cast<const float4*>(a.part + ((long long)e * a.splits + s) * 2 * a.d + at);
            const float4* q = reinterpret_cast<const float4*>(a.part + ((long long)e * a.splits + s) * 2 * a.d + a.d + at);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 u = p[i], v = q[i];
                o[4 * i] = fmaf(f, u.x, o[4 * i]); o[4 * i + 1] = fmaf(f, u.y, o[4 * i + 1]);
                o[4 * i + 2] = fmaf(f, u.z, o[4 * i + 2]); o[4 * i + 3] = fmaf(f, u.w, o[4 * i + 3]);
                o2[4 * i] += v.x; o2[4 * i + 1] += v.y; o2[4 * i + 2] += v.z; o2[4 * i + 3] += v.w;
            }
        }
    }
    const float factor = (a.weight ? a.weight[e] : 1.f) * a.T, li = 1.f / l;
    if (at < a.d) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = none ? 0.f : factor * (o[i] * li - o2[i]);
        store8<TYPE>(a.dh, (long long)e * a.d + at, o);
    }
    if (blockIdx.y == 0) event_loss(a, e, a.draft + (long long)e * a.K, dbuf, fbuf);
}

template <int NC, int RB>
hipError_t rows_as(const KdArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)a.E, (unsigned)a.splits);
    if (a.type == EVOSPEC_FP32) kd_rows_kernel<NC, RB, EVOSPEC_FP32><<<grid, kThreads, 0, stream>>>(a);
    else kd_rows_kernel<NC, RB, EVOSPEC_BF16><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

int kd_splits(int E, int K) {
    int s = 512 / E;
    if (s > K / 8) s = K / 8;
    return s < 1 ? 1 : s > 32 ? 32 : s;
}

hipError_t launch_kd(const KdArgs& a, hipStream_t stream) {
    const int pieces = (a.d / 8 + kThreads - 1) / kThreads;
    const hipError_t e = pieces == 1 ? rows_as<1, 8>(a, stream) : pieces == 2 ? rows_as<2, 8>(a, stream) : pieces <= 4 ? rows_as<4, 4>(a, stream) : rows_as<8, 2>(a, stream);
    if (e != hipSuccess || a.splits == 1) return e;
    const dim3 grid((unsigned)a.E, (unsigned)pieces);
    if (a.type == EVOSPEC_FP32) kd_join_kernel<EVOSPEC_FP32><<<grid, kThreads, 0, stream>>>(a);
    else kd_join_kernel<EVOSPEC_BF16><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace evospec
