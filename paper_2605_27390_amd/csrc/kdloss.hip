// The distillation loss on the retained support and its gradient (EvoSpec paper, Eq. 5): for an event with hidden state h and
// support rows W_j, z_j = h . W_j, q = softmax(z / T), p = softmax(target / T),
//   loss = w T^2 sum p (log p - log q)        dh = w T (sum q_j W_j - sum p_j W_j).
// The gradient is attention of one query whose keys and values are the same rows: a row of W_lm is read once, gives its logit, and
// joins two sums, sum exp((z_j - max) / T) W_j under a running maximum and sum p_j W_j, whose weights the targets alone give.  Bound by
// the rows' bytes (K d 2 of an event); an element costs four vector instructions.
// A workgroup has an event, or a part of its rows; a thread has every 256th piece of 8 elements of the rows, of h and of both sums, in
// registers.  The loss is taken from the K logits in 64 bits at the end: near its minimum it is a small difference of large terms.
#include <hip/hip_runtime.h>

#include <cfloat>

#include "adapt.hpp"
#include "common.hpp"

namespace evospec {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMost = EVOSPEC_KD_K_MAX;

// Sums over the workgroup in a fixed order; every thread has them.
template <int N, typename T>
__device__ __forceinline__ void block_sums(T (&x)[N], T (*buf)[N] /*LDS [kWaves][N]*/) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += __shfl_xor(x[i], o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) buf[threadIdx.x >> 6][i] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = buf[0][i];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) x[i] += buf[w][i];
    }
}
// The largest of each, leaving NaN out.
template <int N>
__device__ __forceinline__ void block_max(float (&x)[N], float (*buf)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = wave_max(x[i], threadIdx.x & 63);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) buf[threadIdx.x >> 6][i] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = buf[0][i];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) x[i] = fmaxf(x[i], buf[w][i]);
    }
}

struct LossShared {
    float top[kWaves][2];
    double sum[kWaves][4];
};
// weight T^2 KL(p || q) of an event in 64 bits, by all threads; draft: its logits.  With t and z relative to their largest, over T:
// KL = sum e^t (t - z) / sum e^t - log sum e^t + log sum e^z.
__device__ __forceinline__ void event_loss(const KdArgs& a, int e, const float* draft, LossShared& sh) {
    constexpr int kPer = kMost / kThreads;
    const float inf = __builtin_inff();
    float t[kPer], z[kPer], top[2] = {-inf, -inf};
    int32_t id[kPer];
    bool mine[kPer];
    // (all loads together, of entries that there are not the last one's)
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int j = min(i * kThreads + (int)threadIdx.x, a.K - 1);
        id[i] = a.support[(long long)e * a.K + j];
        t[i] = a.target[(long long)e * a.K + j];
        z[i] = draft[j];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        mine[i] = i * kThreads + (int)threadIdx.x < a.K && (unsigned)id[i] < (unsigned)a.V;
        t[i] = mine[i] ? t[i] : -inf;
        z[i] = mine[i] ? z[i] : -inf;
        top[0] = fmaxf(top[0], t[i]);
        top[1] = fmaxf(top[1], z[i]);
    }
    block_max(top, sh.top);
    const double inv = 1.0 / (double)a.T;
    double s[4] = {};                                            // (the last counts NaN)
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (mine[i]) {
            const double dt = ((double)t[i] - top[0]) * inv, dz = ((double)z[i] - top[1]) * inv, p = exp(dt);
            s[0] += p;
            s[1] += exp(dz);
            if (!(p == 0.0)) s[2] += p * (dt - dz);
            s[3] += t[i] != t[i] ? 1.0 : 0.0;
        }
    block_sums(s, sh.sum);
    if (threadIdx.x == 0) {
        const bool none = top[0] == -inf && s[3] == 0.0;         // no entry, or no target mass
        const double kl = s[2] / s[0] - log(s[0]) + log(s[1]);
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

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// lanes with bit STRIDE keep b's sum with their partner, the others a's
template <int STRIDE>
__device__ __forceinline__ float fold(float a, float b, int lane) {
    const bool high = lane & STRIDE;
    const float keep = high ? b : a, give = high ? a : b;
    return keep + __uint_as_float(xor_lane<STRIDE>(__float_as_uint(give), lane));
}

// What both kernels of the rows begin with: p of this workgroup's entries [j0, j0 + n) of event e and their ids (-1: not in the support), from all
// entries of the event.  True: nothing is learnt from it (no entry, or no target mass), and p is zero.  `meanwhile` is called when
// the ids are there.
struct Entries {
    float p[kMost + 16];
    float z[kMost + 16];
    int32_t ids[kMost + 16];
    LossShared loss;
};
template <typename F>
__device__ __forceinline__ bool entries_of(const KdArgs& a, int e, int j0, int n, Entries& sh, F meanwhile) {
    constexpr int kPer = kMost / kThreads;
    const float inf = __builtin_inff(), inv = 1.f / a.T;
    const int tid = threadIdx.x;
    float t[kPer], top[1] = {-inf};
    int32_t id[kPer];
    bool nan = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {                             // (all loads together, as above)
        const int j = min(i * kThreads + tid, a.K - 1);
        id[i] = a.support[(long long)e * a.K + j];
        t[i] = a.target[(long long)e * a.K + j];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int j = i * kThreads + tid;
        const bool mine = j < a.K && (unsigned)id[i] < (unsigned)a.V;
        t[i] = mine ? t[i] : -inf;
        top[0] = fmaxf(top[0], t[i]);
        nan |= t[i] != t[i];
        if (j >= j0 && j < j0 + n) sh.ids[j - j0] = mine ? id[i] : -1;
    }
    if (tid < 16) sh.ids[n + tid] = -1;                          // (turns may pass the end)
    __syncthreads();
    meanwhile();
    block_max(top, reinterpret_cast<float (*)[1]>(sh.loss.top));
    nan = __syncthreads_or(nan);
    const bool none = top[0] == -inf && !nan;
    float total[1] = {0.f};
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        t[i] = t[i] == -inf ? 0.f : expf((t[i] - top[0]) * inv);
        total[0] += t[i];
    }
    block_sums(total, reinterpret_cast<float (*)[1]>(sh.loss.top));
    const float per = none ? 0.f : 1.f / total[0];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int j = i * kThreads + tid;
        if (j >= j0 && j < j0 + n) sh.p[j - j0] = t[i] * per;
    }
    __syncthreads();
    return none;
}

// The sums over lanes of RB dots at once: lanes whose low bits are r end up with row r's.
template <int RB>
__device__ __forceinline__ float lane_sums(float (&dot)[RB], int lane) {
    if constexpr (RB == 8) {
        const float a = fold<1>(dot[0], dot[1], lane), b = fold<1>(dot[2], dot[3], lane), c = fold<1>(dot[4], dot[5], lane), d = fold<1>(dot[6], dot[7], lane);
        dot[0] = fold<4>(fold<2>(a, b, lane), fold<2>(c, d, lane), lane);
    } else if constexpr (RB == 4) {
        dot[0] = fold<2>(fold<1>(dot[0], dot[1], lane), fold<1>(dot[2], dot[3], lane), lane);
    } else if constexpr (RB == 2) {
        dot[0] = fold<1>(dot[0], dot[1], lane);
    }
    if constexpr (RB < 2) dot[0] += __uint_as_float(xor_lane<1>(__float_as_uint(dot[0]), lane));
    if constexpr (RB < 4) dot[0] += __uint_as_float(xor_lane<2>(__float_as_uint(dot[0]), lane));
    if constexpr (RB < 8) dot[0] += __uint_as_float(xor_lane<4>(__float_as_uint(dot[0]), lane));
    dot[0] += __uint_as_float(xor_lane<8>(__float_as_uint(dot[0]), lane));
    dot[0] += __uint_as_float(xor_lane<16>(__float_as_uint(dot[0]), lane));
    dot[0] += __uint_as_float(xor_lane<32>(__float_as_uint(dot[0]), lane));
    return dot[0];
}

// Running sums of RB rows at a time.  A lane looks after the logit and weights of row `lane % RB` of a turn; all have the same m and l.
// m is a logit, and distances from it are divided by T: logits over T have errors of their own size, or are infinite where T is small.  It begins
// with the least finite number, so that a logit of -inf is a share of zero also before any other.
template <int NC>
struct Sums {
    float m = -FLT_MAX, l = 0.f, o1[NC][8] = {}, o2[NC][8] = {};
    template <int RB>
    __device__ __forceinline__ void add(const u32x4 (&row)[RB][NC], float x, bool mine, float p, float inv, int lane) {
        x = mine ? x : -__builtin_inff();
        float top = x;
        if constexpr (RB >= 2) top = fmaxf(top, __uint_as_float(xor_lane<1>(__float_as_uint(top), lane)));
        if constexpr (RB >= 4) top = fmaxf(top, __uint_as_float(xor_lane<2>(__float_as_uint(top), lane)));
        if constexpr (RB >= 8) top = fmaxf(top, __uint_as_float(xor_lane<4>(__float_as_uint(top), lane)));
        top = fmaxf(top, m);
        if (__builtin_amdgcn_readfirstlane(top != m)) {          // (the same in all lanes)
            const float back = expf((m - top) * inv);
            l *= back;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) o1[c][i] *= back;
            m = top;
        }
        const float q = mine ? expf((x - m) * inv) : 0.f, w = mine ? p : 0.f;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const float qr = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(q), r));
            const float wr = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), r));
            l += qr;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float v = i & 1 ? __uint_as_float(row[r][c][i / 2] & 0xffff0000u) : __uint_as_float(row[r][c][i / 2] << 16);
                    o1[c][i] = fmaf(qr, v, o1[c][i]);
                    o2[c][i] = fmaf(wr, v, o2[c][i]);
                }
        }
    }
};
template <int RB, int NC>
__device__ __forceinline__ void dots_of(const u32x4 (&row)[RB][NC], const u32x4 (&h)[NC], float (&dot)[RB]) {
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        dot[r] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t w = row[r][c][q], x = h[c][q];    // (a bit_cast of a vector's element takes its first one)
                dot[r] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, x), dot[r], false);
            }
    }
}

// Zeros for rows that are not in the support and for what is behind a row's end, which are loaded like the others, from places that are there: a load
// under a condition leaves the compiler without a count of those on their way, and it waits for all (64 events of 4,096 34.0 -> 32.3 us).
template <int RB, int NC>
__device__ __forceinline__ void zeros_in(u32x4 (&row)[RB][NC], const Entries& sh, int at, bool ends, int column, int step, int d) {
    if (ends)
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int c = 0; c < NC; ++c) row[r][c] = column + step * c < d ? row[r][c] : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int r = 0; r < RB; ++r)
        if (__builtin_amdgcn_readfirstlane(sh.ids[at + r]) < 0)
#pragma unroll
            for (int c = 0; c < NC; ++c) row[r][c] = u32x4{0, 0, 0, 0};
}

// Rows of up to 512 NC elements: one to a wavefront, RB at a time; the wavefronts meet at the end.  The other wavefronts' loads are enough: with the next
// rows under way 842 events of 656 elements take 63.8 us, 59.7 without, 400 of 2,048 74.5 and 70.5 (900 of 128 rows 79.4 and 82.9).  Of 513 to 1,024 elements with a
// gradient in bf16 two registers do not fit the four wavefronts to a SIMD and are kept in memory (outside the loop).
template <int NC, int RB, int TYPE>
__global__ __launch_bounds__(kThreads, NC == 4 ? 2 : 4) void kd_rows_kernel(KdArgs a) {
    __shared__ Entries sh;
    __shared__ float joined[2][2][NC * 512];
    __shared__ float2 ml[kWaves];
    const int e = blockIdx.x, part = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int j0 = (int)((long long)a.K * part / a.splits), j1 = (int)((long long)a.K * (part + 1) / a.splits), n = j1 - j0;
    const float inv = 1.f / a.T;
    u32x4 h[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) h[c] = 8 * (64 * c + lane) < a.d ? *(gvec_ptr)((const uint16_t*)a.h + (long long)e * a.d + 8 * (64 * c + lane)) : u32x4{0, 0, 0, 0};
    u32x4 row[RB][NC];
    auto load = [&](u32x4 (&row)[RB][NC], int at) {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int id = at < n ? __builtin_amdgcn_readfirstlane(sh.ids[at + r]) : -1;
            const uint16_t* w = (const uint16_t*)a.W + (long long)(id < 0 ? 0 : id) * a.d;
#pragma unroll
            for (int c = 0; c < NC; ++c) row[r][c] = *(gvec_ptr)(w + min(8 * (64 * c + lane), a.d - 8));
        }
    };
    const bool none = entries_of(a, e, j0, n, sh, [&] { load(row, RB * wave); });
    Sums<NC> s;
    const int mod = lane & (RB - 1);
    auto add = [&](u32x4 (&row)[RB][NC], int at) {
        if (at >= n) return;                                     // (uniform)
        zeros_in(row, sh, at, a.d % (512 * NC) != 0, 8 * lane, 512, a.d);
        float dot[RB];
        dots_of(row, h, dot);
        const float x = lane_sums(dot, lane);
        const bool mine = sh.ids[at + mod] >= 0;
        if (lane < RB) sh.z[at + mod] = mine ? x : __builtin_nanf("");
        s.add(row, x, mine, sh.p[at + mod], inv, lane);
    };
#pragma unroll 1
    for (int at = RB * wave; at < n; at += RB * kWaves) {
        if (at >= RB * kWaves) load(row, at);
        add(row, at);
    }
    // The wavefronts' sums: two give theirs to the other two, then one to the other.
    if (lane == 0) ml[wave] = make_float2(s.m, s.l);
    __syncthreads();
    float m = -FLT_MAX, l = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, ml[w].x);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) l += ml[w].y * expf((ml[w].x - m) * inv);
    const float mine = expf((s.m - m) * inv);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) s.o1[c][i] *= mine;
#pragma unroll
    for (int half = kWaves / 2; half > 0; half >>= 1) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                store8<EVOSPEC_FP32>(joined[wave - half][0], 8 * (64 * c + lane), s.o1[c]);
                store8<EVOSPEC_FP32>(joined[wave - half][1], 8 * (64 * c + lane), s.o2[c]);
            }
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s.o1[c][i] += joined[wave][0][8 * (64 * c + lane) + i];
                    s.o2[c][i] += joined[wave][1][8 * (64 * c + lane) + i];
                }
        __syncthreads();
    }
    for (int j = tid; j < n; j += kThreads) a.draft[(long long)e * a.K + j0 + j] = sh.z[j];
    if (wave == 0) {
        if (a.splits == 1) {
            const float factor = (a.weight ? a.weight[e] : 1.f) * a.T, li = 1.f / l;
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (8 * (64 * c + lane) < a.d) {
                    float g[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] = none ? 0.f : factor * (s.o1[c][i] * li - s.o2[c][i]);
                    store8<TYPE>(a.dh, (long long)e * a.d + 8 * (64 * c + lane), g);
                }
        } else {
            float* out = a.part + ((long long)e * a.splits + part) * 2 * a.d;
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (8 * (64 * c + lane) < a.d) {
                    store8<EVOSPEC_FP32>(out, 8 * (64 * c + lane), s.o1[c]);
                    store8<EVOSPEC_FP32>(out, a.d + 8 * (64 * c + lane), s.o2[c]);
                }
            if (lane == 0) a.part_ml[(long long)e * a.splits + part] = make_float2(m, none ? -1.f : l);
        }
    }
    if (a.splits == 1) event_loss(a, e, sh.z, sh.loss);
}

// Longer rows: one to the workgroup, NC pieces of 8 elements to a thread.
template <int NC, int RB, int TYPE>
__global__ __launch_bounds__(kThreads, NC * RB <= 4 ? 3 : 1) void kd_long_rows_kernel(KdArgs a) {
    __shared__ Entries sh;
    __shared__ __align__(16) float dots[2][RB][kWaves];
    const int e = blockIdx.x, part = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int j0 = (int)((long long)a.K * part / a.splits), j1 = (int)((long long)a.K * (part + 1) / a.splits), n = j1 - j0;
    const float inv = 1.f / a.T;
    bool in[NC];
    u32x4 h[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        in[c] = 8 * (c * kThreads + tid) < a.d;
        h[c] = in[c] ? *(gvec_ptr)((const uint16_t*)a.h + (long long)e * a.d + 8 * (c * kThreads + tid)) : u32x4{0, 0, 0, 0};
    }
    u32x4 row[RB][NC], next[RB][NC];
    auto load = [&](u32x4 (&row)[RB][NC], int at) {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int id = at < n ? __builtin_amdgcn_readfirstlane(sh.ids[at + r]) : -1;
            const uint16_t* w = (const uint16_t*)a.W + (long long)(id < 0 ? 0 : id) * a.d;
#pragma unroll
            for (int c = 0; c < NC; ++c) row[r][c] = *(gvec_ptr)(w + min(8 * (c * kThreads + tid), a.d - 8));
        }
    };
    const bool none = entries_of(a, e, j0, n, sh, [&] { load(row, 0); });
    Sums<NC> s;
    const int mod = lane & (RB - 1);
    auto add = [&](u32x4 (&row)[RB][NC], int at, int turn) {
        zeros_in(row, sh, at, a.d % (8 * NC * kThreads) != 0, 8 * tid, 8 * kThreads, a.d);
        float dot[RB];
        dots_of(row, h, dot);
        const float sum = lane_sums(dot, lane);
        if (lane < RB) dots[turn][lane][wave] = sum;
        lds_barrier();                                           // (the rows under way stay so; the two halves of dots take turns)
        if (at >= n) return;                                     // (uniform)
        const float4 d = *reinterpret_cast<const float4*>(dots[turn][mod]);
        const float x = (d.x + d.y) + (d.z + d.w);
        const bool mine = sh.ids[at + mod] >= 0;
        if (tid < RB) sh.z[at + mod] = mine ? x : __builtin_nanf("");
        s.add(row, x, mine, sh.p[at + mod], inv, lane);
    };
    // (the next rows are under way; one loop with rows handed on, not two rows' sets in turn: a launch has half the instructions to bring in.  192 events
    // 76.5 and 76.2 us, 300 123 and 115, 64 alike; here and below the launches alone, one after the other: in a pass over other inputs each time 192 events take 79)
#pragma unroll 1
    for (int at = 0, turn = 0; at < n; at += RB, turn ^= 1) {
        load(next, at + RB);
        add(row, at, turn);
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int c = 0; c < NC; ++c) row[r][c] = next[r][c];
    }
    __syncthreads();
    for (int j = tid; j < n; j += kThreads) a.draft[(long long)e * a.K + j0 + j] = sh.z[j];
    if (a.splits == 1) {
        const float factor = (a.weight ? a.weight[e] : 1.f) * a.T, li = 1.f / s.l;
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (in[c]) {
                float g[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = none ? 0.f : factor * (s.o1[c][i] * li - s.o2[c][i]);
                store8<TYPE>(a.dh, (long long)e * a.d + 8 * (c * kThreads + tid), g);
            }
        event_loss(a, e, sh.z, sh.loss);
    } else {
        float* out = a.part + ((long long)e * a.splits + part) * 2 * a.d;
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (in[c]) {
                store8<EVOSPEC_FP32>(out, 8 * (c * kThreads + tid), s.o1[c]);
                store8<EVOSPEC_FP32>(out, a.d + 8 * (c * kThreads + tid), s.o2[c]);
            }
        if (tid == 0) a.part_ml[(long long)e * a.splits + part] = make_float2(s.m, none ? -1.f : s.l);
    }
}

// Joins the parts of an event's rows: V elements of its gradient to a thread, whose parts (N at a time) are asked for together; a workgroup
// of its own takes the loss.
template <int TYPE, int V, int N>
__global__ __launch_bounds__(kThreads) void kd_join_kernel(KdArgs a) {
    __shared__ LossShared loss;
    if (blockIdx.y == 0) {
        event_loss(a, blockIdx.x, a.draft + (long long)blockIdx.x * a.K, loss);
        return;
    }
    typedef float vec __attribute__((ext_vector_type(V)));
    const int e = blockIdx.x, lane = threadIdx.x & 63, at = V * (((int)blockIdx.y - 1) * kThreads + (int)threadIdx.x);
    if (at - V * lane >= a.d) return;                            // (whole wavefronts)
    const float* part = a.part + (long long)e * a.splits * 2 * a.d + min(at, a.d - V);
    const float inf = __builtin_inff();
    // lane s has the reference, sum and factor of part s (there are at most 32)
    const float2 mine = lane < a.splits ? a.part_ml[(long long)e * a.splits + lane] : make_float2(-inf, 0.f);
    vec u[N], v[N], o = {}, o2 = {};
    auto load = [&](int s0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float* p = part + (long long)min(s0 + i, a.splits - 1) * 2 * a.d;
            u[i] = *reinterpret_cast<const vec*>(p);
            v[i] = *reinterpret_cast<const vec*>(p + a.d);
        }
    };
    load(0);
    const float m = wave_max(mine.x, lane);
    const bool none = __ballot(mine.y == -1.f) != 0;
    const float factor = expf((mine.x - m) * (1.f / a.T));       // (a part without entries has sums of zero)
    const float l = wave_sum(mine.y * factor, lane);
    for (int s0 = 0;; load(s0)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            // (without a way past the addition, which would have each part's loads wait for the one before)
            const bool there = s0 + i < a.splits;
            const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(factor), (s0 + i) & 63));
#pragma unroll
            for (int k = 0; k < V; ++k) {
                o[k] = there ? fmaf(f, u[i][k], o[k]) : o[k];
                o2[k] = there ? o2[k] + v[i][k] : o2[k];
            }
        }
        if ((s0 += N) >= a.splits) break;
    }
    if (at >= a.d) return;
    const float all = (a.weight ? a.weight[e] : 1.f) * a.T, li = 1.f / l;
#pragma unroll
    for (int k = 0; k < V; ++k) o[k] = none ? 0.f : all * (o[k] * li - o2[k]);
    if constexpr (TYPE == EVOSPEC_FP32) {
        *reinterpret_cast<vec*>((float*)a.dh + (long long)e * a.d + at) = o;
    } else {
        typedef __bf16 out __attribute__((ext_vector_type(V)));
        out x;
#pragma unroll
        for (int k = 0; k < V; ++k) x[k] = (__bf16)o[k];
        *reinterpret_cast<out*>((__bf16*)a.dh + (long long)e * a.d + at) = x;
    }
}

template <int NC, int RB, bool LONG>
hipError_t rows_as(const KdArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)a.E, (unsigned)a.splits);
    if constexpr (LONG) {
        if (a.type == EVOSPEC_FP32) kd_long_rows_kernel<NC, RB, EVOSPEC_FP32><<<grid, kThreads, 0, stream>>>(a);
        else kd_long_rows_kernel<NC, RB, EVOSPEC_BF16><<<grid, kThreads, 0, stream>>>(a);
    } else {
        if (a.type == EVOSPEC_FP32) kd_rows_kernel<NC, RB, EVOSPEC_FP32><<<grid, kThreads, 0, stream>>>(a);
        else kd_rows_kernel<NC, RB, EVOSPEC_BF16><<<grid, kThreads, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

// An event's rows are split until the parts come to one round of workgroups, two to a compute unit, one above 8,192 elements.  Three to a unit where rows
// have 2,048 to 4,096 elements and two would leave a seventh of the card empty; of more than 3,600, where it takes more than four parts, which have to be joined, a
// fifth.  256 rows, us with two and with three:
//             109 events in 4 and 7 parts   129 in 3 and 5   146 in 3 and 5   192 in 2 and 4   205 in 2 and 3
//   of 3,200          44.6   39.8             55.7   47.4      56.3   49.2      79.0   59.5      79.6   70.2
//   of 3,600          45.5   45.4             56.8   51.0      57.7   55.6      80.7   67.9      81.4   74.0
//   of 3,800          46.1   47.3             57.2   53.6      58.7   59.0      81.6   71.7      82.3   78.1
//   of 4,096          45.7   49.7             56.3   56.1      58.4   61.7      80.5   76.4      82.1   82.5
// (of 4,096, 102 events in 4 and 5 44.8 and 44.1, 256 in 2 and 3 93.3 and 97.1, 300 in 1 and 2 139 and 115, 400 143 and 159.)  Shorter rows gain nothing from three (400
// events of 2,048 in 1 and 2 parts 73.6 and 83.3, 338 of 344 20.0 and 21.3).
int kd_splits(int E, int K, int d) {
    int most = d > 8192 ? 256 : 512;
    if (d > 2048 && d <= 4096 && E > 100 && most / E * E < most - most / (d > 3600 && 768 / E > 4 ? 5 : 7)) most = 768;
    int s = most / E;
    if (s > K / 8) s = K / 8;
    return s < 1 ? 1 : s > 32 ? 32 : s;
}

hipError_t launch_kd(const KdArgs& a, hipStream_t stream) {
    // (a row to a wavefront takes a quarter of the time of a row to a workgroup at 680 elements, 548 events 47 and 179 us, and half at 2,048; at 4,096 its sums and rows
    // spill: 165 us for 192 events, 79.  Two rows of 4,096 at a time, four where a part has 8 rows at most: one event 12.2 and 11.6, 48 events 28.4 and 29.9)
    const hipError_t e = a.d <= 512 ? rows_as<1, 8, false>(a, stream) : a.d <= 1024 ? rows_as<2, 4, false>(a, stream) : a.d <= 2048 ? rows_as<4, 2, false>(a, stream)
                         : a.d <= 4096 ? (a.K <= 8 * a.splits ? rows_as<2, 4, true>(a, stream) : rows_as<2, 2, true>(a, stream)) : a.d <= 8192 ? rows_as<4, 2, true>(a, stream) : rows_as<8, 1, true>(a, stream);
    if (e != hipSuccess || a.splits == 1) return e;
    const int v = a.splits <= 8 ? 4 : 2;
    const dim3 grid((unsigned)a.E, (unsigned)(1 + (a.d + v * kThreads - 1) / (v * kThreads)));
    if (v == 4) {
        if (a.type == EVOSPEC_FP32) kd_join_kernel<EVOSPEC_FP32, 4, 4><<<grid, kThreads, 0, stream>>>(a);
        else kd_join_kernel<EVOSPEC_BF16, 4, 4><<<grid, kThreads, 0, stream>>>(a);
    } else {
        if (a.type == EVOSPEC_FP32) kd_join_kernel<EVOSPEC_FP32, 2, 32><<<grid, kThreads, 0, stream>>>(a);
        else kd_join_kernel<EVOSPEC_BF16, 2, 32><<<grid, kThreads, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace evospec
