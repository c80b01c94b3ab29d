// AdamW over many tensors at once, with moments in 32 or in 8 bits (evospec_adapt.h has the formulas and the codes).
//
// Every element is read and written once: 22 bytes with moments in 32 bits beside bf16 parameters, 10 with 8 bits.  A wavefront has
// blocks of 256 elements, 4 in a row to a lane, so that the largest magnitude of a block is a reduction within it.  Addresses
// of up to kTensors tensors go along with the launch itself; a wavefront finds its block's tensor by one comparison in every lane.
// Measured, bf16: 134 million elements with 32 bits 546 us (5.4 TB/s; a copy of 1 GiB reaches 5.14), with 8 bits 293 us (4.6 TB/s: some 60 vector instructions
// an element, half of them the rounding's hash and codes, are nearly as long), with 8 bits and masters 370 us (5.8 TB/s).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "adapt.hpp"
#include "common.hpp"

namespace evospec {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kBlock = EVOSPEC_ADAMW_BLOCK;
constexpr int kTensors = 112;                 // of a launch: 28 bytes each, of 4 KB of arguments

struct Table {
    uint64_t param[kTensors], grad[kTensors];
    uint64_t n[kTensors];
    uint32_t first[kTensors];                 // block, counted from the launch's first
    int count;
    uint32_t blocks;
    long long base;                           // the launch's first block
};
static_assert(sizeof(Table) <= 3500, "arguments of a launch");

template <int TYPE>
struct Element;
template <>
struct Element<EVOSPEC_BF16> {
    using type = __bf16;
};
template <>
struct Element<EVOSPEC_FP16> {
    using type = _Float16;
};
template <>
struct Element<EVOSPEC_FP32> {
    using type = float;
};

// (addresses that come out of a table: said to be global memory, whose loads do not go through the checks of flat ones)
#define GLOBAL __attribute__((address_space(1)))

// 4 elements from `at` on; of a tensor's end those that there are, and zeros.
template <int TYPE>
__device__ __forceinline__ void load4(uint64_t base, long long at, int there, float (&x)[4]) {
    using T = typename Element<TYPE>::type;
    typedef T vec __attribute__((ext_vector_type(4)));
    const GLOBAL T* p = (const GLOBAL T*)base + at;
    if (there >= 4) {
        const vec v = *(const GLOBAL vec*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = i < there ? (float)p[i] : 0.f;
    }
}
template <int TYPE>
__device__ __forceinline__ void store4(uint64_t base, long long at, int there, const float (&x)[4]) {
    using T = typename Element<TYPE>::type;
    typedef T vec __attribute__((ext_vector_type(4)));
    GLOBAL T* p = (GLOBAL T*)base + at;
    if (there >= 4) {
        *(GLOBAL vec*)p = vec{(T)x[0], (T)x[1], (T)x[2], (T)x[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < there) p[i] = (T)x[i];
    }
}

// 2^e, the least from 2^-100 to 2^100 with amax <= most 2^e, most = (1 + FRACTION / 2^23) 2^LEAST
template <int LEAST, uint32_t FRACTION>
__device__ __forceinline__ float power_for(uint32_t u /*amax as bits*/) {
    const int e = (int)(u >> 23) - 127 - LEAST + ((u & 0x7fffffu) > FRACTION);
    return __uint_as_float((uint32_t)(min(max(e, -100), 100) + 127) << 23);
}
__device__ __forceinline__ float reciprocal(float power) { return __uint_as_float((254u << 23) - __float_as_uint(power)); }

// The largest of the wavefront, as a scalar: within 16 lanes by exchanges that ride on the comparison, then four lanes' values.
template <int CTRL>
__device__ __forceinline__ uint32_t larger(uint32_t x) { return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true)); }
__device__ __forceinline__ uint32_t wave_top(uint32_t x) {
    x = larger<0x140>(larger<0x141>(larger<0x4E>(larger<0xB1>(x))));         // neighbours, pairs, halves of 8 mirrored, 16 mirrored
    const uint32_t a = __builtin_amdgcn_readlane(x, 0), b = __builtin_amdgcn_readlane(x, 16), c = __builtin_amdgcn_readlane(x, 32), d = __builtin_amdgcn_readlane(x, 48);
    const uint32_t ab = a > b ? a : b, cd = c > d ? c : d;
    return ab > cd ? ab : cd;
}

// The code of a magnitude that is divided by its scale; bits: 16 random ones.
template <int BIAS>
__device__ __forceinline__ uint32_t code_of(float y, uint32_t bits) {
    const float least = __uint_as_float((uint32_t)(128 - BIAS) << 23);
    const bool tiny = y < least;
    const uint32_t b = __float_as_uint(tiny ? y + least : y) + (bits << 4);
    return (b >> 20) - (tiny ? (128 - BIAS) * 8 : (127 - BIAS) * 8);
}
__device__ __forceinline__ float v_value(uint32_t code) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(code << 7)); }

__device__ __forceinline__ uint32_t random_bits(uint32_t place, uint32_t key) {
    uint32_t x = place * 0x9e3779b1u + key;
    x = (x ^ (x >> 16)) * 0x21f0aaadu;
    x = (x ^ (x >> 15)) * 0x735a2d97u;
    return x ^ (x >> 15);
}

// A wavefront's blocks, all of whose loads are under way before the first is looked at.
template <int PT, int GT, int KIND, bool MASTER, int U>
__global__ __launch_bounds__(kThreads) void adamw_kernel(Table table, AdamwArgs a) {
    const int lane = threadIdx.x & 63;
    const uint32_t block0 = (blockIdx.x * kWaves + (threadIdx.x >> 6)) * U;
    if (block0 >= table.blocks) return;
    uint32_t first[(kTensors + 63) / 64];
#pragma unroll
    for (int i = 0; i < (kTensors + 63) / 64; ++i) {
        const int t = 64 * i + lane;
        first[i] = t < table.count ? table.first[min(t, kTensors - 1)] : 0xffffffffu;
    }
    const float scale = a.grad_scale ? *a.grad_scale : 1.f;
    if (!(fabsf(scale) < __builtin_inff())) return;
    float decay = a.decay, rate = a.rate, root = a.root;
    uint32_t key = a.seed_key + a.t_key;
    if (a.schedule) {
        const float lr = a.schedule[0], t = a.schedule[1];
        decay = 1.f - lr * a.weight_decay;
        rate = lr / -expm1f(t * a.log_beta1);
        root = 1.f / sqrtf(-expm1f(t * a.log_beta2));
        key = a.seed_key + (uint32_t)t * 0xc2b2ae35u;
    }
    int there[U];
    uint64_t param[U];
    long long within[U];
    float g[U][4], p[U][4], m[U][4], v[U][4];
    uint32_t cm[U], cv[U];
    float2 s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        // the last tensor that begins at or before the block
        const uint32_t block = min(block0 + u, table.blocks - 1);
        int at = -1;
#pragma unroll
        for (int i = 0; i < (kTensors + 63) / 64; ++i) at += __popcll(__ballot(first[i] <= block));
        at = __builtin_amdgcn_readfirstlane(at);
        param[u] = table.param[at];
        within[u] = (long long)(block - table.first[at]) * kBlock + 4 * lane;
        const long long flat = (table.base + block) * kBlock + 4 * lane, rest = (long long)table.n[at] - within[u];
        there[u] = rest >= 4 ? 4 : rest > 0 ? (int)rest : 0;
        load4<GT>(table.grad[at], within[u], there[u], g[u]);
        if constexpr (MASTER) load4<EVOSPEC_FP32>((uint64_t)a.master, flat, 4, p[u]);
        else load4<PT>(param[u], within[u], there[u], p[u]);
        if constexpr (KIND == EVOSPEC_MOMENTS_8BIT) {
            cm[u] = *(const uint32_t*)((const uint8_t*)a.m + flat);
            cv[u] = *(const uint32_t*)((const uint8_t*)a.v + flat);
            s[u] = reinterpret_cast<const float2*>(a.scales)[table.base + block];
        } else {
            load4<EVOSPEC_FP32>((uint64_t)a.m, flat, 4, m[u]);
            load4<EVOSPEC_FP32>((uint64_t)a.v, flat, 4, v[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (block0 + u >= table.blocks) return;                  // (the same in all lanes)
        const long long flat = (table.base + block0 + u) * kBlock + 4 * lane;
        if constexpr (KIND == EVOSPEC_MOMENTS_8BIT) {
            m[u][0] = __builtin_amdgcn_cvt_f32_fp8((int)cm[u], 0) * s[u].x;
            m[u][1] = __builtin_amdgcn_cvt_f32_fp8((int)cm[u], 1) * s[u].x;
            m[u][2] = __builtin_amdgcn_cvt_f32_fp8((int)cm[u], 2) * s[u].x;
            m[u][3] = __builtin_amdgcn_cvt_f32_fp8((int)cm[u], 3) * s[u].x;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[u][i] = v_value((cv[u] >> (8 * i)) & 255u) * s[u].y;
        }
        uint32_t top_m = 0, top_v = 0;                           // magnitudes as bits, whose order is theirs; NaN and infinity are the largest
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i >= there[u]) p[u][i] = m[u][i] = v[u][i] = 0.f;            // (g is)
            const float x = g[u][i] * scale;
            {
                // Each product and sum rounded by itself: a bit in a moment can be a code's step, an eighth of it, and so the codes are those of the
                // formulas computed one operation after the other in fp32, anywhere.  (Fused, 117 of 134 million codes of m differed.)
#pragma clang fp contract(off)
                m[u][i] = a.beta1 * m[u][i] + a.beta1c * x;
                v[u][i] = a.beta2 * v[u][i] + a.beta2c * (x * x);
            }
            // (reciprocal and root to the last bit or so: 2^-23 of an update, which is itself small beside p)
            p[u][i] = fmaf(p[u][i], decay, -(rate * m[u][i]) * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(v[u][i]), root, a.eps)));
            if constexpr (KIND == EVOSPEC_MOMENTS_8BIT) {
                top_m = max(top_m, __float_as_uint(m[u][i]) & 0x7fffffffu);
                top_v = max(top_v, __float_as_uint(v[u][i]));
            }
        }
        store4<PT>(param[u], within[u], there[u], p[u]);
        if constexpr (MASTER) store4<EVOSPEC_FP32>((uint64_t)a.master, flat, 4, p[u]);
        if constexpr (KIND == EVOSPEC_MOMENTS_8BIT) {
            top_m = wave_top(top_m);
            top_v = wave_top(top_v);
            // what is rare, a NaN, an infinity or what the largest scale does not take, has a way of its own
            const bool rare = max(top_m, top_v) >= __float_as_uint(0x1p108f);
            if (rare) {
                top_m = top_v = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (fabsf(m[u][i]) < __builtin_inff() && v[u][i] < __builtin_inff()) {
                        top_m = max(top_m, __float_as_uint(m[u][i]) & 0x7fffffffu);
                        top_v = max(top_v, __float_as_uint(v[u][i]));
                    }
                top_m = wave_top(top_m);
                top_v = wave_top(top_v);
            }
            const float sm = power_for<8, 0x600000u>(top_m), sv = power_for<15, 0x700000u>(top_v);
            const float im = reciprocal(sm), iv = reciprocal(sv);
            uint32_t xm = 0, xv = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t bits = random_bits((uint32_t)(flat + i), key);
                const float y = fabsf(m[u][i]) * im, z = v[u][i] * iv;
                const uint32_t cy = code_of<7>(y, bits & 0xffffu), cz = max(code_of<15>(z, bits >> 16), v[u][i] > 0.f ? 1u : 0u);
                xm |= (cy | (__float_as_uint(m[u][i]) >> 31) << 7) << (8 * i);
                xv |= cz << (8 * i);
            }
            if (rare) {
                xm = xv = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t bits = random_bits((uint32_t)(flat + i), key);
                    const bool fine = fabsf(m[u][i]) < __builtin_inff() && v[u][i] < __builtin_inff();
                    const uint32_t cy = code_of<7>(fminf(fabsf(m[u][i]) * im, 448.f), bits & 0xffffu) | (__float_as_uint(m[u][i]) >> 31) << 7;
                    const uint32_t cz = max(code_of<15>(fminf(v[u][i] * iv, 61440.f), bits >> 16), v[u][i] > 0.f ? 1u : 0u);
                    xm |= (fine ? cy : 0x7fu) << (8 * i);
                    xv |= (fine ? cz : 0xf7u) << (8 * i);
                }
            }
            *(GLOBAL uint32_t*)((uint64_t)a.m + flat) = xm;
            *(GLOBAL uint32_t*)((uint64_t)a.v + flat) = xv;
            if (lane == 0) reinterpret_cast<float2*>(a.scales)[table.base + block0 + u] = make_float2(sm, sv);
        } else {
            store4<EVOSPEC_FP32>((uint64_t)a.m, flat, 4, m[u]);
            store4<EVOSPEC_FP32>((uint64_t)a.v, flat, 4, v[u]);
        }
    }
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void adamw_moments_kernel(const uint8_t* m, const uint8_t* v, const float2* scales, long long blocks,
                                                                 void* out_m, void* out_v) {
    const long long block = (long long)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (block >= blocks) return;
    const long long flat = block * kBlock + 4 * (threadIdx.x & 63);
    const float2 s = scales[block];
    const uint32_t cm = *(const uint32_t*)(m + flat), cv = *(const uint32_t*)(v + flat);
    const float x[4] = {__builtin_amdgcn_cvt_f32_fp8((int)cm, 0) * s.x, __builtin_amdgcn_cvt_f32_fp8((int)cm, 1) * s.x,
                        __builtin_amdgcn_cvt_f32_fp8((int)cm, 2) * s.x, __builtin_amdgcn_cvt_f32_fp8((int)cm, 3) * s.x};
    const float y[4] = {v_value(cv & 255u) * s.y, v_value((cv >> 8) & 255u) * s.y, v_value((cv >> 16) & 255u) * s.y, v_value(cv >> 24) * s.y};
    store4<TYPE>((uint64_t)out_m, flat, 4, x);
    store4<TYPE>((uint64_t)out_v, flat, 4, y);
}

template <int I>
using Const = std::integral_constant<int, I>;

}  // namespace

hipError_t launch_adamw(const evospec_adamw_tensor* tensors, int count, int param_type, int grad_type, int kind, const AdamwArgs& a,
                        hipStream_t stream) {
    long long base = 0;
    for (int at = 0; at < count;) {
        Table t{};
        t.base = base;
        long long blocks = 0;
        for (; at < count && t.count < kTensors; ++at) {
            const long long more = (tensors[at].n + kBlock - 1) / kBlock;
            if (more == 0) continue;
            if (blocks + more > (1ll << 25)) break;              // (the C entry takes tensors of up to that many blocks)
            t.param[t.count] = (uint64_t)tensors[at].param;
            t.grad[t.count] = (uint64_t)tensors[at].grad;
            t.n[t.count] = (uint64_t)tensors[at].n;
            t.first[t.count++] = (uint32_t)blocks;
            blocks += more;
        }
        if (blocks == 0) break;
        t.blocks = (uint32_t)blocks;
        auto go = [&](auto pt, auto gt, auto kd, auto ms) {
            // (134 million elements with 8 bits in 1, 2, 4 blocks to a wavefront 325, 297, 316 us; with masters 373, 391, 401, and with 32 bits 548,
            // 551, 550: enough is under way)
            constexpr int U = kd.value == EVOSPEC_MOMENTS_8BIT && ms.value == 0 ? 2 : 1;
            const dim3 grid((unsigned)((blocks + kWaves * U - 1) / (kWaves * U)));
            adamw_kernel<pt.value, gt.value, kd.value, (bool)ms.value, U><<<grid, kThreads, 0, stream>>>(t, a);
        };
        auto with_kind = [&](auto pt, auto gt) {
            if (kind == EVOSPEC_MOMENTS_8BIT) a.master ? go(pt, gt, Const<1>{}, Const<1>{}) : go(pt, gt, Const<1>{}, Const<0>{});
            else a.master ? go(pt, gt, Const<0>{}, Const<1>{}) : go(pt, gt, Const<0>{}, Const<0>{});
        };
        if (param_type == EVOSPEC_FP32) with_kind(Const<EVOSPEC_FP32>{}, Const<EVOSPEC_FP32>{});
        else if (param_type == EVOSPEC_BF16)
            grad_type == EVOSPEC_FP32 ? with_kind(Const<EVOSPEC_BF16>{}, Const<EVOSPEC_FP32>{}) : with_kind(Const<EVOSPEC_BF16>{}, Const<EVOSPEC_BF16>{});
        else
            grad_type == EVOSPEC_FP32 ? with_kind(Const<EVOSPEC_FP16>{}, Const<EVOSPEC_FP32>{}) : with_kind(Const<EVOSPEC_FP16>{}, Const<EVOSPEC_FP16>{});
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        base += blocks;
    }
    return hipSuccess;
}

hipError_t launch_adamw_moments(const void* m, const void* v, const float* scales, long long blocks, int type, void* out_m, void* out_v,
                                hipStream_t stream) {
    constexpr long long kMost = 1ll << 25;                       // (a launch has fewer than 2^32 threads)
    for (long long at = 0; at < blocks; at += kMost) {
        const long long count = std::min(blocks - at, kMost), place = at * kBlock;
        const dim3 grid((unsigned)((count + kWaves - 1) / kWaves));
        const float2* s = reinterpret_cast<const float2*>(scales) + at;
        const uint8_t *cm = (const uint8_t*)m + place, *cv = (const uint8_t*)v + place;
        if (type == EVOSPEC_FP32) adamw_moments_kernel<EVOSPEC_FP32><<<grid, kThreads, 0, stream>>>(cm, cv, s, count, (float*)out_m + place, (float*)out_v + place);
        else adamw_moments_kernel<EVOSPEC_BF16><<<grid, kThreads, 0, stream>>>(cm, cv, s, count, (__bf16*)out_m + place, (__bf16*)out_v + place);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace evospec
