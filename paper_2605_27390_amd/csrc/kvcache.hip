// The 8-bit key/value cache: new tokens are quantised as they are written, and read back as values.
//
// x is kept as code = round(x / s) of 8 bits, s the scale of a block (32 tokens of one head, K and V apart).  For e4m3, s is
// a power of two, so that a block whose scale grows loses nothing but what falls below the smallest code; int8 codes are
// rounded again.  One workgroup of 4 wavefronts owns a (block, head): its largest magnitude needs all of the block's new
// elements, which stay in registers between the maximum and the rounding (one pass over the input).  Both ways go
// through LDS: global memory sees rows of `dim` elements on the caller's side, and 16-byte pieces in the order of the
// matrix cores' operands (evospec_decode.h) on the cache's.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "common.hpp"
#include "decode.hpp"

namespace evospec {
namespace {

constexpr int kThreads = 256;

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

// 4 codes of a dword from 4 values that are divided by the scale already.  v_cvt_pk_fp8_f32 rounds to nearest even.
template <int KIND>
__device__ __forceinline__ uint32_t encode4(const float* y) {
    if constexpr (KIND == EVOSPEC_KV_E4M3) {
        float c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = y[i] != y[i] ? y[i] : fminf(fmaxf(y[i], -448.f), 448.f);
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], p, true);
    } else {
        uint32_t p = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int q = y[i] != y[i] ? -128 : (int)fminf(fmaxf(rintf(y[i]), -127.f), 127.f);
            p |= (uint32_t)(q & 255) << (8 * i);
        }
        return p;
    }
}
template <int KIND>
__device__ __forceinline__ void decode4(uint32_t p, float* y) {
    if constexpr (KIND == EVOSPEC_KV_E4M3) {
        y[0] = __builtin_amdgcn_cvt_f32_fp8((int)p, 0);
        y[1] = __builtin_amdgcn_cvt_f32_fp8((int)p, 1);
        y[2] = __builtin_amdgcn_cvt_f32_fp8((int)p, 2);
        y[3] = __builtin_amdgcn_cvt_f32_fp8((int)p, 3);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int q = (int)(int8_t)(p >> (8 * i));
            y[i] = q == -128 ? __uint_as_float(0x7fc00000u) : (float)q;
        }
    }
}

// The scale of a block whose largest finite magnitude is amax.
template <int KIND>
__device__ __forceinline__ float scale_of(float amax) {
    if constexpr (KIND == EVOSPEC_KV_E4M3) {
        const uint32_t u = __float_as_uint(amax);
        // amax = f 2^x, f in [1, 2); 448 = 1.75 * 2^8
        int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
        e = e < -100 ? -100 : e > 120 ? 120 : e;
        return __uint_as_float((uint32_t)(e + 127) << 23);
    } else {
        return fmaxf(amax / 127.f, 0x1p-100f);
    }
}

// Sequence, head and block of a workgroup, and which of the block's tokens are rows of the call.
struct Task {
    int s, head;
    int block;                  // of the sequence
    int first, last;            // tokens [first, last) of the block (0 .. 32) are rows
    int row;                    // row of the block's token 0 (may be negative; only tokens in [first, last) are rows)
    bool fresh;                 // token 0 of the block is among them, or no token is older
    int old;                    // tokens [0, old) of the block are older
    long long at;               // its place: (page * heads + head) blocks in, -1 if it has none
};
__device__ __forceinline__ Task task_of(const Cache& c, const Rows& r, int per, int id) {
    Task t;
    t.head = id % c.heads;
    id /= c.heads;
    const int j = id % per;
    t.s = id / per;
    const int n0 = min(max(r.row_off[t.s], 0), r.T), n1 = min(max(r.row_off[t.s + 1], n0), r.T);
    const int n = min(n1 - n0, r.max_rows);
    const int start = max(r.at[t.s], 0);
    t.block = start / kBlock + j;
    const long long token = (long long)t.block * kBlock;
    t.first = (int)max(0ll, start - token);
    t.last = (int)min((long long)kBlock, (long long)start + n - token);      // <= first where the block is not touched
    t.old = t.first;
    t.fresh = t.old == 0;
    t.row = n0 + (int)(token - start);
    t.at = -1;
    if (t.last > t.first && (t.block >> c.shift) < r.width) {
        const int page = r.table[(long long)t.s * r.width + (t.block >> c.shift)];
        if ((unsigned)page < (unsigned)c.pages)
            t.at = ((((long long)page * c.heads + t.head) << c.shift) + (t.block & ((1 << c.shift) - 1)));
    }
    return t;
}

// Bytes of a block's tokens in LDS: a row of dim bytes, 16 more so that pieces of neighbouring tokens lie in other banks.
template <int DIM>
constexpr int kRow = DIM + 16;

// Piece p (16 bytes) of a block: K's is one token's 16 dimensions, V's 16 tokens of one dimension.
template <int DIM, bool V>
__device__ __forceinline__ u32x4 piece_from_rows(const uint8_t* rows, int p) {
    const int s = p >> 6, g = (p >> 5) & 1, m = p & 31;
    if constexpr (!V) {
        return *reinterpret_cast<const u32x4*>(rows + m * kRow<DIM> + 32 * s + 16 * g);
    } else {
        u32x4 x;
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) w |= (uint32_t)rows[(8 * a + 4 * g + i) * kRow<DIM> + 32 * s + m] << (8 * i);
            x[a] = w;
        }
        return x;
    }
}
template <int DIM, bool V>
__device__ __forceinline__ void piece_to_rows(uint8_t* rows, int p, u32x4 x) {
    const int s = p >> 6, g = (p >> 5) & 1, m = p & 31;
    if constexpr (!V) {
        *reinterpret_cast<u32x4*>(rows + m * kRow<DIM> + 32 * s + 16 * g) = x;
    } else {
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int i = 0; i < 4; ++i) rows[(8 * a + 4 * g + i) * kRow<DIM> + 32 * s + m] = (uint8_t)(x[a] >> (8 * i));
    }
}

// 8 elements of a row as floats
template <int TYPE>
__device__ __forceinline__ void load8(const typename Element<TYPE>::type* p, float* x) {
    if constexpr (TYPE == EVOSPEC_FP32) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        typedef typename Element<TYPE>::type vec __attribute__((ext_vector_type(8)));
        const vec v = *reinterpret_cast<const vec*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
    }
}
template <int TYPE>
__device__ __forceinline__ void store8(typename Element<TYPE>::type* p, const float* x) {
    if constexpr (TYPE == EVOSPEC_FP32) {
        reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        typedef typename Element<TYPE>::type vec __attribute__((ext_vector_type(8)));
        vec v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (typename Element<TYPE>::type)x[i];
        *reinterpret_cast<vec*>(p) = v;
    }
}

// Quantises the new tokens of one block (K or V) and writes the block.
template <int DIM, int KIND, int TYPE, bool V>
__device__ __forceinline__ void write_half(const Task& t, const typename Element<TYPE>::type* x, long long stride, uint8_t* data,
                                           float* scale, uint8_t* rows, float* reduce) {
    constexpr int kChunks = kBlock * DIM / 8;                    // of 8 elements
    constexpr int kPer = (kChunks + kThreads - 1) / kThreads;
    constexpr int kPieces = 2 * DIM;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    float y[kPer][8];
    float amax = 0.f;
    bool nan = false;
#pragma unroll
    for (int c = 0; c < kPer; ++c) {
        const int chunk = c * kThreads + tid, m = chunk / (DIM / 8), d = chunk % (DIM / 8) * 8;
        if (m >= t.first && m < t.last && (kChunks % kThreads == 0 || chunk < kChunks)) {
            load8<TYPE>(x + (long long)(t.row + m) * stride + (long long)t.head * DIM + d, y[c]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[c][i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = fabsf(y[c][i]);
            nan |= a != a;
            amax = fmaxf(amax, a < __builtin_inff() ? a : 0.f);
        }
    }
    amax = wave_max(amax, lane);
    const bool any = __ballot(nan) != 0;
    if (lane == 0) reduce[wave] = any ? -amax : amax;            // (the sign bit, also of a zero)
    __syncthreads();
    amax = 0.f;
    nan = false;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        const float a = reduce[w];
        nan |= __float_as_uint(a) >> 31;
        amax = fmaxf(amax, fabsf(a));
    }
    float s = scale_of<KIND>(amax), s_old = 0.f;
    if (!t.fresh) {
        const float o = *scale;
        nan |= __float_as_uint(o) >> 31;
        s_old = fabsf(o);
        s = fmaxf(s, s_old);
    }
    const bool keep = !t.fresh;                                  // (uniform)
    __syncthreads();                                             // every thread has read the scale and `reduce`
    if (keep) {                                                  // the block's bytes first, as rows
        for (int p = tid; p < kPieces; p += kThreads) {
            const u32x4 b = *reinterpret_cast<const u32x4*>(data + p * 16);
            piece_to_rows<DIM, V>(rows, p, b);
        }
        __syncthreads();
    }
#pragma unroll
    for (int c = 0; c < kPer; ++c) {
        const int chunk = c * kThreads + tid, m = chunk / (DIM / 8), d = chunk % (DIM / 8) * 8;
        if (kChunks % kThreads != 0 && chunk >= kChunks) break;
        uint2* at = reinterpret_cast<uint2*>(rows + m * kRow<DIM> + d);
        if (m < t.old) {
            if (s == s_old) continue;                            // (uniform)
            const uint2 b = *at;
            decode4<KIND>(b.x, y[c]);
            decode4<KIND>(b.y, y[c] + 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[c][i] = y[c][i] * s_old;
        } else if (m >= t.last && keep) {
            continue;                                            // what is behind the new tokens stays
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[c][i] = y[c][i] / s;
        *at = make_uint2(encode4<KIND>(y[c]), encode4<KIND>(y[c] + 4));
    }
    __syncthreads();
    for (int p = tid; p < kPieces; p += kThreads) *reinterpret_cast<u32x4*>(data + p * 16) = piece_from_rows<DIM, V>(rows, p);
    if (tid == 0) *scale = nan ? -s : s;
}

template <int DIM, int KIND, int TYPE>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(Cache c, Rows r, int per, const typename Element<TYPE>::type* k,
                                                            long long k_stride, const typename Element<TYPE>::type* v,
                                                            long long v_stride) {
    __shared__ __align__(16) uint8_t rows[2][kBlock * kRow<DIM>];
    __shared__ float reduce[2][kThreads / 64];
    const Task t = task_of(c, r, per, blockIdx.x);
    if (t.at < 0) return;
    uint8_t* data = c.data + t.at * (2 * kBlock * DIM);
    float* scale = c.scales + t.at * 2;
    write_half<DIM, KIND, TYPE, false>(t, k, k_stride, data, scale, rows[0], reduce[0]);
    write_half<DIM, KIND, TYPE, true>(t, v, v_stride, data + kBlock * DIM, scale + 1, rows[1], reduce[1]);
}

template <int DIM, int KIND, int TYPE>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(Cache c, Rows r, int per, typename Element<TYPE>::type* out_k,
                                                           typename Element<TYPE>::type* out_v) {
    __shared__ __align__(16) uint8_t rows[2][kBlock * kRow<DIM>];
    const Task t = task_of(c, r, per, blockIdx.x);
    if (t.last <= t.first) return;
    constexpr int kChunks = kBlock * DIM / 8, kPieces = 2 * DIM;
    const int tid = threadIdx.x;
    float s[2] = {0.f, 0.f};
    if (t.at >= 0) {
        const uint8_t* data = c.data + t.at * (2 * kBlock * DIM);
        s[0] = fabsf(c.scales[t.at * 2]);
        s[1] = fabsf(c.scales[t.at * 2 + 1]);
        for (int p = tid; p < kPieces; p += kThreads) {
            piece_to_rows<DIM, false>(rows[0], p, *reinterpret_cast<const u32x4*>(data + p * 16));
            piece_to_rows<DIM, true>(rows[1], p, *reinterpret_cast<const u32x4*>(data + kBlock * DIM + p * 16));
        }
    }
    __syncthreads();
    for (int chunk = tid; chunk < kChunks; chunk += kThreads) {
        const int m = chunk / (DIM / 8), d = chunk % (DIM / 8) * 8;
        if (m < t.first || m >= t.last) continue;
        const long long at = ((long long)(t.row + m) * c.heads + t.head) * DIM + d;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (t.at >= 0) {                                     // (uniform)
                const uint2 b = *reinterpret_cast<const uint2*>(rows[w] + m * kRow<DIM> + d);
                decode4<KIND>(b.x, y);
                decode4<KIND>(b.y, y + 4);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = y[i] * s[w];
            }
            store8<TYPE>((w ? out_v : out_k) + at, y);
        }
    }
}

template <int DIM, int KIND, int TYPE>
hipError_t write_as(const Cache& c, const void* k, long long k_stride, const void* v, long long v_stride, const Rows& r,
                    hipStream_t stream) {
    using T = typename Element<TYPE>::type;
    const int per = touched_blocks(r.max_rows);
    kv_write_kernel<DIM, KIND, TYPE><<<dim3((unsigned)(r.S * per * c.heads)), kThreads, 0, stream>>>(
        c, r, per, static_cast<const T*>(k), k_stride, static_cast<const T*>(v), v_stride);
    return hipGetLastError();
}
template <int DIM, int KIND, int TYPE>
hipError_t read_as(const Cache& c, const Rows& r, void* out_k, void* out_v, hipStream_t stream) {
    using T = typename Element<TYPE>::type;
    const int per = touched_blocks(r.max_rows);
    kv_read_kernel<DIM, KIND, TYPE><<<dim3((unsigned)(r.S * per * c.heads)), kThreads, 0, stream>>>(
        c, r, per, static_cast<T*>(out_k), static_cast<T*>(out_v));
    return hipGetLastError();
}

// f(integral constants dim, kind, type) for run-time values that the C entry has checked
template <int I>
using Const = std::integral_constant<int, I>;
template <class F>
hipError_t with_type(int type, F f) {
    return type == EVOSPEC_BF16 ? f(Const<EVOSPEC_BF16>{}) : type == EVOSPEC_FP16 ? f(Const<EVOSPEC_FP16>{}) : f(Const<EVOSPEC_FP32>{});
}
template <class F>
hipError_t with_kind(int kind, F f) {
    return kind == EVOSPEC_KV_E4M3 ? f(Const<EVOSPEC_KV_E4M3>{}) : f(Const<EVOSPEC_KV_INT8>{});
}
template <class F>
hipError_t with_dim(int dim, F f) {
    switch (dim) {
        case 64: return f(Const<64>{});
        case 96: return f(Const<96>{});
        case 128: return f(Const<128>{});
        case 192: return f(Const<192>{});
        default: return f(Const<256>{});
    }
}

}  // namespace

hipError_t launch_kv_write(const Cache& c, int dim, int kind, const void* k, long long k_stride, const void* v, long long v_stride,
                           int type, const Rows& r, hipStream_t stream) {
    return with_dim(dim, [&](auto d) {
        return with_kind(kind, [&](auto kd) {
            return with_type(type, [&](auto ty) {
                return write_as<d.value, kd.value, ty.value>(c, k, k_stride, v, v_stride, r, stream);
            });
        });
    });
}

hipError_t launch_kv_read(const Cache& c, int dim, int kind, const Rows& r, int type, void* out_k, void* out_v, hipStream_t stream) {
    return with_dim(dim, [&](auto d) {
        return with_kind(kind, [&](auto kd) {
            return with_type(type, [&](auto ty) { return read_as<d.value, kd.value, ty.value>(c, r, out_k, out_v, stream); });
        });
    });
}

}  // namespace evospec
