// The 8-bit key/value cache: new tokens are quantised as they are written, and read back as values.
//
// x is kept as code = round(x / s) of 8 bits, s the scale of a block (32 tokens of one head, K and V apart).  For e4m3, s is
// a power of two, so that a block whose scale grows loses nothing but what falls below the smallest code; int8 codes are
// rounded again.  One workgroup of 4 wavefronts owns a (block, head): its largest magnitude needs all of the block's new
// elements, which stay in registers between the maximum and the rounding (one pass over the input).  Both ways go
// through LDS: global memory sees rows of `dim` elements on the caller's side, and 16-byte pieces in the order of the
// matrix cores' operands (evospec_decode.h) on the cache's.  Measured: 12,000 tokens of 8 x 128 elements written in 24 us (74 MB, 3.1
// TB/s), 49,000 read back in 65 us (5.2 TB/s, a copy's rate).
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
    return t;
}
// A task's place: (page * heads + head) blocks in, -1 if it has none.
__device__ __forceinline__ long long place_of(const Cache& c, const Rows& r, const Task& t) {
    if ((t.block >> c.shift) >= r.width) return -1;
    const int page = r.table[(long long)t.s * r.width + (t.block >> c.shift)];
    if ((unsigned)page >= (unsigned)c.pages) return -1;
    return (((long long)page * c.heads + t.head) << c.shift) + (t.block & ((1 << c.shift) - 1));
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

// 8 elements of a row as they come, and as floats
template <int TYPE>
struct Raw {
    u32x4 a, b;                                                  // (b: fp32 only)
    __device__ __forceinline__ void load(const typename Element<TYPE>::type* p) {
        a = reinterpret_cast<const u32x4*>(p)[0];
        if constexpr (TYPE == EVOSPEC_FP32) b = reinterpret_cast<const u32x4*>(p)[1];
    }
    __device__ __forceinline__ void clear() { a = b = u32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ float at(int i) const {
        if constexpr (TYPE == EVOSPEC_FP32) return __uint_as_float(i < 4 ? a[i] : b[i - 4]);
        else if constexpr (TYPE == EVOSPEC_BF16) return __uint_as_float(i & 1 ? a[i >> 1] & 0xffff0000u : a[i >> 1] << 16);
        else return (float)__builtin_bit_cast(_Float16, (uint16_t)(a[i >> 1] >> (16 * (i & 1))));
    }
    // the largest magnitude so far as bits, whose order is that of the magnitudes; 16-bit types two at a time
    __device__ __forceinline__ u32x4 larger(u32x4 m) const {
        typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
        if constexpr (TYPE == EVOSPEC_FP32)
            return __builtin_elementwise_max(m, __builtin_elementwise_max(a & 0x7fffffffu, b & 0x7fffffffu));
        else
            return __builtin_bit_cast(u32x4, __builtin_elementwise_max(__builtin_bit_cast(u16x8, m), __builtin_bit_cast(u16x8, a & 0x7fff7fffu)));
    }
};
// of four words of such bits, as a float (infinity and NaN as they are)
template <int TYPE>
__device__ __forceinline__ float magnitude(u32x4 m) {
    uint32_t x = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (TYPE == EVOSPEC_FP32) x = max(x, m[i]);
        else x = max(x, max(m[i] & 0xffffu, m[i] >> 16));
    }
    if constexpr (TYPE == EVOSPEC_FP32) return __uint_as_float(x);
    else if constexpr (TYPE == EVOSPEC_BF16) return __uint_as_float(x << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)x);
}

// Codes of 8 values that are finite and no larger than the largest code times s.  e4m3's s is a power of two, whose reciprocal is
// exact; int8 multiplies too, and divides only where the quotient lies so near to the middle between two codes that the
// product may be on the other side of it.  x / s + 1.5 * 2^23 has the rounded quotient in its low bits.
template <int KIND, int TYPE>
__device__ __forceinline__ uint2 encode_plain(const Raw<TYPE>& x, float s, float inv) {
    uint32_t out[2];
    if constexpr (KIND == EVOSPEC_KV_E4M3) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int p = __builtin_amdgcn_cvt_pk_fp8_f32(x.at(4 * j) * inv, x.at(4 * j + 1) * inv, 0, false);
            out[j] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x.at(4 * j + 2) * inv, x.at(4 * j + 3) * inv, p, true);
        }
    } else {
        constexpr float kMagic = 12582912.f;
        uint32_t f[8];
        float far = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = x.at(i), y = fmaf(v, inv, kMagic);
            far = fmaxf(far, fabsf(fmaf(v, inv, kMagic - y)));
            f[i] = __float_as_uint(y);
        }
        if (far > 0.5f - 0x1p-12f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = __float_as_uint(x.at(i) / s + kMagic);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
            out[j] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(f[4 * j + 3], f[4 * j + 2], 0x0c0c0400u),
                                           __builtin_amdgcn_perm(f[4 * j + 1], f[4 * j], 0x0c0c0400u), 0x05040100u);
    }
    return make_uint2(out[0], out[1]);
}
// Codes of any 8 values.
template <int KIND>
__device__ __forceinline__ uint2 encode_any(float* y, float s) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = y[i] / s;
    return make_uint2(encode4<KIND>(y), encode4<KIND>(y + 4));
}

// Quantises the new tokens of one block, K and V side by side, and writes the block.  What is rare (a NaN, an infinity, older codes
// that have to be scaled) has code of its own: with it in the way of all, 64 elements of a thread took 1,600 instructions, and
// 12,000 tokens of 8 heads 28 us.
template <int DIM, int KIND, int TYPE>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(Cache c, Rows r, int per, const typename Element<TYPE>::type* k,
                                                            long long k_stride, const typename Element<TYPE>::type* v,
                                                            long long v_stride) {
    __shared__ __align__(16) uint8_t rows[2][kBlock * kRow<DIM>];
    __shared__ float reduce[2][2][kThreads / 64];
    constexpr int kChunks = kBlock * DIM / 8;                    // of 8 elements
    constexpr int kPer = (kChunks + kThreads - 1) / kThreads;
    constexpr int kPieces = 2 * DIM;
    const Task t = task_of(c, r, per, blockIdx.x);
    if (t.last <= t.first) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Raw<TYPE> x[2][kPer];
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int p = 0; p < kPer; ++p) {
            const int chunk = p * kThreads + tid, m = chunk / (DIM / 8), d = chunk % (DIM / 8) * 8;
            if (m >= t.first && m < t.last && (kChunks % kThreads == 0 || chunk < kChunks))
                x[w][p].load((w ? v : k) + (long long)(t.row + m) * (w ? v_stride : k_stride) + (long long)t.head * DIM + d);
            else
                x[w][p].clear();
        }
    const long long place = place_of(c, r, t);                   // (while the new tokens are under way)
    if (place < 0) return;
    uint8_t* data = c.data + place * (2 * kBlock * DIM);
    float* scale = c.scales + place * 2;
    const bool keep = !t.fresh;                                  // (uniform)
    float old[2] = {0.f, 0.f};
    if (keep) {                                                  // the block's bytes first, as rows
        for (int p = tid; p < kPieces; p += kThreads) {
            piece_to_rows<DIM, false>(rows[0], p, *reinterpret_cast<const u32x4*>(data + p * 16));
            piece_to_rows<DIM, true>(rows[1], p, *reinterpret_cast<const u32x4*>(data + kBlock * DIM + p * 16));
        }
        old[0] = scale[0];
        old[1] = scale[1];
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        u32x4 m = {0, 0, 0, 0};
#pragma unroll
        for (int p = 0; p < kPer; ++p) m = x[w][p].larger(m);
        // (as numbers of bits: a NaN is larger than all)
        uint32_t top = __float_as_uint(magnitude<TYPE>(m));
        top = max(top, xor_lane<1>(top, lane));
        top = max(top, xor_lane<2>(top, lane));
        top = max(top, xor_lane<4>(top, lane));
        top = max(top, xor_lane<8>(top, lane));
        top = max(top, xor_lane<16>(top, lane));
        top = max(top, xor_lane<32>(top, lane));
        if (lane == 0) reduce[0][w][wave] = __uint_as_float(top);
    }
    __syncthreads();
    float final[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        uint32_t bits = 0;
#pragma unroll
        for (int i = 0; i < kThreads / 64; ++i) bits = max(bits, __float_as_uint(reduce[0][w][i]));
        float amax = __uint_as_float(bits);
        bool nan = __float_as_uint(old[w]) >> 31;
        const bool special = bits >= 0x7f800000u;                // (uniform) a NaN or an infinity: the largest of the others
        if (special) {
            amax = 0.f;
            bool mine = false;
#pragma unroll
            for (int p = 0; p < kPer; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float a = fabsf(x[w][p].at(i));
                    mine |= a != a;
                    amax = fmaxf(amax, a < __builtin_inff() ? a : 0.f);
                }
            amax = wave_max(amax, lane);
            mine = __ballot(mine) != 0;
            if (lane == 0) reduce[1][w][wave] = mine ? -amax : amax;         // (the sign bit, also of a zero)
            __syncthreads();
            amax = 0.f;
#pragma unroll
            for (int i = 0; i < kThreads / 64; ++i) {
                const float a = reduce[1][w][i];
                nan |= __float_as_uint(a) >> 31;
                amax = fmaxf(amax, fabsf(a));
            }
        }
        const float s_old = fabsf(old[w]), s = fmaxf(scale_of<KIND>(amax), s_old);
        const bool plain = !special && (KIND == EVOSPEC_KV_INT8 || amax <= 448.f * s);
        const float inv = 1.f / s;
        final[w] = nan ? -s : s;
#pragma unroll
        for (int p = 0; p < kPer; ++p) {
            const int chunk = p * kThreads + tid, m = chunk / (DIM / 8), d = chunk % (DIM / 8) * 8;
            if (kChunks % kThreads != 0 && chunk >= kChunks) break;
            uint2* at = reinterpret_cast<uint2*>(rows[w] + m * kRow<DIM> + d);
            float y[8];
            if (m < t.old) {
                if (s == s_old) continue;                        // (uniform)
                const uint2 b = *at;
                decode4<KIND>(b.x, y);
                decode4<KIND>(b.y, y + 4);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = y[i] * s_old;
                *at = encode_any<KIND>(y, s);
            } else if (m < t.last || !keep) {                    // (what is behind the new tokens of an older block stays)
                if (plain) {
                    *at = encode_plain<KIND, TYPE>(x[w][p], s, inv);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = x[w][p].at(i);
                    *at = encode_any<KIND>(y, s);
                }
            }
        }
    }
    __syncthreads();
    for (int p = tid; p < kPieces; p += kThreads) {
        *reinterpret_cast<u32x4*>(data + p * 16) = piece_from_rows<DIM, false>(rows[0], p);
        *reinterpret_cast<u32x4*>(data + kBlock * DIM + p * 16) = piece_from_rows<DIM, true>(rows[1], p);
    }
    if (tid < 2) scale[tid] = final[tid];
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
    const long long place = place_of(c, r, t);
    if (place >= 0) {
        const uint8_t* data = c.data + place * (2 * kBlock * DIM);
        s[0] = fabsf(c.scales[place * 2]);
        s[1] = fabsf(c.scales[place * 2 + 1]);
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
            if (place >= 0) {                                    // (uniform)
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
