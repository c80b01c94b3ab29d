// Low-rank adapters of many requests beside a shared projection: y += s (x A^T) B^T, and the gradients.
//
// Three kinds of product, all on v_mfma_f32_16x16x32_bf16 with tiles of the rows of one request:
//   down   h[rank][row] = sum_k w[rank][k] x[row][k]      (x A^T; dy B)
//   up     y[row][c] += sum_rank h[rank][row] w[rank][c]   (h B^T; g A)
//   grads  out[rank][c] = sum_row h[rank][row] x[row][c]   (dA, dB)
// An operand's lane holds 8 numbers along the axis that is summed over.  Where memory has the other axis contiguous (B in dy B, A in
// g A, the rows' elements in the gradients), a lane takes 2, 4 or 8 bytes of 8 neighbours along the summed axis and puts halves of
// dwords together (one v_perm_b32 for two numbers): its 1, 2 or 4 columns belong to as many tiles, so that column RT m + j is
// row m of tile j.  No LDS, and whole lines of memory.
// h stays in fp32 between the kernels.  As an operand it is a sum of bf16 numbers, two (2^-16 of it) where the result is rounded to bf16,
// three (all 24 bits) where the result is fp32.
#include <hip/hip_runtime.h>

#include "adapt.hpp"
#include "common.hpp"

namespace evospec {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
typedef const uint16_t __attribute__((address_space(1))) * gu16;

__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// halves of two dwords as one: those of `lo` go low
__device__ __forceinline__ uint32_t low_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }

// The next 8 bits of each number's mantissa, cut off (not rounded): N parts of 8 bits are the first 8 N bits, exactly.
__device__ __forceinline__ u32x4 next_part(float (&x)[8]) {
    u32x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        out[i] = high_halves(__float_as_uint(x[2 * i]), __float_as_uint(x[2 * i + 1]));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            // (what is left of an infinity or a NaN is nothing, and not NaN or 0 x infinity)
            const uint32_t top = __float_as_uint(x[2 * i + j]) & 0xffff0000u;
            x[2 * i + j] = (top & 0x7f800000u) == 0x7f800000u ? 0.f : x[2 * i + j] - __uint_as_float(top);
        }
    }
    return out;
}

struct Tile {
    int row0, rows, adapter;
};
struct Request {
    int row0, rows, adapter;
};
__device__ __forceinline__ Request request_of(const Requests& q, int s) {
    Request t{0, 0, -1};
    if (s < q.S) {
        t.row0 = min(max(q.row_off[s], 0), q.T);
        t.rows = min(max(q.row_off[s + 1], t.row0), q.T) - t.row0;
        t.adapter = q.adapter[s];
        if ((unsigned)t.adapter >= (unsigned)q.n) t.rows = 0;
    }
    return t;
}
// Tile `index` of the requests that have an adapter, in their order; no rows if there are fewer.  64 requests at a time.
__device__ __forceinline__ Tile find_tile(const Requests& q, int shift, int index) {
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < q.S; base += 64) {
        const Request t = request_of(q, base + lane);
        const int tiles = (t.rows + (1 << shift) - 1) >> shift;
        int incl = tiles;
        if (q.S > 1) {
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int up = __shfl_up(incl, o);
                if (lane >= o) incl += up;
            }
        }
        const int total = __builtin_amdgcn_readlane(incl, q.S > 1 ? 63 : 0);
        if (index < total) {
            const int at = __ffsll((unsigned long long)__ballot(incl > index)) - 1;
            const int first = (index - __builtin_amdgcn_readlane(incl, at) + __builtin_amdgcn_readlane(tiles, at)) << shift;
            return Tile{__builtin_amdgcn_readlane(t.row0, at) + first, min(__builtin_amdgcn_readlane(t.rows, at) - first, 1 << shift),
                        __builtin_amdgcn_readlane(t.adapter, at)};
        }
        index -= total;
    }
    return Tile{0, 0, 0};
}

// ---------------------------------------------------------------- down

// RT tiles of 16 ranks, NT tiles of 16 rows; the part of d is split over the wavefronts, whose sums are added in LDS.
template <int RT, int NT, bool RANK_LAST>
__global__ __launch_bounds__(kThreads) void lora_down_kernel(DownArgs a, int splits) {
    __shared__ __align__(16) f32x4 sums[kWaves][RT * NT][64];
    const Tile t = find_tile(a.q, a.shift, blockIdx.x);
    if (t.rows == 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, kg = lane >> 4;
    const int steps = (a.d + 31) / 32, parts = splits * kWaves, part = blockIdx.y * kWaves + wave;
    const int s0 = (int)((long long)steps * part / parts), s1 = (int)((long long)steps * (part + 1) / parts);
    gu16 x[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
        x[i] = (gu16)a.x + (long long)(t.row0 + min(16 * i + m, t.rows - 1)) * a.x_stride + 8 * kg;
    const gu16 w = (gu16)a.w + (long long)t.adapter * a.r * a.d;
    f32x4 acc[RT][NT] = {};
    auto load_x = [&](int step, u32x4 (&xs)[NT]) {
        const bool in = step * 32 + 8 * kg < a.d;                // (d ends within a step: zeros on both sides)
#pragma unroll
        for (int i = 0; i < NT; ++i) xs[i] = in ? *(gvec_ptr)(x[i] + (long long)step * 32) : u32x4{0, 0, 0, 0};
    };
    auto load_w = [&](int step, u32x4 (&ws)[RT]) {
        const int k = step * 32 + 8 * kg;
        const bool in = k < a.d;
        if constexpr (!RANK_LAST) {
#pragma unroll
            for (int j = 0; j < RT; ++j)                         // (ranks from r on: any, nobody stores them)
                ws[j] = in ? *(gvec_ptr)(w + (long long)min(16 * j + m, a.r - 1) * a.d + k) : u32x4{0, 0, 0, 0};
        } else {
            const int rank = RT * m < a.r ? RT * m : 0;
            uint32_t raw[8][(RT + 1) / 2];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const gu16 p = w + (long long)(in ? k + i : 0) * a.r + rank;
                if constexpr (RT == 1) raw[i][0] = *p;
                else if constexpr (RT == 2) raw[i][0] = *(const uint32_t __attribute__((address_space(1)))*)p;
                else {
                    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
                    const u32x2 v = *(const u32x2 __attribute__((address_space(1)))*)p;
                    raw[i][0] = v[0];
                    raw[i][1] = v[1];
                }
            }
#pragma unroll
            for (int j = 0; j < RT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t v = j & 1 ? high_halves(raw[2 * i][j / 2], raw[2 * i + 1][j / 2]) : low_halves(raw[2 * i][j / 2], raw[2 * i + 1][j / 2]);
                    ws[j][i] = in ? v : 0u;
                }
        }
    };
    constexpr int U = 4;
    u32x4 xs[U][NT], ws[U][RT];
    for (int s = s0; s < s1; s += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            load_x(s + u < s1 ? s + u : steps, xs[u]);
            load_w(s + u < s1 ? s + u : steps, ws[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < RT; ++j)
#pragma unroll
                for (int i = 0; i < NT; ++i) acc[j][i] = mfma(ws[u][j], xs[u][i], acc[j][i]);
    }
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
        for (int i = 0; i < NT; ++i) sums[wave][j * NT + i][lane] = acc[j][i];
    __syncthreads();
    const float factor = a.factor ? a.factor[t.adapter] : 1.f;
    float* out = a.out + (long long)blockIdx.y * a.r * a.q.T;
    for (int e = wave; e < RT * NT; e += kWaves) {
        f32x4 v = sums[0][e][lane];
#pragma unroll
        for (int w4 = 1; w4 < kWaves; ++w4) v += sums[w4][e][lane];
        const int j = e / NT, row = 16 * (e % NT) + m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int rank = RANK_LAST ? RT * (4 * kg + i) + j : 16 * j + 4 * kg + i;
            if (rank < a.r && row < t.rows) out[(long long)rank * a.q.T + t.row0 + row] = v[i] * factor;
        }
    }
}

// ---------------------------------------------------------------- up

// KS steps of 32 ranks, NT tiles of 16 rows.  A wavefront takes 64 columns at a time, of which a lane holds 16 in a row of the output.
template <int KS, int NT, bool RANK_LAST>
__global__ __launch_bounds__(kThreads) void lora_up_kernel(UpArgs a, int slices) {
    const Tile t = find_tile(a.q, a.shift, blockIdx.x);
    if (t.rows == 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, kg = lane >> 4;
    const float factor = a.factor ? a.factor[t.adapter] : 1.f;
    const bool keep = a.out_h && blockIdx.y == 0 && wave == 0;
    u32x4 h[NT][KS][2];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            float v[8];
            const long long row = t.row0 + 16 * i + m;
            const bool in = 16 * i + m < t.rows && 32 * s + 8 * kg < a.r;
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 0.f;
            if (in)
                for (int p = 0; p < a.splits; ++p)
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] += a.h[((long long)p * a.r + 32 * s + 8 * kg + k) * a.q.T + row];
            if (in && keep)
#pragma unroll
                for (int k = 0; k < 8; ++k) a.out_h[(long long)(32 * s + 8 * kg + k) * a.q.T + row] = v[k];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= factor;
            h[i][s][0] = next_part(v);
            h[i][s][1] = next_part(v);
        }
    const gu16 w = (gu16)a.w + (long long)t.adapter * a.r * a.d;
    const int groups = (a.d + 63) / 64, parts = slices * kWaves, part = blockIdx.y * kWaves + wave;
    const int g0 = (int)((long long)groups * part / parts), g1 = (int)((long long)groups * (part + 1) / parts);
    for (int g = g0; g < g1; ++g) {
        const int c0 = 64 * g, mine = c0 + 16 * kg;              // this lane's 16 columns of the output
        u32x4 y[NT][2];
        uint16_t* at[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            at[i] = (uint16_t*)a.y + (long long)(t.row0 + min(16 * i + m, t.rows - 1)) * a.y_stride + mine;
#pragma unroll
            for (int b = 0; b < 2; ++b)
                if (mine + 8 * b < a.d) y[i][b] = *(gvec_ptr)(at[i] + 8 * b);
        }
        f32x4 acc[4][NT] = {};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            u32x4 op[4];
            const int k0 = 32 * s + 8 * kg;
            if constexpr (!RANK_LAST) {                          // w [r][d]
                typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
                u32x2 raw[8];
                const int c = c0 + 4 * m < a.d ? c0 + 4 * m : 0;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    raw[k] = k0 < a.r ? *(const u32x2 __attribute__((address_space(1)))*)(w + (long long)(k0 + k) * a.d + c) : u32x2{0, 0};
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        op[j][k] = j & 1 ? high_halves(raw[2 * k][j / 2], raw[2 * k + 1][j / 2]) : low_halves(raw[2 * k][j / 2], raw[2 * k + 1][j / 2]);
            } else {                                             // w [d][r]
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = c0 + 16 * (m >> 2) + 4 * j + (m & 3);
                    op[j] = k0 < a.r ? *(gvec_ptr)(w + (long long)min(c, a.d - 1) * a.r + k0) : u32x4{0, 0, 0, 0};
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    acc[j][i] = mfma(op[j], h[i][s][0], acc[j][i]);
                    acc[j][i] = mfma(op[j], h[i][s][1], acc[j][i]);
                }
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (16 * i + m >= t.rows || mine + 8 * b >= a.d) continue;
                u32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t old = y[i][b][e];
                    float z[2];
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        const int c = 8 * b + 2 * e + f;         // of the lane's 16: rows 4 kg .. of the tiles
                        const float up = RANK_LAST ? acc[c / 4][i][c % 4] : acc[c % 4][i][c / 4];
                        z[f] = __uint_as_float(f ? old & 0xffff0000u : old << 16) + up;
                    }
                    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                    v[e] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)z[0], (__bf16)z[1]});
                }
                *reinterpret_cast<u32x4*>(at[i] + 8 * b) = v;
            }
    }
}

// ---------------------------------------------------------------- gradients

// The steps of 32 rows of an adapter, request by request.  Everything is the same in all lanes but the 64 requests at hand.
struct Steps {
    const Requests& q;
    const int adapter;
    int base = -64, at = -1, row = 0, left = 0;
    unsigned long long rest = 0;
    Request mine{};
    __device__ Steps(const Requests& q_, int adapter_) : q(q_), adapter(adapter_) {}
    // false: there is no further one
    __device__ __forceinline__ bool next(int& row0, int& rows) {
        while (left <= 0) {
            while (rest == 0) {
                base += 64;
                if (base >= q.S) return false;
                mine = request_of(q, base + (int)(threadIdx.x & 63));
                rest = __ballot(mine.rows > 0 && mine.adapter == adapter);
            }
            at = __ffsll(rest) - 1;
            rest &= rest - 1;
            row = __builtin_amdgcn_readlane(mine.row0, at);
            left = __builtin_amdgcn_readlane(mine.rows, at);
        }
        row0 = row;
        rows = min(left, 32);
        row += 32;
        left -= 32;
        return true;
    }
};

// RT tiles of 16 ranks; a workgroup has 64 columns of one adapter, its wavefronts and `parts` workgroups every so many-th step.
template <int RT>
__global__ __launch_bounds__(kThreads) void lora_grads_kernel(GradArgs a, int groups0, long long partial_stride) {
    __shared__ __align__(16) f32x4 sums[kWaves][4 * RT][64];
    const bool second = (int)blockIdx.x >= groups0;
    const GradJob job = second ? a.job[1] : a.job[0];
    const int c0 = 64 * (blockIdx.x - (second ? groups0 : 0)), adapter = blockIdx.y, part = blockIdx.z;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, kg = lane >> 4;
    const float factor = job.factor ? job.factor[adapter] : 1.f;
    const gu16 x = (gu16)job.x + (c0 + 4 * m < job.d ? c0 + 4 * m : 0);
    f32x4 acc[4][RT] = {};
    Steps steps(a.q, adapter);
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    int row0, rows;
    for (int n = 0; steps.next(row0, rows); ++n) {
        if (n % (kWaves * a.parts) != part * kWaves + wave) continue;
        u32x2 raw[8];
        float h[RT][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool in = 8 * kg + i < rows;
            raw[i] = *(const u32x2 __attribute__((address_space(1)))*)(x + (long long)(row0 + min(8 * kg + i, rows - 1)) * job.x_stride);
            if (!in) raw[i] = u32x2{0, 0};
#pragma unroll
            for (int j = 0; j < RT; ++j) {
                h[j][i] = 0.f;
                if (in && 16 * j + m < a.r)
                    for (int p = 0; p < job.splits; ++p) h[j][i] += job.h[((long long)p * a.r + 16 * j + m) * a.q.T + row0 + 8 * kg + i];
                h[j][i] *= factor;
            }
        }
        u32x4 op[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                op[j][k] = j & 1 ? high_halves(raw[2 * k][j / 2], raw[2 * k + 1][j / 2]) : low_halves(raw[2 * k][j / 2], raw[2 * k + 1][j / 2]);
#pragma unroll
        for (int part3 = 0; part3 < 3; ++part3)
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const u32x4 hs = next_part(h[r]);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j][r] = mfma(op[j], hs, acc[j][r]);
            }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int r = 0; r < RT; ++r) sums[wave][j * RT + r][lane] = acc[j][r];
    __syncthreads();
    float* out = a.parts > 1 ? a.partial + part * partial_stride + (second ? (long long)a.q.n * a.r * a.job[0].d : 0ll) : job.out;
    out += (long long)adapter * a.r * job.d;
    for (int e = wave; e < 4 * RT; e += kWaves) {
        f32x4 v = sums[0][e][lane];
#pragma unroll
        for (int w4 = 1; w4 < kWaves; ++w4) v += sums[w4][e][lane];
        const int j = e / RT, rank = 16 * (e % RT) + m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = c0 + 4 * (4 * kg + i) + j;
            if (rank < a.r && c < job.d) out[job.rank_last ? (long long)c * a.r + rank : (long long)rank * job.d + c] = v[i];
        }
    }
}

__global__ __launch_bounds__(kThreads) void lora_grads_sum_kernel(const float4* partial, int parts, long long count0, long long count1,
                                                                  float4* out0, float4* out1) {
    const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (i >= count0 + count1) return;
    float4 s = partial[i];
    for (int p = 1; p < parts; ++p) {
        const float4 v = partial[p * (count0 + count1) + i];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    if (i < count0) out0[i] = s;
    else out1[i - count0] = s;
}

template <int RT, int NT>
hipError_t down_as(const DownArgs& a, const LoraPlan& p, bool rank_last, hipStream_t stream) {
    const dim3 grid((unsigned)p.tiles, (unsigned)p.down_splits);
    if (rank_last) lora_down_kernel<RT, NT, true><<<grid, kThreads, 0, stream>>>(a, p.down_splits);
    else lora_down_kernel<RT, NT, false><<<grid, kThreads, 0, stream>>>(a, p.down_splits);
    return hipGetLastError();
}
template <int KS, int NT>
hipError_t up_as(const UpArgs& a, const LoraPlan& p, bool rank_last, hipStream_t stream) {
    const dim3 grid((unsigned)p.tiles, (unsigned)p.up_slices);
    if (rank_last) lora_up_kernel<KS, NT, true><<<grid, kThreads, 0, stream>>>(a, p.up_slices);
    else lora_up_kernel<KS, NT, false><<<grid, kThreads, 0, stream>>>(a, p.up_slices);
    return hipGetLastError();
}

}  // namespace

LoraPlan lora_plan(int S, int T, int d_down, int d_up) {
    LoraPlan p{};
    p.shift = T > 16 * S ? 5 : 4;
    p.tiles = ((T + (1 << p.shift) - 1) >> p.shift) + S;
    const int whole = p.tiles - S > S ? p.tiles - S : S;         // about as many have rows
    const int down = (d_down + 255) / 256, up = (d_up + 255) / 256;       // parts that leave a wavefront two steps of 32, a group of 64
    p.down_splits = 512 / whole < 1 ? 1 : 512 / whole < 16 ? 512 / whole : 16;
    if (p.down_splits > down) p.down_splits = down;
    p.up_slices = 1024 / whole < 1 ? 1 : 1024 / whole < up ? 1024 / whole : up;
    return p;
}

hipError_t launch_lora_down(const DownArgs& a, const LoraPlan& p, bool rank_last, hipStream_t stream) {
    const int rt = a.r <= 16 ? 1 : a.r <= 32 ? 2 : 4;
    if (p.shift == 4) return rt == 1 ? down_as<1, 1>(a, p, rank_last, stream) : rt == 2 ? down_as<2, 1>(a, p, rank_last, stream) : down_as<4, 1>(a, p, rank_last, stream);
    return rt == 1 ? down_as<1, 2>(a, p, rank_last, stream) : rt == 2 ? down_as<2, 2>(a, p, rank_last, stream) : down_as<4, 2>(a, p, rank_last, stream);
}

hipError_t launch_lora_up(const UpArgs& a, const LoraPlan& p, bool rank_last, hipStream_t stream) {
    if (p.shift == 4) return a.r <= 32 ? up_as<1, 1>(a, p, rank_last, stream) : up_as<2, 1>(a, p, rank_last, stream);
    return a.r <= 32 ? up_as<1, 2>(a, p, rank_last, stream) : up_as<2, 2>(a, p, rank_last, stream);
}

int lora_grad_parts(int n, int T, int d0, int d1) {
    const long long groups = (long long)n * ((d0 + 63) / 64 + (d1 + 63) / 64);
    const int steps = (T + 31) / 32;
    int parts = (int)(1024 / groups);
    if (parts > (steps + 2 * kWaves - 1) / (2 * kWaves)) parts = (steps + 2 * kWaves - 1) / (2 * kWaves);
    return parts < 1 ? 1 : parts > 16 ? 16 : parts;
}

hipError_t launch_lora_grads(const GradArgs& a, hipStream_t stream) {
    const int groups0 = (a.job[0].d + 63) / 64, groups1 = (a.job[1].d + 63) / 64;
    const long long count0 = (long long)a.q.n * a.r * a.job[0].d, count1 = (long long)a.q.n * a.r * a.job[1].d;
    const dim3 grid((unsigned)(groups0 + groups1), (unsigned)a.q.n, (unsigned)a.parts);
    if (a.r <= 16) lora_grads_kernel<1><<<grid, kThreads, 0, stream>>>(a, groups0, count0 + count1);
    else if (a.r <= 32) lora_grads_kernel<2><<<grid, kThreads, 0, stream>>>(a, groups0, count0 + count1);
    else lora_grads_kernel<4><<<grid, kThreads, 0, stream>>>(a, groups0, count0 + count1);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.parts == 1) return e;
    lora_grads_sum_kernel<<<dim3((unsigned)(((count0 + count1) / 4 + kThreads - 1) / kThreads)), kThreads, 0, stream>>>(
        reinterpret_cast<const float4*>(a.partial), a.parts, count0 / 4, count1 / 4, reinterpret_cast<float4*>(a.job[0].out), reinterpret_cast<float4*>(a.job[1].out));
    return hipGetLastError();
}

}  // namespace evospec
