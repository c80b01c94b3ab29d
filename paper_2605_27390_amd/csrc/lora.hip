// Low-rank adapters of many requests beside a shared projection: y += s (x A^T) B^T, and the gradients.
//
// Three kinds of product, all on v_mfma_f32_16x16x32_bf16 with tiles of the rows of one request:
//   h[rank][row] = sum_k w[rank][k] x[row][k]             (x A^T; dy B)
//   y[row][c] += sum_rank h[rank][row] w[rank][c]         (h B^T; g A), in the same kernel
//   out[rank][c] = sum_row h[rank][row] x[row][c]         (dA, dB)
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

// Operands of four tiles from 4 columns of 8 neighbours along the summed axis: column 4 m + j is row m of tile j.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void columns_of(const u32x2 (&raw)[8], u32x4 (&op)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            op[j][k] = j & 1 ? high_halves(raw[2 * k][j / 2], raw[2 * k + 1][j / 2]) : low_halves(raw[2 * k][j / 2], raw[2 * k + 1][j / 2]);
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

// ---------------------------------------------------------------- rows

typedef const u32x2 __attribute__((address_space(1))) * gpair;
typedef const uint32_t __attribute__((address_space(1))) * gword;

// One tile of 16 NT rows: h = x W_down^T, then y += h W_up for a slice of the columns.  Forward, W_down = A [r][d] and W_up = B [d][r]; backward
// W_down = B^T and W_up = A^T of the same arrays.  The long axis of the first product is split over W wavefronts, whose sums are added
// in LDS; in the second each takes 64 columns at a time, of which a lane holds 16 in a row of y.  Every slice computes h again: it is
// launched with slices where tiles are few and the time is that of a launch.
template <int RT, int NT, bool BACK, int W>
__global__ __launch_bounds__(64 * W) void lora_rows_kernel(LoraArgs a) {
    constexpr int KS = (RT + 1) / 2, kRows = 16 * NT;
    __shared__ __align__(16) f32x4 sums[W][RT * NT][64];
    __shared__ float hs[16 * RT][kRows + 1];
    const Tile t = find_tile(a.q, NT == 1 ? 4 : NT == 2 ? 5 : 6, blockIdx.x);
    if (t.rows == 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, kg = lane >> 4;
    const float factor = a.factor ? a.factor[t.adapter] : 1.f;
    // 64 columns of the second product: y's, and of the weights what this lane's operands are made of.  Columns 32 b + 8 kg + e of a
    // row of y are a lane's: row 4 kg + i of tile j is number 4 j + i (forward) or 4 i + j of them, 8 b + e.
    struct Columns {
        u32x4 y[NT][2];
        u32x4 w[BACK ? 1 : KS][4];
        u32x2 raw[BACK ? KS : 1][8];
    };
    const gu16 w_up = (gu16)a.w_up + (long long)t.adapter * a.r * a.d_up;
    auto load_columns = [&](Columns& col, int g) {
        const int c0 = 64 * g;
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int c = c0 + 32 * b + 8 * kg;
                col.y[i][b] = *(gvec_ptr)((gu16)a.y + (long long)(t.row0 + min(16 * i + m, t.rows - 1)) * a.y_stride + min(c, a.d_up - 8));
            }
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int k0 = 32 * s + 8 * kg;
            if constexpr (BACK) {                                // [r][d]
                const int c = min(c0 + 32 * ((m >> 1) & 1) + 8 * (m >> 2) + 4 * (m & 1), a.d_up - 4);
#pragma unroll
                for (int k = 0; k < 8; ++k) col.raw[s][k] = k0 < a.r ? *(gpair)(w_up + (long long)(k0 + k) * a.d_up + c) : u32x2{0, 0};
            } else {                                             // [d][r]
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = min(c0 + 32 * (j >> 1) + 8 * (m >> 2) + 4 * (j & 1) + (m & 3), a.d_up - 1);
                    col.w[s][j] = k0 < a.r ? *(gvec_ptr)(w_up + (long long)c * a.r + k0) : u32x4{0, 0, 0, 0};
                }
            }
        }
    };
    const int groups = (a.d_up + 63) / 64, parts = gridDim.y * W, part = blockIdx.y * W + wave;
    const int n0 = (int)((long long)groups * part / parts), n1 = a.y ? (int)((long long)groups * (part + 1) / parts) : 0;
    // (as the first product's: every tile begins at another place)
    auto group_of = [&](int n) {
        const int len = n1 - n0, at = n - n0 + (int)(blockIdx.x % (unsigned)len);
        return n0 + (at < len ? at : at - len);
    };
    Columns first;
    if (NT == 1 && n0 < n1) load_columns(first, group_of(n0));
    {
        const int steps = (a.d_down + 31) / 32;
        gu16 x[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) x[i] = (gu16)a.x + (long long)(t.row0 + min(16 * i + m, t.rows - 1)) * a.x_stride + 8 * kg;
        const gu16 w = (gu16)a.w_down + (long long)t.adapter * a.r * a.d_down;
        f32x4 acc[RT][NT] = {};
        auto load_x = [&](int step, u32x4 (&xs)[NT]) {
            const bool in = step * 32 + 8 * kg < a.d_down;       // (d ends within a step: zeros on both sides)
#pragma unroll
            for (int i = 0; i < NT; ++i) xs[i] = in ? *(gvec_ptr)(x[i] + (long long)step * 32) : u32x4{0, 0, 0, 0};
        };
        auto load_w = [&](int step, u32x4 (&ws)[RT]) {
            const int k = step * 32 + 8 * kg;
            const bool in = k < a.d_down;
            if constexpr (!BACK) {
#pragma unroll
                for (int j = 0; j < RT; ++j)                     // (ranks from r on: any, they end in nothing)
                    ws[j] = in ? *(gvec_ptr)(w + (long long)min(16 * j + m, a.r - 1) * a.d_down + k) : u32x4{0, 0, 0, 0};
            } else {
                const int rank = RT * m < a.r ? RT * m : 0;
                uint32_t raw[8][(RT + 1) / 2];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const gu16 p = w + (long long)(in ? k + i : 0) * a.r + rank;
                    if constexpr (RT == 1) raw[i][0] = *p;
                    else if constexpr (RT == 2) raw[i][0] = *(gword)p;
                    else {
                        const u32x2 v = *(gpair)p;
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
        // Chunks of U steps go round the wavefronts; every tile begins at another one, or all workgroups would ask the same
        // channels of memory at the same time (rows are often a multiple of 4 KB apart).
        constexpr int U = NT > 1 ? 4 : RT == 4 ? 8 : 16;
        const int chunks = (steps + U - 1) / U, turn = (int)(blockIdx.x * 5u % (unsigned)chunks);
        u32x4 xs[U][NT], ws[U][RT];
        for (int n = wave; n < chunks; n += W) {
            const int c = n + turn < chunks ? n + turn : n + turn - chunks;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                load_x(c * U + u, xs[u]);                        // (zeros behind the end)
                load_w(c * U + u, ws[u]);
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
    }
    if (NT > 1 && n0 < n1) load_columns(first, group_of(n0));
    lds_barrier();
    for (int e = wave; e < RT * NT; e += W) {
        f32x4 v = sums[0][e][lane];
#pragma unroll
        for (int o = 1; o < W; ++o) v += sums[o][e][lane];
        const int j = e / NT, row = 16 * (e % NT) + m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int rank = BACK ? RT * (4 * kg + i) + j : 16 * j + 4 * kg + i;
            const float scaled = v[i] * factor;
            hs[rank][row] = scaled;
            if (a.h && blockIdx.y == 0 && rank < a.r && row < t.rows) a.h[(long long)rank * a.q.T + t.row0 + row] = BACK ? scaled : v[i];
        }
    }
    if (!a.y) return;
    lds_barrier();
    u32x4 h[NT][KS][2];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 32 * s + 8 * kg < a.r ? hs[(32 * s + 8 * kg + k) % (16 * RT)][16 * i + m] : 0.f;
            h[i][s][0] = next_part(v);
            h[i][s][1] = next_part(v);
        }
    auto add = [&](const Columns& col, int g) {
        f32x4 acc[4][NT] = {};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            u32x4 op[4];
            if constexpr (BACK) {
                columns_of(col.raw[s], op);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) op[j] = col.w[s][j];
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
                const int c0 = 64 * g + 32 * b + 8 * kg;
                if (16 * i + m >= t.rows || c0 >= a.d_up) continue;
                u32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t old = col.y[i][b][e];
                    float z[2];
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        const int c = 8 * b + 2 * e + f;         // of the lane's 16: rows 4 kg .. of the tiles
                        const float up = BACK ? acc[c % 4][i][c / 4] : acc[c / 4][i][c % 4];
                        z[f] = __uint_as_float(f ? old & 0xffff0000u : old << 16) + up;
                    }
                    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                    v[e] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)z[0], (__bf16)z[1]});
                }
                *reinterpret_cast<u32x4*>((uint16_t*)a.y + (long long)(t.row0 + 16 * i + m) * a.y_stride + c0) = v;
            }
    };
    // (two sets of registers in turn; the first is on its way since before h was there)
    Columns next;
    for (int n = n0; n < n1; n += 2) {
        if (n + 1 < n1) load_columns(next, group_of(n + 1));
        add(first, group_of(n));
        if (n + 1 >= n1) break;
        if (n + 2 < n1) load_columns(first, group_of(n + 2));
        add(next, group_of(n + 1));
    }
}

// ---------------------------------------------------------------- gradients

// The steps of 32 rows of an adapter, request by request.  Everything is the same in all lanes but the 64 requests at hand.
struct Steps {
    const Requests& q;
    const int adapter;
    int base = -64, row = 0, left = 0;
    unsigned long long rest = 0;
    Request mine{};
    __device__ Steps(const Requests& q_, int adapter_) : q(q_), adapter(adapter_) {}
    // Passes over n steps; the next one's first row and how many there are, 0 if there is none.
    __device__ __forceinline__ int skip(int n, int& row0) {
        while (left <= 32 * n) {
            n -= left > 0 ? (left + 31) / 32 : 0;
            while (rest == 0) {
                base += 64;
                if (base >= q.S) {
                    left = 0;
                    base = q.S;                                  // (stays at the end)
                    return 0;
                }
                mine = request_of(q, base + (int)(threadIdx.x & 63));
                rest = __ballot(mine.rows > 0 && mine.adapter == adapter);
            }
            const int at = __ffsll(rest) - 1;
            rest &= rest - 1;
            row = __builtin_amdgcn_readlane(mine.row0, at);
            left = __builtin_amdgcn_readlane(mine.rows, at);
        }
        row0 = row + 32 * n;
        const int rows = min(left - 32 * n, 32);
        row += 32 * (n + 1);
        left -= 32 * (n + 1);
        return rows;
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
    const gu16 x = (gu16)job.x + (c0 + 4 * m < job.d ? c0 + 4 * m : 0);
    const float* hp[RT];
#pragma unroll
    for (int j = 0; j < RT; ++j) hp[j] = job.h + (long long)min(16 * j + m, a.r - 1) * a.q.T;       // (ranks from r on end in nothing)
    f32x4 acc[4][RT] = {};
    struct Rows {
        u32x2 raw[8];
        float h[RT][8];
    };
    auto load = [&](Rows& b, int row0, int rows) {
        if (rows == 32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) b.raw[i] = *(gpair)(x + (long long)(row0 + 8 * kg + i) * job.x_stride);
#pragma unroll
            for (int j = 0; j < RT; ++j) {
                typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
                const f32x4_u u = *reinterpret_cast<const f32x4_u*>(hp[j] + row0 + 8 * kg), v = *reinterpret_cast<const f32x4_u*>(hp[j] + row0 + 8 * kg + 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    b.h[j][i] = u[i];
                    b.h[j][4 + i] = v[i];
                }
            }
        } else if (rows > 0) {
            u32x2 raw[8];
            float h[RT][8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int row = row0 + min(8 * kg + i, rows - 1);
                raw[i] = *(gpair)(x + (long long)row * job.x_stride);
#pragma unroll
                for (int j = 0; j < RT; ++j) h[j][i] = hp[j][row];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = 8 * kg + i < rows;
                b.raw[i] = in ? raw[i] : u32x2{0, 0};
#pragma unroll
                for (int j = 0; j < RT; ++j) b.h[j][i] = in ? h[j][i] : 0.f;
            }
        }
    };
    auto add = [&](Rows& b) {
        u32x4 op[4];
        columns_of(b.raw, op);
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const u32x4 hs = next_part(b.h[r]);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j][r] = mfma(op[j], hs, acc[j][r]);
            }
    };
    Steps steps(a.q, adapter);
    const int stride = kWaves * a.parts;
    Rows even, odd;
    int row0 = 0, rows = steps.skip(part * kWaves + wave, row0);
    load(even, row0, rows);
    while (rows) {
        rows = steps.skip(stride - 1, row0);
        load(odd, row0, rows);
        add(even);
        if (!rows) break;
        rows = steps.skip(stride - 1, row0);
        load(even, row0, rows);
        add(odd);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int r = 0; r < RT; ++r) sums[wave][j * RT + r][lane] = acc[j][r];
    __syncthreads();
    const float factor = job.factor ? job.factor[adapter] : 1.f;
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
            if (rank < a.r && c < job.d) out[job.rank_last ? (long long)c * a.r + rank : (long long)rank * job.d + c] = v[i] * factor;
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

template <int RT, int NT, bool BACK>
hipError_t rows_as(const LoraArgs& a, const LoraPlan& p, hipStream_t stream) {
    constexpr int W = 8;
    lora_rows_kernel<RT, NT, BACK, W><<<dim3((unsigned)p.tiles, (unsigned)(a.y ? p.slices : 1)), 64 * W, 0, stream>>>(a);
    return hipGetLastError();
}
template <int RT, bool BACK>
hipError_t rows_of(const LoraArgs& a, const LoraPlan& p, hipStream_t stream) {
    return p.shift == 4 ? rows_as<RT, 1, BACK>(a, p, stream) : rows_as<RT, 2, BACK>(a, p, stream);
}

}  // namespace

LoraPlan lora_plan(int S, int T, int d_up) {
    LoraPlan p{};
    p.shift = T > 16 * S ? 5 : 4;
    p.tiles = ((T + (1 << p.shift) - 1) >> p.shift) + S;
    const int whole = p.tiles - S > S ? p.tiles - S : S;         // about as many have rows
    const int most = (d_up + 511) / 512;                         // slices that leave a wavefront 64 columns
    p.slices = 512 / whole < 1 ? 1 : 512 / whole < most ? 512 / whole : most;
    return p;
}

hipError_t launch_lora_rows(const LoraArgs& a, const LoraPlan& p, bool back, hipStream_t stream) {
    if (back) return a.r <= 16 ? rows_of<1, true>(a, p, stream) : a.r <= 32 ? rows_of<2, true>(a, p, stream) : rows_of<4, true>(a, p, stream);
    return a.r <= 16 ? rows_of<1, false>(a, p, stream) : a.r <= 32 ? rows_of<2, false>(a, p, stream) : rows_of<4, false>(a, p, stream);
}

int lora_grad_parts(int n, int T, int d0, int d1) {
    const long long groups = (long long)n * ((d0 + 63) / 64 + (d1 + 63) / 64);
    const int steps = (T + 31) / 32;
    int parts = (int)(512 / groups);
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
