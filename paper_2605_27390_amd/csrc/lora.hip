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
// h stays in fp32 between the kernels.  As an operand it is a sum of three bf16 numbers, which are all of its 24 bits.  (Two, cut off, leave up to
// 2^-15 of it, always towards zero, which shows where ranks' shares of y cancel; y of 8,386 rows differed by 1.1e-4 of its size from fp32's, by 1.2e-5 now.  One row of
// 4,096, rank 32, 7.1 -> 7.3 us, 8,386 rows of rank 16 51.0 -> 51.1; 9,229 of rank 32, backward, 110.7 -> 112.1.
// Figures further down that compare two forms of a step are from before that: with the third part few tiles take 0.1 to 0.3 us longer, many up to 2 %, rank
// 64 forward 4 %, and backward, where places take fewer registers now, from 2 % longer to 2 % less, 700 requests of 3 rows 43.9 -> 36.6 us.)
#include <hip/hip_runtime.h>

#include <algorithm>

#include "adapt.hpp"
#include "common.hpp"

namespace evospec {
namespace {

constexpr int kThreads = 256;
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

// Neighbouring rows of one adapter.
struct Run {
    int row0, rows, adapter;
};
// No rows of a request that has no adapter, or is none.
__device__ __forceinline__ Run request_of(const Requests& q, int s) {
    Run t{0, 0, -1};
    if (s >= 0 && s < q.S) {
        t.row0 = min(max(q.row_off[s], 0), q.T);
        t.rows = min(max(q.row_off[s + 1], t.row0), q.T) - t.row0;
        t.adapter = q.adapter[s];
        if ((unsigned)t.adapter >= (unsigned)q.n) t.rows = 0;
    }
    return t;
}
// Whether a lane's request goes on with the run of the lane before it.  (All lanes take part in all exchanges: a lane that is switched off has
// nothing to give.)
__device__ __forceinline__ bool goes_on(const Run& t) {
    const int end = __shfl_up(t.row0 + t.rows, 1), adapter = __shfl_up(t.adapter, 1), rows = __shfl_up(t.rows, 1);
    return (threadIdx.x & 63) > 0 && t.rows > 0 && rows > 0 && end == t.row0 && adapter == t.adapter;
}
// Of 64 requests, lane l has request base + l: in the first lane of a run, the run; no rows in the others, or where the adapter is none.
__device__ __forceinline__ Run runs_of(const Requests& q, int base) {
    const int lane = threadIdx.x & 63;
    Run t = request_of(q, base + lane);
    if (q.S > 1) {
        const bool mine = goes_on(t);
        const u64 on = __ballot(mine);
        const int more = __ffsll((unsigned long long)~(lane < 63 ? on >> (lane + 1) : 0ull)) - 1;        // lanes that go on with this one's
        const int last = __shfl(t.row0 + t.rows, lane + more);
        t.rows = mine ? 0 : t.rows > 0 ? last - t.row0 : 0;
    }
    return t;
}
// Work item `index` of up to 1 << SHIFT rows: how many, their adapter, and in `where` (LDS; every wavefront writes the same) which.  Of 64 requests
// with one row each, as in a decode step, those with one adapter are an item together, wherever they are; otherwise runs are cut into items.
// Up to 64 requests with more rows: the items are counted, and have numbers without gaps.  Workgroups go round the card's parts by number, and
// where ones without rows lay badly some parts had twice what others had (23 requests of up to 95 rows, 7,392 -> 3,760, rank 64, 55.7 us, of up
// to 100 33.1).
// Else request s has the numbers from row0 / size + s on, one for each block of rows that it touches (the call's rows, blocks begin at multiples of
// size), so that the last request whose first number is not larger is found by looking at 64 of them at a time, however many there are; an
// item of several requests has the number of its first one there.
template <int SHIFT>
__device__ __forceinline__ Run find_rows(const Requests& q, int index, int* where) {
    constexpr int kSize = 1 << SHIFT;
    const int lane = threadIdx.x & 63;
    const auto first_number = [&](int s) { return (min(max(q.row_off[s], 0), q.T) >> SHIFT) + s; };
    int lo = 0;
    if (q.S > 64) {
        int hi = q.S;
        while (hi - lo > 1) {
            const int step = (hi - lo + 63) >> 6, s = lo + lane * step;
            const bool at_most = s < hi && first_number(s) <= index;
            const int n = __popcll(__ballot(at_most));
            if (n == 0) return Run{0, 0, 0};
            lo += (n - 1) * step;
            hi = min(lo + step, hi);
        }
    }
    const Run t = request_of(q, (lo & ~63) + lane);
    const bool one_each = __ballot(t.rows > 1) == 0;
    const u64 on = __ballot(goes_on(t));
    if (q.S <= 64 && !one_each) {
        const int more = __ffsll((unsigned long long)~(lane < 63 ? on >> (lane + 1) : 0ull)) - 1;    // lanes that go on with this one's
        const int end = __shfl(t.row0 + t.rows, lane + more);
        const int own = t.rows > 0 && !(on >> lane & 1) ? (end - t.row0 + kSize - 1) >> SHIFT : 0;
        int number = own;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int v = __shfl_up(number, o);
            number += lane >= o ? v : 0;
        }
        number -= own;
        const u64 before = __ballot(own > 0 && number <= index);
        if (before == 0) return Run{0, 0, 0};
        const int at = 63 - __clzll((long long)before);
        const int first = __builtin_amdgcn_readlane(t.row0 - (number << SHIFT), at) + (index << SHIFT);
        const int count = min(__builtin_amdgcn_readlane(end, at) - first, kSize);
        if (count <= 0) return Run{0, 0, 0};
        if (lane < kSize) where[lane] = first + min(lane, count - 1);
        return Run{first, count, __builtin_amdgcn_readlane(t.adapter, at)};
    }
    if (q.S <= 64) {
        const u64 before = __ballot(lane < q.S && (t.row0 >> SHIFT) + lane <= index);
        if (before == 0) return Run{0, 0, 0};
        lo = 63 - __clzll((long long)before);
    }
    const int at = lo & 63, block = index - lo;                  // of the call's rows
    const int row0 = __builtin_amdgcn_readlane(t.row0, at), rows = __builtin_amdgcn_readlane(t.rows, at), adapter = __builtin_amdgcn_readlane(t.adapter, at);
    const int first = max(row0, block << SHIFT), past = (block + 1) << SHIFT, last = row0 + rows;
    if (first >= last) return Run{0, 0, 0};                      // (a number that no block of the request has, or no rows)
    int count;
    if (one_each) {
        const bool mine = t.rows > 0 && t.adapter == adapter;
        const u64 same = __ballot(mine);
        const int before = __popcll(same & ((1ull << at) - 1));
        if (before & (kSize - 1)) return Run{0, 0, 0};
        const int rank = __popcll(same & ((1ull << lane) - 1)) - before;
        count = min((int)__popcll(same) - before, kSize);
        if (lane >= count && lane < kSize) where[lane] = row0;
        if (mine && rank >= 0 && rank < kSize) where[rank] = t.row0;
    } else {
        if ((on >> at & 1) && first == row0 && (row0 & (kSize - 1))) return Run{0, 0, 0};
        const int more = __ffsll((unsigned long long)~(at < 63 ? on >> (at + 1) : 0ull)) - 1;
        const int end = min(__builtin_amdgcn_readlane(t.row0 + t.rows, at + more), past);
        count = (last < past ? end : past) - first;
        if (lane < kSize) where[lane] = min(first + lane, first + count - 1);
    }
    return Run{first, count, adapter};
}

// Zeros for what h has in columns [base, base + size) of rows that no adapter is for.  (All of a workgroup of W wavefronts.)
template <int W>
__device__ __forceinline__ void zeros_of_none(const Requests& q, int base, int size, float* h, int r) {
    const int lane = threadIdx.x & 63, end = min(base + size, q.T);
    int lo = 0;                                                  // the last request, of those at multiples of 64, that begins at or before base
    for (int hi = (q.S + 63) >> 6; hi - lo > 1;) {
        const int step = (hi - lo + 63) >> 6, s = lo + lane * step;
        const bool at_most = s < hi && min(max(q.row_off[64 * s], 0), q.T) <= base;
        const int n = max((int)__popcll(__ballot(at_most)), 1);
        lo += (n - 1) * step;
        hi = min(lo + step, hi);
    }
    u64 there = 0;
    for (int s = 64 * lo; s < q.S; s += 64) {
        const Run t = request_of(q, s + lane);
        const int from = max(t.row0, base) - base, to = min(t.row0 + t.rows, end) - base;
        u64 mine = to > from ? ((1ull << (to - from)) - 1) << from : 0;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) mine |= __shfl_xor(mine, o);
        there |= mine;
        if (s + 64 < q.S && q.row_off[s + 64] >= end) break;
    }
    for (int e = threadIdx.x; e < size * r; e += 64 * W) {
        const int row = e % size;
        if (base + row < end && !(there >> row & 1)) h[(long long)(e / size) * q.T + base + row] = 0.f;
    }
}

// ---------------------------------------------------------------- rows

typedef const void __attribute__((address_space(1))) * gptr;
typedef void __attribute__((address_space(3))) * lptr;
typedef const u32x2 __attribute__((address_space(1))) * gpair;
typedef const uint32_t __attribute__((address_space(1))) * gword;
typedef const char __attribute__((address_space(1))) * gbyte;
typedef const float __attribute__((address_space(1))) * gfloat;
typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef const f32x4_u __attribute__((address_space(1))) * gfloat4;

// One tile of 16 NT rows: h = x W_down^T, then y += h W_up for a slice of the columns.  Forward, W_down = A [r][d] and W_up = B [d][r]; backward
// W_down = B^T and W_up = A^T of the same arrays.  The long axis of the first product is split over W wavefronts, whose sums are added
// in LDS; in the second each takes 64 columns at a time.  Every slice computes h again: it is launched with slices where tiles are
// few and the time is that of a launch.
// An operand's neighbouring lanes are neighbouring rows, and a load that follows them touches 64 lines of memory for 1 KB, one a clock: 16 KB of
// a compute unit's time for 256 KB.  So rows (x, and A forward) are loaded 128 bytes of a row to 8 lanes and change lanes in LDS (a
// wavefront's own, no barriers; piece c of row m in place c ^ (m mod 8), without bank conflicts), B forward in the order of memory.  Of y a
// lane has 4 columns in 4 rows, the columns of a row in 16 lanes.
// DEEP, where tiles and slices leave a compute unit one workgroup at most: 8 wavefronts.  Else four workgroups of 4 to a unit (two of rank 40 and
// more), so that some load while others store.  ONCE: y past the caches.
template <int RT, int NT, bool BACK, bool DEEP, bool ONCE>
__global__ __launch_bounds__(DEEP ? 512 : 256, RT < 4 ? 4 : NT == 1 && !DEEP ? 3 : 2) void lora_rows_kernel(LoraArgs a) {
    constexpr int W = DEEP ? 8 : 4;
    constexpr int KS = (RT + 1) / 2;
    constexpr int kSets = BACK ? NT : NT + RT;                   // of 16 rows through LDS: x's, then A's
    constexpr int kAhead = BACK || !DEEP || RT == 4 ? 1 : RT == 2 ? 3 : 4;               // chunks of a wavefront on their way to LDS
    constexpr int kOwn = kAhead * kSets * 128 > RT * NT * 64 ? kAhead * kSets * 128 : RT * NT * 64;      // 16-byte pieces of a wavefront (64 columns of B: up to 128 RT)
    __shared__ __align__(16) u32x4 own[W][kOwn];
    __shared__ float hs[16 * RT][16 * NT + 1];
    __shared__ int where[16 * NT];
    const int tile = blockIdx.x / 8 / a.slices * 8 + blockIdx.x % 8, slice = blockIdx.x / 8 % a.slices;        // a tile's slices on one of the 8 dies
    const Run t = find_rows<NT == 1 ? 4 : 5>(a.q, tile, where);
    if constexpr (!BACK)
        if (a.h && a.y && slice == 0 && 16 * NT * tile < a.q.T) zeros_of_none<W>(a.q, 16 * NT * tile, 16 * NT, a.h, a.r);
    if (t.rows == 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, kg = lane >> 4;
    const float factor = a.factor ? a.factor[t.adapter] : 1.f;
    u32x4* mine = own[wave];

    int row_of[NT][4];                                           // this lane's rows of y
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) row_of[i][k] = where[16 * i + 4 * kg + k];
    // 64 columns of the second product: what this lane has of y, and of the weights what operands are made of.  Column 4 m + j of them is
    // column m of tile j.
    struct Columns {
        u32x2 y[NT][4];
        u32x4 w[BACK ? 1 : 2 * RT];
        u32x2 raw[BACK ? KS : 1][8];
    };
    const gu16 w_up = (gu16)a.w_up + (long long)__builtin_amdgcn_readfirstlane(t.adapter) * a.r * a.d_up;
    auto load_columns = [&](Columns& col, int g) {
        const int c = min(64 * g + 4 * m, a.d_up - 4);
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const gpair p = (gpair)((gu16)a.y + (long long)row_of[i][k] * a.y_stride + c);
                col.y[i][k] = ONCE ? __builtin_nontemporal_load(p) : *p;
            }
        if constexpr (BACK) {                                    // [r][d]
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                // (a uniform address and a lane's 32 bits of offset: 16 registers less than a place of its own for each load)
                const uint32_t at = 2u * ((uint32_t)(32 * s + 8 * kg < a.r ? 32 * s + 8 * kg : 0) * (uint32_t)a.d_up + (uint32_t)c);
#pragma unroll
                for (int k = 0; k < 8; ++k) col.raw[s][k] = *(gpair)((gbyte)(w_up + (long long)k * a.d_up) + at);
            }
        } else {                                                 // [d][r]: r / 8 KB
            const int pieces = min(64, a.d_up - 64 * g) * a.r / 8;
#pragma unroll
            for (int k = 0; k < 2 * RT; ++k) col.w[k] = *(gvec_ptr)(w_up + (long long)(64 * g) * a.r + 8 * min(64 * k + lane, pieces - 1));
        }
    };
    // Groups of a slice go round the wavefronts; every tile begins at another one (as in the first product).
    const int groups = (a.d_up + 63) / 64, g0 = (int)((long long)groups * slice / a.slices);
    const int count = a.y ? (int)((long long)groups * (slice + 1) / a.slices) - g0 : 0, shift = count ? (int)(tile * 5u % (unsigned)count) : 0;
    auto group_of = [&](int n) { return g0 + (n + shift < count ? n + shift : n + shift - count); };
    Columns first;
    if (DEEP && RT < 4 && wave < count) load_columns(first, group_of(wave));
    {
        // Chunks of 64 along the summed axis go round the wavefronts; every tile begins at another one, or all workgroups would ask the same
        // channels of memory at the same time (rows are often a multiple of 4 KB apart).  One chunk at a time: the next one's loads ahead, or three
        // and four chunks in registers, cost more in instructions, which every launch has to bring in, than they hide (1, 2, 3 chunks ahead at one row
        // of 4,096, rank 32: 8.3, 9.1, 9.8 us, none ahead 8.1; 9,000 rows 57.5, none ahead 55.5).
        const int chunks = (a.d_down + 63) / 64, turn = (int)(tile * 5u % (unsigned)chunks);
        const int row8 = lane >> 3, piece = lane & 7;
        gu16 from[kSets][2];
#pragma unroll
        for (int i = 0; i < kSets; ++i)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (i < NT) from[i][b] = (gu16)a.x + (long long)where[16 * i + 8 * b + row8] * a.x_stride + 8 * piece;
                else from[i][b] = (gu16)a.w_down + ((long long)t.adapter * a.r + min(16 * (i - NT) + 8 * b + row8, a.r - 1)) * a.d_down + 8 * piece;
            }
        const gu16 w = (gu16)a.w_down + (long long)t.adapter * a.r * a.d_down;
        f32x4 acc[RT][NT] = {};
        // (8 rows that a tile does not have are not loaded: what their lanes find in LDS ends in rows that are not stored.  8.1 -> 7.7 us for one row.)
        if constexpr (kAhead > 1) {
            // Few tiles, forward: what an operand is made of goes to LDS by itself, three or four chunks at a time (lane l loads what belongs in
            // place l: of row l / 8 the piece (l mod 8) ^ (l / 8)).  One row of 4,096, rank 32, 7.65 -> 7.04 us, 64 requests of one row 8.2 -> 7.6,
            // 600 rows 10.7 -> 10.1; 2,000 rows of 7,392, which begin between lines, 22.0 -> 22.9.
            const int moved = 8 * ((piece ^ row8) - piece);
            for (int n = wave; n < chunks; n += kAhead * W) {
                const int there = min(kAhead, (chunks - n + W - 1) / W);
#pragma unroll 1
                for (int u = 0; u < there; ++u) {
                    const int c = n + W * u + turn, at = c < chunks ? c : c - chunks, here = 64 * at + 8 * (piece ^ row8) < a.d_down ? 64 * at + moved : -8 * piece;
                    u32x4* to = mine + u * kSets * 128;
#pragma unroll
                    for (int i = 0; i < kSets; ++i)
#pragma unroll
                        for (int b = 0; b < 2; ++b)
                            if (i >= NT || 16 * i + 8 * b < t.rows) __builtin_amdgcn_global_load_lds((gptr)(from[i][b] + here), (lptr)(to + 128 * i + 64 * b), 16, 0, 0);
                }
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll 1
                for (int u = 0; u < there; ++u) {
                    const int c = n + W * u + turn, at = c < chunks ? c : c - chunks;
                    const u32x4* have = mine + u * kSets * 128;
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const int place = 8 * m + ((4 * s + kg) ^ (m & 7));
                        u32x4 x[NT], ws[RT];
#pragma unroll
                        for (int i = 0; i < NT; ++i) x[i] = have[128 * i + place];
#pragma unroll
                        for (int j = 0; j < RT; ++j) ws[j] = have[128 * (NT + j) + place];
                        if (64 * at + 64 > a.d_down) {           // zeros for what the last chunk does not have
                            const bool in = 64 * at + 8 * (4 * s + kg) < a.d_down;
#pragma unroll
                            for (int i = 0; i < NT; ++i) x[i] = in ? x[i] : u32x4{0, 0, 0, 0};
#pragma unroll
                            for (int j = 0; j < RT; ++j) ws[j] = in ? ws[j] : u32x4{0, 0, 0, 0};
                        }
#pragma unroll
                        for (int i = 0; i < NT; ++i)
#pragma unroll
                            for (int j = 0; j < RT; ++j) acc[j][i] = mfma(ws[j], x[i], acc[j][i]);
                    }
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");               // (read, before the next chunks come)
            }
        } else
        for (int n = wave; n < chunks; n += W) {
            const int at = n + turn < chunks ? n + turn : n + turn - chunks, here = 64 * at + 8 * piece < a.d_down ? 64 * at : -8 * piece;
            u32x4 rows[kSets][2];
            uint32_t raw[BACK ? 2 : 1][8][(RT + 1) / 2];
#pragma unroll
            for (int i = 0; i < kSets; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b)
                    if (i >= NT || 16 * i + 8 * b < t.rows) rows[i][b] = *(gvec_ptr)(from[i][b] + here);
            if constexpr (BACK) {
                const int rank = RT * m < a.r ? RT * m : 0;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int k = 64 * at + 32 * s + 8 * kg < a.d_down ? 64 * at + 32 * s + 8 * kg : 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const gu16 p = w + (long long)(k + i) * a.r + rank;
                        if constexpr (RT == 1) raw[s][i][0] = *p;
                        else if constexpr (RT == 2) raw[s][i][0] = *(gword)p;
                        else {
                            const u32x2 v = *(gpair)p;
                            raw[s][i][0] = v[0];
                            raw[s][i][1] = v[1];
                        }
                    }
                }
            }
            if (64 * at + 64 > a.d_down) {                       // zeros for what the last chunk does not have
#pragma unroll
                for (int i = 0; i < kSets; ++i)
#pragma unroll
                    for (int b = 0; b < 2; ++b) rows[i][b] = 64 * at + 8 * piece < a.d_down ? rows[i][b] : u32x4{0, 0, 0, 0};
                if constexpr (BACK) {
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int i = 0; i < 8; ++i)
#pragma unroll
                            for (int e = 0; e < (RT + 1) / 2; ++e) raw[s][i][e] = 64 * at + 32 * s + 8 * kg < a.d_down ? raw[s][i][e] : 0u;
                }
            }
#pragma unroll
            for (int i = 0; i < kSets; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b)
                    if (i >= NT || 16 * i + 8 * b < t.rows) mine[128 * i + 64 * b + 8 * row8 + (piece ^ row8)] = rows[i][b];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                u32x4 ws[RT];
#pragma unroll
                for (int j = 0; j < RT; ++j) {
                    if constexpr (!BACK) {
                        ws[j] = mine[128 * (NT + j) + 8 * m + ((4 * s + kg) ^ (m & 7))];
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            ws[j][i] = j & 1 ? high_halves(raw[s][2 * i][j / 2], raw[s][2 * i + 1][j / 2]) : low_halves(raw[s][2 * i][j / 2], raw[s][2 * i + 1][j / 2]);
                    }
                }
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const u32x4 x = mine[128 * i + 8 * m + ((4 * s + kg) ^ (m & 7))];
#pragma unroll
                    for (int j = 0; j < RT; ++j) acc[j][i] = mfma(ws[j], x, acc[j][i]);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < RT; ++j)
#pragma unroll
            for (int i = 0; i < NT; ++i) mine[64 * (j * NT + i) + lane] = __builtin_bit_cast(u32x4, acc[j][i]);
    }
    if ((!DEEP || RT == 4) && wave < count) load_columns(first, group_of(wave));
    lds_barrier();
    for (int e = wave; e < RT * NT; e += W) {
        f32x4 v = __builtin_bit_cast(f32x4, own[0][64 * e + lane]);
#pragma unroll
        for (int o = 1; o < W; ++o) v += __builtin_bit_cast(f32x4, own[o][64 * e + lane]);
        const int j = e / NT, row = 16 * (e % NT) + m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int rank = BACK ? RT * (4 * kg + i) + j : 16 * j + 4 * kg + i;
            const float scaled = v[i] * factor;
            hs[rank][row] = scaled;
            if (a.h && slice == 0 && rank < a.r && row < t.rows) a.h[(long long)rank * a.q.T + where[row]] = BACK ? scaled : v[i];
        }
    }
    if (!a.y) return;
    lds_barrier();
    u32x4 h[NT][KS][3];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 32 * s + 8 * kg < a.r ? hs[(32 * s + 8 * kg + k) % (16 * RT)][16 * i + m] : 0.f;
#pragma unroll
            for (int k = 0; k < 3; ++k) h[i][s][k] = next_part(v);
        }
    // B's 16-byte pieces in LDS: number p, of column p / (r / 8), with its low 4 bits turned by what the columns of a read differ in
    const int turned = a.r > 32 ? 5 : 4, per = a.r / 8;
    auto add = [&](Columns& col, int g) {
        if constexpr (!BACK) {
#pragma unroll
            for (int k = 0; k < 2 * RT; ++k)
                if (64 * k < 8 * a.r) {
                    const int p = 64 * k + lane;
                    mine[p ^ ((p >> turned) & 15)] = col.w[k];
                }
        }
        f32x4 acc[4][NT] = {};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            u32x4 op[4];
            if constexpr (BACK) {
                if (a.r < 32 * s + 32) {
                    const bool in = 32 * s + 8 * kg < a.r;
#pragma unroll
                    for (int k = 0; k < 8; ++k) col.raw[s][k] = in ? col.raw[s][k] : u32x2{0, 0};
                }
                columns_of(col.raw[s], op);
            } else {
                const bool in = 32 * s + 8 * kg < a.r;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int p = (4 * m + j) * per + (in ? 4 * s + kg : 0);
                    const u32x4 v = mine[p ^ ((p >> turned) & 15)];
                    op[j] = in ? v : u32x4{0, 0, 0, 0};
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int k = 0; k < 3; ++k) acc[j][i] = mfma(h[i][s][k], op[j], acc[j][i]);
        }
        const int c = 64 * g + 4 * m;
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int row = 16 * i + 4 * kg + k;
                if (row >= t.rows || c >= a.d_up) continue;
                const uint32_t y0 = col.y[i][k][0], y1 = col.y[i][k][1];
                typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                const bf16x4 v = {(__bf16)(__uint_as_float(y0 << 16) + acc[0][i][k]), (__bf16)(__uint_as_float(y0 & 0xffff0000u) + acc[1][i][k]),
                                  (__bf16)(__uint_as_float(y1 << 16) + acc[2][i][k]), (__bf16)(__uint_as_float(y1 & 0xffff0000u) + acc[3][i][k])};
                bf16x4* p = reinterpret_cast<bf16x4*>((uint16_t*)a.y + (long long)row_of[i][k] * a.y_stride + c);
                if constexpr (ONCE) __builtin_nontemporal_store(v, p);
                else *p = v;
            }
    };
    // (two sets of registers in turn; the first is on its way since before h was there, or, where registers are few, since the sums are.  A load under a
    // condition would leave the compiler without a count of those on their way, and it would wait for all: 55.3 -> 51.1 us for 8,400 rows of rank 16.)
    Columns next;
    int n = wave;
    for (; n + 2 * W < count; n += 2 * W) {
        load_columns(next, group_of(n + W));
        add(first, group_of(n));
        load_columns(first, group_of(n + 2 * W));
        add(next, group_of(n + W));
    }
    if (n + W < count) {
        load_columns(next, group_of(n + W));
        add(first, group_of(n));
        add(next, group_of(n + W));
    } else if (n < count) {
        add(first, group_of(n));
    }
}

// ---------------------------------------------------------------- gradients

// The steps of 32 rows of an adapter, run by run.  Everything is the same in all lanes but the 64 requests at hand.
struct Steps {
    const Requests& q;
    const int adapter;
    int base = -64, row = 0, left = 0;
    u64 rest = 0;
    Run mine{};
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
                if (q.S - base > 256) {                          // many: groups of 64 without the adapter are passed over four at a time
                    u64 there[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) there[i] = __ballot(q.adapter[base + 64 * i + (int)(threadIdx.x & 63)] == adapter);
                    const int at = there[0] ? 0 : there[1] ? 1 : there[2] ? 2 : 3;
                    base += 64 * at;
                    if (!there[at]) continue;
                }
                mine = runs_of(q, base);
                rest = __ballot(mine.rows > 0 && mine.adapter == adapter);
            }
            const int at = __ffsll((unsigned long long)rest) - 1;
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

// How many of `parts` an adapter's rows are split into: its share of the call's rows, so that workgroups are as many wherever the rows are.
// (All threads of a workgroup; every workgroup finds the same.)
__device__ int parts_of(const Requests& q, int adapter, int parts) {
    __shared__ unsigned found[kThreads / 64 * 2];
    if (parts == 1) return 1;
    const unsigned all = (unsigned)q.T;
    unsigned rows = 0;                                           // (up to T, if offsets are not in order)
    const int step = q.S <= 64 ? 64 : blockDim.x;                // (few: every wavefront by itself)
    for (int s = threadIdx.x & (step - 1); s < q.S; s += step) {
        const Run t = request_of(q, s);
        rows = min(rows + (t.adapter == adapter ? (unsigned)t.rows : 0u), all);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) rows = min(rows + __shfl_xor(rows, o), all);
    if (q.S > 64) {
        if ((threadIdx.x & 63) == 0) found[threadIdx.x >> 6] = rows;
        __syncthreads();
        rows = 0;
        for (unsigned w = 0; w < blockDim.x / 64; ++w) rows = min(rows + found[w], all);
    }
    return max(1, (int)((rows * (unsigned)parts + all / 2) / all));
}

// RT tiles of 16 ranks (rank 33 and more in two halves); a workgroup has 64 CG columns of one adapter, its wavefronts and `parts` workgroups every so many-th step.  A step of
// 64 CG columns and 32 rows is 4 CG KB of x and, from L2, 2 RT KB of h, which becomes an operand in three parts.
template <int RT, int CG, int W>
__global__ __launch_bounds__(64 * W, 2) void lora_grads_kernel(GradArgs a, int groups0, int halves, long long partial_stride) {
    constexpr int kTiles = 4 * CG * RT;
    __shared__ __align__(16) f32x4 sums[W / 2][kTiles][64];
    static_assert(sizeof(sums) >= (size_t)W * RT * 2048, "h of every wavefront's step");
    const bool second = (int)blockIdx.x >= groups0;
    const GradJob job = second ? a.job[1] : a.job[0];
    const int c0 = 64 * CG * (blockIdx.x - (second ? groups0 : 0)), adapter = blockIdx.y, part = blockIdx.z / halves, rank0 = 32 * (blockIdx.z % halves);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, kg = lane >> 4;
    // Places as a uniform address and a lane's 32 bits of offset (row strides are below 2^26, h is smaller than 4 GB): half the registers.
    const uint32_t down = (uint32_t)(8 * kg * job.x_stride) * 2u;
    uint32_t x[CG];
#pragma unroll
    for (int g = 0; g < CG; ++g) x[g] = 2u * (c0 + 64 * g + 4 * m < job.d ? c0 + 64 * g + 4 * m : 0);
    // h goes through LDS as the rows of lora_rows_kernel do: 32 numbers of a rank are 8 pieces, loaded by 8 lanes, the even pieces first
    const int rank8 = lane >> 3, piece = lane & 7, slot = ((piece >> 1) + 4 * (piece & 1)) ^ rank8;
    uint32_t hp[2 * RT];
#pragma unroll
    for (int j = 0; j < 2 * RT; ++j) hp[j] = 4u * ((uint32_t)min(rank0 + 8 * j + rank8, a.r - 1) * (uint32_t)a.q.T + 4u * piece);    // (ranks from r on end in nothing)
    f32x4* mine = &sums[0][0][0] + wave * RT * 128;
    f32x4 acc[CG][4][RT] = {};
    struct Rows {
        u32x2 raw[CG][8];
        f32x4 h[2 * RT];
    };
    auto load = [&](Rows& b, int row0, int rows) {
        if (rows == 32) {
#pragma unroll
            for (int g = 0; g < CG; ++g)
#pragma unroll
                for (int i = 0; i < 8; ++i) b.raw[g][i] = *(gpair)((gbyte)((gu16)job.x + (long long)(row0 + i) * job.x_stride) + (down + x[g]));
#pragma unroll
            for (int j = 0; j < 2 * RT; ++j) b.h[j] = *(gfloat4)((gbyte)(job.h + row0) + hp[j]);
        } else {                                                 // a run's end
            const int last = max(rows - 1, 0);
#pragma unroll
            for (int g = 0; g < CG; ++g)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    b.raw[g][i] = *(gpair)((gbyte)((gu16)job.x + (long long)row0 * job.x_stride) + ((uint32_t)min(8 * kg + i, last) * (uint32_t)job.x_stride * 2u + x[g]));
#pragma unroll
            for (int j = 0; j < 2 * RT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) b.h[j][i] = *(gfloat)((gbyte)(job.h + row0) + (hp[j] + 4u * min(4 * piece + i, last) - 16u * piece));
        }
    };
    auto add = [&](Rows& b, int rows) {
        if (rows < 32) {
#pragma unroll
            for (int g = 0; g < CG; ++g)
#pragma unroll
                for (int i = 0; i < 8; ++i) b.raw[g][i] = 8 * kg + i < rows ? b.raw[g][i] : u32x2{0, 0};
#pragma unroll
            for (int j = 0; j < 2 * RT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) b.h[j][i] = 4 * piece + i < rows ? b.h[j][i] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 2 * RT; ++j) mine[64 * j + 8 * rank8 + slot] = b.h[j];
        // (x's operands of one group at a time, h's of one rank tile or of all: what fewer registers hold)
        u32x4 op[4], hs[CG > 1 ? RT : 1][3];
        auto parts_of = [&](int r, u32x4 (&to)[3]) {
            const f32x4 u = mine[128 * r + 8 * m + (kg ^ (m & 7))], v = mine[128 * r + 8 * m + ((4 + kg) ^ (m & 7))];
            float h[8] = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
#pragma unroll
            for (int k = 0; k < 3; ++k) to[k] = next_part(h);
        };
        if constexpr (CG > 1) {
#pragma unroll
            for (int r = 0; r < RT; ++r) parts_of(r, hs[r]);
        }
#pragma unroll
        for (int g = 0; g < CG; ++g) {
            columns_of(b.raw[g], op);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if constexpr (CG == 1) parts_of(r, hs[0]);
#pragma unroll
                for (int k = 0; k < 3; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[g][j][r] = mfma(op[j], hs[CG > 1 ? r : 0][k], acc[g][j][r]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const int parts = parts_of(a.q, adapter, a.parts);
    if (part >= parts) return;
    float* out = parts > 1 ? a.partial + part * partial_stride + (second ? (long long)a.q.n * a.r * a.job[0].d : 0ll) : job.out;
    out += (long long)adapter * a.r * job.d;
    Steps steps(a.q, adapter);
    const int stride = W * parts;
    Rows now;
    int row0 = 0, rows = steps.skip(part * W, row0);
    if (rows == 0) {                                             // (the same in all wavefronts) nothing to add: an adapter without rows, often
        const int ranks = min(a.r - rank0, 16 * RT) / 4, columns = min(64 * CG, job.d - c0);
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        if (job.rank_last)
            for (int e = threadIdx.x; e < columns * ranks; e += 64 * W)
                *reinterpret_cast<f32x4*>(out + (long long)(c0 + e / ranks) * a.r + rank0 + 4 * (e % ranks)) = zero;
        else
            for (int e = threadIdx.x; e < columns * ranks; e += 64 * W)
                *reinterpret_cast<f32x4*>(out + (long long)(rank0 + e / (columns / 4)) * job.d + c0 + 4 * (e % (columns / 4))) = zero;
        return;
    }
    if (wave > 0) rows = steps.skip(wave - 1, row0);
    load(now, row0, rows);
    // (one step's registers: the next one's loads ahead double the instructions that a launch brings in and leave fewer wavefronts; 64 rows of 16 adapters
    // 14.5 us, 11.1 without, 6,400 of 16 46.0 and 40.1, 9,000 of 2 43.0 and 42.5; where few workgroups have rows 24.2 and 27.7, 72.6 and 79.5)
#pragma unroll 1
    while (rows) {
        add(now, rows);
        rows = steps.skip(stride - 1, row0);
        if (rows) load(now, row0, rows);
    }
    // The upper half of the wavefronts first, whose sums the lower half takes along.
    __syncthreads();
    f32x4* own = sums[wave & (W / 2 - 1)][0];
    if (wave >= W / 2)
#pragma unroll
        for (int g = 0; g < CG; ++g)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < RT; ++r) own[64 * ((g * 4 + j) * RT + r) + lane] = acc[g][j][r];
    __syncthreads();
    if (wave < W / 2)
#pragma unroll
        for (int g = 0; g < CG; ++g)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < RT; ++r) own[64 * ((g * 4 + j) * RT + r) + lane] += acc[g][j][r];
    __syncthreads();
    const float factor = job.factor ? job.factor[adapter] : 1.f;
    if (job.rank_last) {
        for (int e = wave; e < kTiles; e += W) {
            f32x4 v = sums[0][e][lane];
#pragma unroll
            for (int o = 1; o < W / 2; ++o) v += sums[o][e][lane];
            const int g = e / (4 * RT), j = e / RT % 4, rank = rank0 + 16 * (e % RT) + m;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = c0 + 64 * g + 4 * (4 * kg + i) + j;
                if (rank < a.r && c < job.d) out[(long long)c * a.r + rank] = v[i] * factor;
            }
        }
    } else {
        // (a thread has 16 columns in a row of a rank, its neighbours the next ones)
        for (int e = threadIdx.x; e < 64 * RT * CG; e += 64 * W) {
            const int k = e % 4, g = e / 4 % CG, rank = e / (4 * CG), c = c0 + 64 * g + 16 * k;
            f32x4 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = (g * 4 + j) * RT + rank / 16;
                v[j] = sums[0][at][16 * k + rank % 16];
#pragma unroll
                for (int o = 1; o < W / 2; ++o) v[j] += sums[o][at][16 * k + rank % 16];
            }
            if (rank0 + rank >= a.r) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + 4 * i < job.d) *reinterpret_cast<f32x4*>(out + (long long)(rank0 + rank) * job.d + c + 4 * i) = f32x4{v[0][i], v[1][i], v[2][i], v[3][i]} * factor;
        }
    }
}

__global__ __launch_bounds__(kThreads) void lora_grads_sum_kernel(GradArgs a, long long partial_stride) {
    const int parts = parts_of(a.q, blockIdx.y, a.parts);
    if (parts == 1) return;
    const long long of0 = (long long)a.r * a.job[0].d / 4, of1 = (long long)a.r * a.job[1].d / 4;
    for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < of0 + of1; i += (long long)gridDim.x * kThreads) {
        const bool second = i >= of0;
        const long long at = second ? blockIdx.y * of1 + i - of0 : blockIdx.y * of0 + i;         // (in its output, and, behind the first output's, in a part)
        const f32x4* partial = reinterpret_cast<const f32x4*>(a.partial) + (second ? a.q.n * of0 : 0ll) + at;
        f32x4 s = *partial;
        for (int p = 1; p < parts; ++p) s += partial[p * (partial_stride / 4)];
        reinterpret_cast<f32x4*>(a.job[second].out)[at] = s;
    }
}

template <int RT, int NT, bool BACK>
hipError_t rows_as(LoraArgs a, const LoraPlan& p, hipStream_t stream) {
    a.slices = a.y ? p.slices : 1;
    const unsigned grid = (unsigned)(p.tiles + 7) / 8 * 8 * a.slices;
    if (p.deep) lora_rows_kernel<RT, NT, BACK, true, false><<<grid, 512, 0, stream>>>(a);
    else if (p.once) lora_rows_kernel<RT, NT, BACK, false, true><<<grid, 256, 0, stream>>>(a);
    else lora_rows_kernel<RT, NT, BACK, false, false><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}
template <bool BACK>
hipError_t rows_of(const LoraArgs& a, const LoraPlan& p, hipStream_t stream) {
    if (a.r <= 16) return rows_as<1, 1, BACK>(a, p, stream);
    if (a.r <= 32) return rows_as<2, 1, BACK>(a, p, stream);
    return p.wide ? rows_as<4, 2, BACK>(a, p, stream) : rows_as<4, 1, BACK>(a, p, stream);
}

}  // namespace

// Measured at d = 4,096, rank 32: 64 rows in 1, 4, 8 slices 14.3, 9.6, 9.0 us; 1,024 rows in 1, 2, 4, 8 16.7, 13.6, 12.1, 15.5; 2,048 in
// 1, 2, 4 17.2, 14.7, 17.5; with smaller workgroups at best 11.0, 16.2, 19.1.  4,096 rows (a tile to a compute unit) 19.3, and 24.7 with smaller
// workgroups, which win from there on (4,500 rows of rank 64, 141 tiles of 32 rows, 29.9, and 39.6 with smaller ones).
// As many tiles as T rows and half a tile for every request have: with more than units, the last ones begin when the others end (2,000 rows of 23
// requests, rank 64, 7,392 -> 3,760: 61.8 us in 4 slices, 34.2 in 3).
// Rank 40 and more in tiles of 32 rows where tiles of 16 are many: backward, 9,000 rows of 4,096, rank 40 83.3 -> 69.6 us, 6,554 of 6,208, rank 64,
// 92.7 -> 73.9; 600 rows of 4,096, rank 64, 18.1, and 15.8 in tiles of 16, 2,000 20.7 and 19.9, 3,000 25.0 and 25.8.
// y past the caches where x and y are 128 MB or more: 8,400 rows of rank 16, other rows between, 58.3 -> 50.0 us; 4,096 rows of rank 32, which are
// found in the caches, 24.7 -> 29.7.
LoraPlan lora_plan(int S, int T, int r, int d_down, int d_up) {
    LoraPlan p{};
    p.wide = r > 32 && T > 16 * S && (T + 15) / 16 + S / 2 > 128;
    const int size = p.wide ? 32 : 16, full = (T + size - 1) / size, whole = full + S / 2 > S ? full + S / 2 : S;      // about as many have rows
    p.tiles = full + S;
    p.deep = whole <= 256;
    const int most = (d_up + 511) / 512;                         // slices that leave a wavefront 64 columns
    p.slices = std::max(1, std::min(32 / ((whole + 7) / 8), most));      // (of 32 units on a die)
    p.once = !p.deep && (size_t)T * ((size_t)d_down + d_up) * 2 >= (size_t)128 << 20;
    return p;
}

hipError_t launch_lora_rows(const LoraArgs& a, const LoraPlan& p, bool back, hipStream_t stream) {
    return back ? rows_of<true>(a, p, stream) : rows_of<false>(a, p, stream);
}

// Columns of a workgroup of the gradients, and halves of the ranks: what 256 registers hold without spilling.
static int grad_columns(int r) { return r <= 16 ? 128 : 64; }
static int grad_halves(int r) { return r <= 32 ? 1 : 2; }

long long lora_grad_groups(int n, int r, int d0, int d1) {
    const int c = grad_columns(r);
    return (long long)n * grad_halves(r) * ((d0 + c - 1) / c + (d1 + c - 1) / c);
}

// Parts that fill the card if all rows are of one adapter, of at least two steps to a wavefront (parts_of shares them out).  Where there are several
// adapters the parts, and the launch that adds them, may turn out not to be needed: four steps, and one adapter alone would have a third of the
// card.  (5 adapters, all rows of one, 7,000 rows of rank 8 39.1 -> 20.7 us, 5,900 of rank 16 55.9 -> 43.5; 9,000 rows of 2, which then have as
// many parts as before, 32.9 -> 33.6, 12 adapters 19.1 -> 21.0; with two parts, rank 32, 42.9 -> 45.1.  One request of 8,735 rows, 73.3 -> 46.7.)
// A workspace of 128 MB at most.
int lora_grad_parts(int n, int r, int S, int T, int d0, int d1) {
    const bool several = n > 1 && S > 1;                         // adapters, among which the rows may lie anyhow
    const int each = several ? 32 : 16;
    const long long most = ((T + 31) / 32 + each - 1) / each, fit = (128 << 20) / ((long long)n * r * (d0 + d1) * 4);
    const long long parts = std::min(std::min(256 / lora_grad_groups(1, r, d0, d1), 16ll), std::min(most, fit));
    return parts < (several ? 3 : 2) ? 1 : (int)parts;
}

hipError_t launch_lora_grads(const GradArgs& a, hipStream_t stream) {
    const int c = grad_columns(a.r), groups0 = (a.job[0].d + c - 1) / c, groups1 = (a.job[1].d + c - 1) / c, halves = grad_halves(a.r);
    const long long count0 = (long long)a.q.n * a.r * a.job[0].d, count1 = (long long)a.q.n * a.r * a.job[1].d;
    const dim3 grid((unsigned)(groups0 + groups1), (unsigned)a.q.n, (unsigned)(a.parts * halves));
    // One workgroup of 8 wavefronts to a compute unit; where there are more than units that have rows, of 4, or of 2 with few rows each, so that some
    // load while others store (9,000 rows of 2 adapters, rank 32, 8 / 4 / 2 wavefronts 42.6 / 44.5 / 72.7 us; rank 64, twice as many workgroups,
    // 73.0 / 67.7 / 99.9; 6,400 rows of 16 adapters 55.6 / 40.2 / 44.0; 64 rows of 16 21.9 / 15.9 / 11.2).
    const int used = a.q.n < a.q.S ? a.q.n : a.q.S;
    const long long full = lora_grad_groups(used, a.r, a.job[0].d, a.job[1].d);
    const int waves = full <= 256 ? 8 : a.q.T <= 32 * used ? 2 : 4;
    auto go = [&](auto kernel) { kernel<<<grid, 64 * waves, 0, stream>>>(a, groups0, halves, count0 + count1); };
    if (a.r <= 16) waves == 8 ? go(lora_grads_kernel<1, 2, 8>) : waves == 4 ? go(lora_grads_kernel<1, 2, 4>) : go(lora_grads_kernel<1, 2, 2>);
    else waves == 8 ? go(lora_grads_kernel<2, 1, 8>) : waves == 4 ? go(lora_grads_kernel<2, 1, 4>) : go(lora_grads_kernel<2, 1, 2>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.parts == 1) return e;
    const unsigned blocks = (unsigned)(((count0 + count1) / a.q.n / 4 + kThreads - 1) / kThreads);
    lora_grads_sum_kernel<<<dim3(std::min(blocks, 256u), (unsigned)a.q.n), kThreads, 0, stream>>>(a, count0 + count1);
    return hipGetLastError();
}

}  // namespace evospec
