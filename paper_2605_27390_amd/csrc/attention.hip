// Attention over the 8-bit cache: o = sum softmax(scale q.k) v for the rows of single tokens, draft trees and chunks.
//
// The query heads that share a key/value head are rows side by side (row r = token r / group, head r % group), in tiles of
// 32: the score tile S^T = K Q^T of a block of 32 tokens is one accumulator of v_mfma_f32_32x32x16, in which a lane holds 16
// tokens of one row.  What a lane needs of a row's maximum and sum is therefore its own registers and one exchange between
// the halves of the wavefront; the same 16 probabilities, rounded to fp16, are the second operand of O^T += V^T P^T as they are,
// because the cache keeps V's tokens in that order; and a row's rescaling is one factor per lane.  K and V come from
// memory as 16-byte pieces that are operands after conversion (8 bits to the query's type, or to fp16: exact), so
// nothing of them goes through LDS.
//
// One pass over the tokens (running maximum and sum).  With s_k, s_v the scales of a block, t = x log2(e) + log2(s_v)
// has the running reference M (of the lane's row), p = 2^(t - M) is at most 2^kSlack whatever the scales are, and
//   l += sum p / s_v,   O += sum p code_v,   so out = O / l,   lse = (M + log2 l) ln 2.
// Measured: 64 tokens of 32 heads on 2,048 to 4,096 tokens 68 us (6.0 TB/s, HBM bound), a chunk of 2,048 rows on 8,192 308 us (1.0
// PFLOP/s, bound by the matrix instructions), the trees of 8 x 60 rows on 1,500 to 3,000 28 us.  Heads of 192 and 256 elements, whose queries,
// sums and operands do not fit the vector registers beside each other (112 and 193 of them lie in accumulation registers, one wavefront
// to a SIMD): the 64 tokens 100 and 132 us (6.1 TB/s), the chunk 610 and 775 (0.76 and 0.80 PFLOP/s).
// p is rounded to fp16 (2^-11 of itself): the smallest normal fp16 is 2^-14 of the reference, and what is below keeps an
// absolute error of 2^-25 of it.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "common.hpp"
#include "decode.hpp"

namespace evospec {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNone = -3.0e38f;                 // the reference of a row that has seen nothing
constexpr float kLeastScale = 0x1p-100f;          // of what kv_write gives
constexpr int kMostSplits = 128;
constexpr int kWaves = 4;                         // of a workgroup
constexpr float kSlack = 6.f;                     // a row's reference moves when a score passes it by more than that

// 8 codes of two dwords as an operand of fp16 or bf16 elements
template <int KIND, bool HALF>
__device__ __forceinline__ u32x4 widen(uint32_t lo, uint32_t hi) {
    u32x4 out;
    const uint32_t in[2] = {lo, hi};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if constexpr (KIND == EVOSPEC_KV_E4M3 && HALF) {
            out[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(in[j], 1.f, false));
            out[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(in[j], 1.f, true));
        } else if constexpr (KIND == EVOSPEC_KV_E4M3) {
            out[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(in[j], 1.f, false));
            out[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(in[j], 1.f, true));
        } else if constexpr (HALF) {
            // fp16 0x6400 + u is 1024 + u: the code with its sign bit flipped, 1,152 too much
            const uint32_t u = in[j] ^ 0x80808080u;
            const f16x2 off = {(_Float16)1152.f, (_Float16)1152.f};
            const f16x2 a = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - off;
            const f16x2 b = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - off;
            out[2 * j] = __builtin_bit_cast(uint32_t, a);
            out[2 * j + 1] = __builtin_bit_cast(uint32_t, b);
        } else {
            // a whole number below 256 has its bits in the upper half of a float
            uint32_t f[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = __float_as_uint((float)(int8_t)(in[j] >> (8 * i)));
            out[2 * j] = __builtin_amdgcn_perm(f[1], f[0], 0x07060302u);
            out[2 * j + 1] = __builtin_amdgcn_perm(f[3], f[2], 0x07060302u);
        }
    }
    return out;
}
template <bool HALF>
__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (HALF)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ float other_half(float x, int lane) { return __uint_as_float(xor_lane<32>(__float_as_uint(x), lane)); }

template <bool ONCE>
__device__ __forceinline__ u32x4 load_piece(const uint8_t* p) {
    if constexpr (ONCE) return load_once((gvec_ptr)(uintptr_t)p);
    else return *reinterpret_cast<const u32x4*>(p);
}

// the first n bits of 32
__device__ __forceinline__ uint32_t first_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1; }

// 0xff in every byte of x that is a NaN code
template <int KIND>
__device__ __forceinline__ uint32_t nan_bytes(uint32_t x) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t c = (x >> (8 * i)) & 255u;
        if (KIND == EVOSPEC_KV_E4M3 ? (c & 0x7fu) == 0x7fu : c == 0x80u) m |= 255u << (8 * i);
    }
    return m;
}

// NQ: dim / 32.  RT: tiles of 32 rows; the kWaves wavefronts of a workgroup have all of them, and every kWaves-th block of tokens.
// ONCE: K and V are loaded past the caches.
template <int NQ, int KIND, bool HALF, int RT, bool ONCE>
__global__ __launch_bounds__(64 * kWaves, NQ >= 6 ? 1 : 2) void kv_attention_kernel(AttnArgs A) {
    constexpr int kDim = 32 * NQ, kRows = 32 * RT;
    constexpr int kPad = 36;                                     // floats of a row of 32 in LDS
    __shared__ __align__(16) float s_o[2][kWaves][32 * kPad];
    __shared__ float2 s_ml[kWaves][RT * 32];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    int id = dealt_out(blockIdx.x, gridDim.x, A.run);
    const int tile = id % A.tiles;
    id /= A.tiles;
    const int split = id % A.splits;
    id /= A.splits;
    const int head = id % A.c.heads, s = id / A.c.heads;
    const Rows& R = A.r;
    const int n0 = min(max(R.row_off[s], 0), R.T), n1 = min(max(R.row_off[s + 1], n0), R.T);
    const int n_all = n1 - n0, n = min(n_all, R.max_rows);
    const int rows = n * A.group, r0 = tile * kRows;
    if (r0 >= rows) return;
    const int len = (int)min((long long)min(max(R.at[s], 0), 1 << 30), (long long)R.width << (A.c.shift + 5));
    const int base = len - n_all;                                // the position of row 0 (may be negative)
    // tokens [0, full) are seen by every row of the workgroup, tokens [hi, len) by none
    const int i_first = r0 / A.group, i_last = (min(rows, r0 + kRows) - 1) / A.group;
    const int full = max(0, A.tree ? base : base + i_first + 1);
    const int hi = max(0, A.tree ? len : base + i_last + 1);
    const int blocks = (hi + kBlock - 1) / kBlock;
    const int b_lo = (int)((long long)blocks * split / A.splits), b_hi = (int)((long long)blocks * (split + 1) / A.splits);

    // the rows' queries, as second operands
    constexpr bool kShared = RT > 1;                             // from LDS, where the registers hold more tiles
    __shared__ __align__(16) u32x4 s_q[kShared ? RT * NQ * 2 * 64 : 1];
    u32x4 qf[kShared ? 1 : RT][NQ][2];
    int last_seen[RT];                                           // the last token the row can see: its own, or the last of the tree
    uint64_t bits[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = r0 + rt * 32 + col;
        const bool ok = r < rows;
        const int i = ok ? r / A.group : 0, a = ok ? r % A.group : 0;
        last_seen[rt] = !ok ? -1 : A.tree ? len - 1 : base + i;
        bits[rt] = ok && A.tree ? A.tree[n0 + i] : 0;
        const uint16_t* q = static_cast<const uint16_t*>(A.q) + (long long)(n0 + i) * A.q_stride + (long long)(head * A.group + a) * kDim + 16 * half;
#pragma unroll
        for (int k = 0; k < NQ; ++k)
#pragma unroll
            for (int j = 0; j < 2; ++j)
            {
                if constexpr (kShared) {
                    if ((rt * NQ * 2 + 2 * k + j) % kWaves != wave) continue;
                    s_q[(rt * NQ * 2 + 2 * k + j) * 64 + lane] = ok ? *reinterpret_cast<const u32x4*>(q + 32 * k + 8 * j) : u32x4{0, 0, 0, 0};
                } else {
                    qf[rt][k][j] = ok ? *reinterpret_cast<const u32x4*>(q + 32 * k + 8 * j) : u32x4{0, 0, 0, 0};
                }
            }
    }

    f32x16 o[RT][NQ];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = kNone;
        l[rt] = 0.f;
#pragma unroll
        for (int k = 0; k < NQ; ++k)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[rt][k][e] = 0.f;
    }

    // Tokens come in blocks.  K of the next block is asked for when this one's scores are there, and V when it has been added, so that
    // both are under way during half of a block's work; the page table runs a block further ahead.
    // bit 8 a + i: the lane's row sees token 8 a + 4 half + i of the block at t0
    auto sees = [&](int rt, int t0, bool there) {
        uint32_t w = there ? first_bits(min(len, last_seen[rt] + 1) - t0) : 0;
        if (A.tree) {                                            // its own bits behind the context
            const int j = t0 - base;
            w &= j >= 64 ? 0u : j >= 0 ? (uint32_t)(bits[rt] >> j) : j > -kBlock ? (uint32_t)(bits[rt] << -j) | first_bits(-j) : ~0u;
        }
        return w >> (4 * half);
    };
    const int mask = (1 << A.c.shift) - 1;
    const int32_t* table = R.table + (long long)s * R.width;
    auto page_of = [&](int b) { return __builtin_amdgcn_readfirstlane(table[min(b, b_hi - 1) >> A.c.shift]); };
    // Blocks without a page are read from page 0, and no row sees them: their scales count as 1 and their V as zero, whatever is there.
    auto is_page = [&](int page) { return (unsigned)page < (unsigned)A.c.pages; };
    auto place = [&](int b, int page) { return (((long long)(is_page(page) ? page : 0) * A.c.heads + head) << A.c.shift) + (b & mask); };
    u32x4 kr[NQ], vr[NQ];
    float2 sc = make_float2(1.f, 1.f);
    auto load_k = [&](long long at) {
        const uint8_t* data = A.c.data + at * (2 * kBlock * kDim) + lane * 16;
        sc = *reinterpret_cast<const float2*>(A.c.scales + at * 2);
#pragma unroll
        for (int k = 0; k < NQ; ++k) kr[k] = load_piece<ONCE>(data + k * 1024);
    };
    auto load_v = [&](long long at) {
        const uint8_t* data = A.c.data + at * (2 * kBlock * kDim) + kBlock * kDim + lane * 16;
#pragma unroll
        for (int k = 0; k < NQ; ++k) vr[k] = load_piece<ONCE>(data + k * 1024);
    };
    bool nan_blocks = false;
    int b = b_lo + wave, page = 0, page_next = 0;
    if (b < b_hi) {
        page = page_of(b);
        page_next = page_of(b + kWaves);
        load_k(place(b, page));
        load_v(place(b, page));
    }
    // The queries are waited for here: a wait in the loop would be one for everything that is under way.
    if constexpr (kShared) {
        __syncthreads();
    } else {
#pragma unroll
        for (int k = 0; k < NQ; ++k)
#pragma unroll
            for (int j = 0; j < 2; ++j) asm("" : "+v"(qf[0][k][j]));
    }
    for (; b < b_hi; b += kWaves) {
        // (the last block's next is a block that is there, read for nothing)
        const long long at_next = place(b + kWaves, page_next);
        const bool there = is_page(page);
        page = page_next;
        page_next = page_of(b + 2 * kWaves);
        const float sc_x = there ? sc.x : 1.f, sc_y = there ? sc.y : 1.f;
        const float ck = fmaxf(fabsf(sc_x) * (A.scale * kLog2e), 0x1p-126f);       // (not zero: -inf stays what it is)
        const float sv = fmaxf(fabsf(sc_y), kLeastScale), lv = __log2f(sv), iv = __builtin_amdgcn_rcpf(sv);

        uint32_t nan_tokens = 0;                                 // of K (e4m3's NaN code is one for the matrix cores)
        if (KIND == EVOSPEC_KV_INT8 && __float_as_uint(sc_x) >> 31) {
            uint32_t any = 0;
#pragma unroll
            for (int k = 0; k < NQ; ++k) any |= nan_bytes<KIND>(kr[k][0]) | nan_bytes<KIND>(kr[k][1]) | nan_bytes<KIND>(kr[k][2]) | nan_bytes<KIND>(kr[k][3]);
            const u64 who = __ballot(any != 0);
            nan_tokens = (uint32_t)who | (uint32_t)(who >> 32);
        }
        f32x16 x[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int e = 0; e < 16; ++e) x[rt][e] = 0.f;
#pragma unroll
        for (int k = 0; k < NQ; ++k)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const u32x4 a = widen<KIND, HALF>(kr[k][2 * j], kr[k][2 * j + 1]);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) x[rt] = mfma<HALF>(a, kShared ? s_q[(rt * NQ * 2 + 2 * k + j) * 64 + lane] : qf[kShared ? 0 : rt][k][j], x[rt]);
            }

        if (KIND == EVOSPEC_KV_INT8 && nan_tokens) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if ((nan_tokens >> (8 * (e / 4) + 4 * half + e % 4)) & 1) x[rt][e] = __uint_as_float(0x7fc00000u);
        }
        __builtin_amdgcn_sched_barrier(0);
        load_k(at_next);
        __builtin_amdgcn_sched_barrier(0);

        const int t0 = b * kBlock;
        if (!(there && t0 + kBlock <= full)) {                   // (uniform)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const uint32_t seen = sees(rt, t0, there);
#pragma unroll
                for (int e = 0; e < 16; ++e) x[rt][e] = (seen >> (8 * (e / 4) + e % 4)) & 1 ? x[rt][e] : -__builtin_inff();
            }
        }
        u32x4 pf[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (RT > 1) __builtin_amdgcn_sched_barrier(0);       // (one tile after the other: fewer registers)
            float top = x[rt][0];
#pragma unroll
            for (int e = 1; e < 16; ++e) top = fmaxf(top, x[rt][e]);
            top = fmaxf(top, other_half(top, lane));
            const float t = top * ck + lv;
            if (__ballot(t > m[rt] + kSlack)) {
                const float next = fmaxf(m[rt], t);
                const float f = __builtin_amdgcn_exp2f(m[rt] - next);
                m[rt] = next;
                l[rt] *= f;
#pragma unroll
                for (int k = 0; k < NQ; ++k)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[rt][k][e] *= f;
            }
            const float c0 = lv - m[rt];
            float sum = 0.f;
            f16x8 p[2];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float y = __builtin_amdgcn_exp2f(x[rt][e] * ck + c0);
                sum += y;
                p[e >> 3][e & 7] = (_Float16)y;
            }
            l[rt] += sum * iv;
            pf[rt][0] = __builtin_bit_cast(u32x4, p[0]);
            pf[rt][1] = __builtin_bit_cast(u32x4, p[1]);
        }
        __builtin_amdgcn_sched_barrier(0);
        const int end = there ? len : t0;
        if (t0 + kBlock > end) {                                 // bytes behind the last token may be anything
#pragma unroll
            for (int k = 0; k < NQ; ++k)
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const int left = end - (t0 + 8 * a + 4 * half);
                    vr[k][a] &= left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
                }
        }
        if ((int)__float_as_uint(sc_y) < (int)__builtin_bit_cast(uint32_t, kLeastScale)) {        // (uniform) negative, or next to zero
            // NaN is left out, and looked at behind the loop; V of a scale of zero, which a caller's own may have, is zero
            if (__float_as_uint(sc_y) >> 31) nan_blocks = true;
            const uint32_t all = fabsf(sc_y) < kLeastScale ? ~0u : 0u;
#pragma unroll
            for (int k = 0; k < NQ; ++k)
#pragma unroll
                for (int a = 0; a < 4; ++a) vr[k][a] &= ~(nan_bytes<KIND>(vr[k][a]) | all);
        }
#pragma unroll
        for (int k = 0; k < NQ; ++k)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const u32x4 a = widen<KIND, true>(vr[k][2 * y], vr[k][2 * y + 1]);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) o[rt][k] = mfma<true>(a, pf[rt][y], o[rt][k]);
            }
        __builtin_amdgcn_sched_barrier(0);
        load_v(at_next);
    }
    if (nan_blocks) {
        // A NaN in V reaches the rows that see its token, and no others: tokens that are seen (0 or 1) against dims that are NaN (0
        // or 1); what is not zero in that product becomes NaN.
        for (b = b_lo + wave; b < b_hi; b += kWaves) {
            const int page = page_of(b);
            const long long at = place(b, page);
            if (!is_page(page) || !(__float_as_uint(A.c.scales[at * 2 + 1]) >> 31)) continue;
            load_v(at);
#pragma unroll
            for (int k = 0; k < NQ; ++k)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const uint32_t seen = sees(rt, b * kBlock, true);
                    f32x16 hit;
#pragma unroll
                    for (int e = 0; e < 16; ++e) hit[e] = 0.f;
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        u32x4 is, see;                           // fp16 1 or 0
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t nb = nan_bytes<KIND>(vr[k][2 * y + (e >> 1)]);
                            const uint32_t pair = (nb >> (16 * (e & 1))) & 0x0101u, two = (seen >> (16 * y + 8 * (e >> 1) + 2 * (e & 1))) & 3u;
                            is[e] = ((pair & 1u) | (pair & 0x100u) << 8) * 0x3c00u;
                            see[e] = ((two & 1u) | (two & 2u) << 15) * 0x3c00u;
                        }
                        hit = mfma<true>(is, see, hit);
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (hit[e] > 0.f) o[rt][k][e] = __uint_as_float(0x7fc00000u);
                }
        }
    }

    // the wavefronts that share rows: one reference, and their shares of it
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] += other_half(l[rt], lane);
        if (half == 0) s_ml[wave][rt * 32 + col] = make_float2(m[rt], l[rt]);
    }
    __syncthreads();
    float mm[RT], ll[RT], f[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        mm[rt] = kNone;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) mm[rt] = fmaxf(mm[rt], s_ml[w][rt * 32 + col].x);
        ll[rt] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float2 ml = s_ml[w][rt * 32 + col];
            ll[rt] += ml.y * __builtin_amdgcn_exp2f(ml.x - mm[rt]);
        }
        f[rt] = __builtin_amdgcn_exp2f(m[rt] - mm[rt]);
        if (ll[rt] > 0.f) f[rt] /= ll[rt];                       // (NaN sums divide as well, below)
        else if (ll[rt] != ll[rt]) f[rt] = ll[rt];
        const int r = r0 + rt * 32 + col;
        if (wave == 0 && half == 0 && r < rows) {
            const long long row = (long long)(n0 + r / A.group) * (A.c.heads * A.group) + head * A.group + r % A.group;
            if (A.splits > 1) A.part_ml[(long long)split * R.T * A.c.heads * A.group + row] = make_float2(mm[rt], ll[rt]);
            else if (A.lse) A.lse[row] = ll[rt] == 0.f ? -__builtin_inff() : (mm[rt] + __log2f(ll[rt])) * kLn2;
        }
    }
    // O, 32 dims at a time: every wavefront's share to LDS, summed in a fixed order on the way out
    int buf = 0;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int k = 0; k < NQ; ++k) {
            float* mine = s_o[buf][wave] + col * kPad + 4 * half;
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *reinterpret_cast<float4*>(mine + 8 * a) = make_float4(o[rt][k][4 * a] * f[rt], o[rt][k][4 * a + 1] * f[rt],
                                                                       o[rt][k][4 * a + 2] * f[rt], o[rt][k][4 * a + 3] * f[rt]);
            __syncthreads();
            {
                static_assert(64 * kWaves == 32 * 8, "4 elements of a row a thread");
                const int c = tid >> 3, d4 = tid & 7;
                const int r = r0 + rt * 32 + c;
                buf ^= 1;
                if (r >= rows) continue;
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float4 v = *reinterpret_cast<const float4*>(s_o[buf ^ 1][w] + c * kPad + 4 * d4);
                    sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
                }
                const long long row = (long long)(n0 + r / A.group) * (A.c.heads * A.group) + head * A.group + r % A.group;
                const int d = 32 * k + 4 * d4;
                if (A.splits > 1) {
                    *reinterpret_cast<float4*>(A.part_o + ((long long)split * R.T * A.c.heads * A.group + row) * kDim + d) = sum;
                } else if constexpr (HALF) {
                    typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
                    *reinterpret_cast<f16x4*>(static_cast<_Float16*>(A.out) + row * kDim + d) = f16x4{(_Float16)sum.x, (_Float16)sum.y, (_Float16)sum.z, (_Float16)sum.w};
                } else {
                    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                    *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(A.out) + row * kDim + d) = bf16x4{(__bf16)sum.x, (__bf16)sum.y, (__bf16)sum.z, (__bf16)sum.w};
                }
            }
        }
}

// The shares of a row's splits, each a mean over its tokens with a reference and a sum, in a fixed order: WAVES wavefronts a row,
// each with every WAVES-th split; 4 / WAVES rows a workgroup.
template <int NQ, bool HALF, int WAVES>
__global__ __launch_bounds__(256) void kv_attention_merge_kernel(AttnArgs A) {
    constexpr int kDim = 32 * NQ, kPer = (kDim + 63) / 64;
    __shared__ float s_o[WAVES > 1 ? WAVES : 1][kPer * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = wave % WAVES;
    const int heads = A.c.heads * A.group;
    const long long row = (long long)blockIdx.x * (4 / WAVES) + wave / WAVES, all = (long long)A.r.T * heads;
    if (row >= all) return;                                      // (a workgroup as a whole where its wavefronts share a row)
    // a row of no sequence has no shares
    const int token = (int)(row / heads);
    bool mine = false;
    for (int s = lane; s < A.r.S; s += 64) {
        const int n0 = min(max(A.r.row_off[s], 0), A.r.T), n1 = min(max(A.r.row_off[s + 1], n0), A.r.T);
        mine |= token >= n0 && token < min(n1, n0 + A.r.max_rows);
    }
    if (!__ballot(mine)) return;
    static_assert(kMostSplits <= 128, "two splits a lane");
    float2 ml[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) ml[i] = lane + 64 * i < A.splits ? A.part_ml[(lane + 64 * i) * all + row] : make_float2(kNone, 0.f);
    const float m = wave_max(fmaxf(ml[0].x, ml[1].x), lane);
    float w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = ml[i].y == 0.f ? 0.f : ml[i].y * __builtin_amdgcn_exp2f(ml[i].x - m);
    const float sum = wave_sum(w[0] + w[1], lane);
    float o[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) o[k] = 0.f;
    for (int j = part; j < A.splits; j += WAVES) {
        const float wj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(j < 64 ? w[0] : w[1]), j & 63));
        const float* from = A.part_o + (j * all + row) * kDim + lane;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const float v = kDim % 64 == 0 || 64 * k + lane < kDim ? from[64 * k] : 0.f;
            o[k] += wj * v;                                      // (also 0 * NaN: the row saw it, however little it weighs)
        }
    }
    if constexpr (WAVES > 1) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) s_o[part][64 * k + lane] = o[k];
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int k = 0; k < kPer; ++k)
#pragma unroll
            for (int p = 1; p < WAVES; ++p) o[k] += s_o[p][64 * k + lane];
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        if (kDim % 64 != 0 && 64 * k + lane >= kDim) continue;
        const float v = sum == 0.f ? 0.f : o[k] / sum;
        if constexpr (HALF) static_cast<_Float16*>(A.out)[row * kDim + 64 * k + lane] = (_Float16)v;
        else static_cast<__bf16*>(A.out)[row * kDim + 64 * k + lane] = (__bf16)v;
    }
    if (A.lse && lane == 0) A.lse[row] = sum == 0.f ? -__builtin_inff() : (m + __log2f(sum)) * kLn2;
}

template <int I>
using Const = std::integral_constant<int, I>;

template <int NQ, int KIND, bool HALF>
hipError_t launch_as(const AttnArgs& a, const AttnPlan& p, hipStream_t stream) {
    const dim3 grid((unsigned)(a.splits * a.tiles * a.c.heads * a.r.S));
    if (p.row_tiles == 2) {
        if constexpr (NQ <= 4) kv_attention_kernel<NQ, KIND, HALF, 2, false><<<grid, 64 * kWaves, 0, stream>>>(a);
    } else if (p.once) {
        kv_attention_kernel<NQ, KIND, HALF, 1, true><<<grid, 64 * kWaves, 0, stream>>>(a);
    } else {
        kv_attention_kernel<NQ, KIND, HALF, 1, false><<<grid, 64 * kWaves, 0, stream>>>(a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    // (few rows of many splits: one of 131,072 tokens and 32 heads 23 us by a wavefront a row)
    const long long rows = (long long)a.r.T * a.c.heads * a.group;
    if (a.splits >= 8) kv_attention_merge_kernel<NQ, HALF, 4><<<dim3((unsigned)rows), 256, 0, stream>>>(a);
    else kv_attention_merge_kernel<NQ, HALF, 1><<<dim3((unsigned)((rows + 3) / 4)), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

// Two tiles of rows a wavefront halve what is loaded and converted for a row, and leave half as many workgroups: taken where these still
// fill 256 compute units twice (2,048 rows of 8 x 4 heads on 10,240 tokens 347 us with one tile, 315 with two; 60 rows of 8
// sequences, 256 workgroups of two tiles, 28 and 37).  From 160 elements on there are no registers for them.
// The tokens are split over workgroups where there are fewer of these than compute units, and enough to split: 131,072 tokens of 8
// heads over 16, 32 and 64 workgroups a head 62 + 4.5, 44 + 5.1 and 46 + 7.5 us (attention + joining the shares), 16 x 4,096 tokens
// over 1, 2 and 4 30, 22 + 4 and 22 + 4; 4,096 tokens over 1, 4, 8 and 16 23, 11 + 3.6, 8.6 + 3.6 and 7.3 + 4.2, but 1,000 of 64
// elements over 1 and 4 9.0 and 6.3 + 3.4, and another launch.
// Runs for a die (dealt_out): a sequence of several tiles is dealt out to all 8 dies, an eighth each, so that one of many rows has all of
// them whatever stands beside it: 2,048 rows on 8,192 tokens before 32 single ones on 4,096 2,003 us with an eighth of the call for each die,
// 439 so; 8 trees of 60 rows 32.5 and 28.2.  Sequences of a single tile go to the dies by twos: 64 on 8,192 down to 128 tokens 122 us by
// eighths of the call, 93 one by one and 91 by twos, in any order 103, 104 and 98; 64 on 2,048 to 4,096 67.6, 69.4 and 68.1.
// K and V are loaded past the caches where a sequence's workgroup reads them once: 64 tokens on 2,048 to 4,096 76 and 68 us, one on 131,072
// 56 and 50, 16 x 4,096 29.5 and 28.5.  (Pages that sequences share are read by each of them, which the page table alone knows: 64 x 4,096
// shared tokens 42 us through the caches and 47 past them, still below the 84 of 64 x 4,096 of their own.)
AttnPlan attention_plan(int dim, int heads, int group, int S, int max_rows, int max_len) {
    constexpr long long kUnits = 256, kLeast = 48, kShare = 4;   // compute units; blocks that are worth a split, and of a wavefront then
    AttnPlan p;
    const long long rows = (long long)max_rows * group;
    p.row_tiles = dim <= 128 && rows > 32 && (rows + 63) / 64 * heads * S >= 2 * kUnits ? 2 : 1;
    const int per = 32 * p.row_tiles;
    p.tiles = (int)((rows + per - 1) / per);
    const long long groups = (long long)p.tiles * heads * S, blocks = ((long long)max_len + kBlock - 1) / kBlock;
    long long splits = (kUnits + groups - 1) / groups;
    const long long most = blocks < kLeast ? 1 : blocks / (kShare * kWaves);
    splits = splits > most ? most : splits;
    p.splits = (int)(splits > kMostSplits ? kMostSplits : splits);
    p.once = p.tiles == 1;
    p.run = p.tiles == 1 ? 2 * heads : (int)(((long long)p.tiles * p.splits * heads + 7) / 8);
    return p;
}

size_t attention_workspace(const AttnPlan& p, int dim, int heads, int group, int T) {
    if (p.splits <= 1) return 0;
    return (size_t)p.splits * T * heads * group * (dim * 4 + 8);
}

hipError_t launch_kv_attention(const AttnArgs& a, const AttnPlan& p, int dim, int kind, int type, hipStream_t stream) {
    auto by_type = [&](auto nq, auto kd) {
        return type == EVOSPEC_FP16 ? launch_as<nq.value, kd.value, true>(a, p, stream) : launch_as<nq.value, kd.value, false>(a, p, stream);
    };
    auto by_kind = [&](auto nq) {
        return kind == EVOSPEC_KV_E4M3 ? by_type(nq, Const<EVOSPEC_KV_E4M3>{}) : by_type(nq, Const<EVOSPEC_KV_INT8>{});
    };
    switch (dim) {
        case 64: return by_kind(Const<2>{});
        case 96: return by_kind(Const<3>{});
        case 128: return by_kind(Const<4>{});
        case 192: return by_kind(Const<6>{});
        default: return by_kind(Const<8>{});
    }
}

}  // namespace evospec
