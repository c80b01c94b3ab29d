// C ABI of the 8-bit cache, the attention over it and the sampler (declared in include/evospec_decode.h): argument
// validation on the host and the launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "decode.hpp"
#include "launch.hpp"

using namespace evospec;

namespace {

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
size_t type_bytes(int type) { return type == EVOSPEC_FP32 ? 4 : 2; }
int failed(hipError_t e) { return e == hipSuccess ? EVOSPEC_OK : record_hip_error(e); }

int check_cache(const evospec_kv_cache* c) {
    if (!c) return EVOSPEC_NULL_POINTER;
    if (c->kind != EVOSPEC_KV_E4M3 && c->kind != EVOSPEC_KV_INT8) return EVOSPEC_BAD_TYPE;
    if (c->pages < 1 || c->heads < 1 || c->heads > 1024) return EVOSPEC_BAD_SHAPE;
    if (c->page != 32 && c->page != 64 && c->page != 128 && c->page != 256) return EVOSPEC_BAD_SHAPE;
    if (c->dim != 64 && c->dim != 96 && c->dim != 128 && c->dim != 192 && c->dim != 256) return EVOSPEC_BAD_SHAPE;
    return EVOSPEC_OK;
}
int check_buffers(const evospec_kv_cache* c) {
    if (!c->data || !c->scales) return EVOSPEC_NULL_POINTER;
    return aligned(c->data, 16) && aligned(c->scales, 8) ? EVOSPEC_OK : EVOSPEC_MISALIGNED;
}
Cache cache_of(const evospec_kv_cache* c) {
    int shift = 0;
    while ((kBlock << shift) < c->page) ++shift;
    return Cache{static_cast<uint8_t*>(c->data), c->scales, c->pages, c->heads, shift};
}
// Rows of at least `least` elements that lie `stride` apart and start on 16 bytes.
int check_stride(long long stride, long long least, int type) {
    if (stride < least) return EVOSPEC_BAD_SHAPE;
    return stride * (long long)type_bytes(type) % 16 == 0 ? EVOSPEC_OK : EVOSPEC_MISALIGNED;
}
int check_rows(int width, int S, int max_rows, int T) {
    return width < 1 || S < 0 || max_rows < 0 || T < 0 || max_rows > (1 << 28) || width > (1 << 24) ? EVOSPEC_BAD_SHAPE : EVOSPEC_OK;
}
bool grid_fits(long long a, long long b, long long c) {
    const long long most = (1ll << 24) - 1024;                   // workgroups: a launch takes fewer than 2^32 threads, of 256 here
    return a * b <= most && a * b * c <= most;
}

bool sample_fits(int M, int V) { return M >= 0 && V >= 1 && V <= (1 << 20) && (long long)M * sample_slices(V) < (1 << 22); }

}  // namespace

extern "C" {

int evospec_kv_cache_bytes(const evospec_kv_cache* cache, size_t* out_data_bytes, size_t* out_scale_bytes) {
    if (!out_data_bytes || !out_scale_bytes) return EVOSPEC_NULL_POINTER;
    const int rc = check_cache(cache);
    if (rc) return rc;
    const size_t blocks = (size_t)cache->pages * cache->heads * (cache->page / kBlock);
    *out_data_bytes = blocks * 2 * kBlock * cache->dim;
    *out_scale_bytes = blocks * 2 * sizeof(float);
    return EVOSPEC_OK;
}

int evospec_kv_write(const evospec_kv_cache* cache, const void* k, long long k_stride, const void* v, long long v_stride, int type,
                     int T, const int32_t* page_table, int width, const int32_t* starts, const int32_t* row_off, int S, int max_rows,
                     void* stream) {
    int rc = check_cache(cache);
    if (rc) return rc;
    if (type < EVOSPEC_BF16 || type > EVOSPEC_FP32) return EVOSPEC_BAD_TYPE;
    if ((rc = check_rows(width, S, max_rows, T))) return rc;
    const long long least = (long long)cache->heads * cache->dim;
    if ((rc = check_stride(k_stride, least, type)) || (rc = check_stride(v_stride, least, type))) return rc;
    if (!grid_fits(touched_blocks(max_rows), cache->heads, S)) return EVOSPEC_BAD_SHAPE;
    if (S == 0 || T == 0 || max_rows == 0) return EVOSPEC_OK;
    if (!k || !v || !page_table || !starts || !row_off) return EVOSPEC_NULL_POINTER;
    if ((rc = check_buffers(cache))) return rc;
    if (!aligned(k, 16) || !aligned(v, 16)) return EVOSPEC_MISALIGNED;
    const Rows r{page_table, width, starts, row_off, S, T, max_rows < T ? max_rows : T};
    return failed(launch_kv_write(cache_of(cache), cache->dim, cache->kind, k, k_stride, v, v_stride, type, r, static_cast<hipStream_t>(stream)));
}

int evospec_kv_read(const evospec_kv_cache* cache, const int32_t* page_table, int width, const int32_t* starts, const int32_t* row_off,
                    int S, int max_rows, int T, int type, void* out_k, void* out_v, void* stream) {
    int rc = check_cache(cache);
    if (rc) return rc;
    if (type < EVOSPEC_BF16 || type > EVOSPEC_FP32) return EVOSPEC_BAD_TYPE;
    if ((rc = check_rows(width, S, max_rows, T))) return rc;
    if (!grid_fits(touched_blocks(max_rows), cache->heads, S)) return EVOSPEC_BAD_SHAPE;
    if (S == 0 || T == 0 || max_rows == 0) return EVOSPEC_OK;
    if (!out_k || !out_v || !page_table || !starts || !row_off) return EVOSPEC_NULL_POINTER;
    if ((rc = check_buffers(cache))) return rc;
    if (!aligned(out_k, 16) || !aligned(out_v, 16)) return EVOSPEC_MISALIGNED;
    const Rows r{page_table, width, starts, row_off, S, T, max_rows < T ? max_rows : T};
    return failed(launch_kv_read(cache_of(cache), cache->dim, cache->kind, r, type, out_k, out_v, static_cast<hipStream_t>(stream)));
}

static int check_attention(const evospec_kv_cache* cache, int group, int S, int T, int max_rows, int max_len) {
    int rc = check_cache(cache);
    if (rc) return rc;
    if (group < 1 || group > 1024 || max_len < 0 || max_len > (1 << 30)) return EVOSPEC_BAD_SHAPE;
    if ((rc = check_rows(1, S, max_rows, T))) return rc;
    if ((long long)max_rows * group > (1 << 30) || (long long)T * cache->heads > (1 << 30) / group) return EVOSPEC_BAD_SHAPE;
    // (splits come to no more than 256 workgroups beyond the tiles)
    if (!grid_fits(((long long)max_rows * group + 31) / 32, cache->heads, S)) return EVOSPEC_BAD_SHAPE;
    if (S == 0 || T == 0 || max_rows == 0) return EVOSPEC_OK;    // (nothing to plan)
    const AttnPlan p = attention_plan(cache->dim, cache->heads, group, S, max_rows, max_len);
    return p.splits == 1 || grid_fits(T, cache->heads, group) ? EVOSPEC_OK : EVOSPEC_BAD_SHAPE;      // rows of the merge
}

int evospec_kv_attention_workspace_bytes(const evospec_kv_cache* cache, int group, int S, int T, int max_rows, int max_len,
                                         size_t* out_bytes) {
    if (!out_bytes) return EVOSPEC_NULL_POINTER;
    const int rc = check_attention(cache, group, S, T, max_rows, max_len);
    if (rc) return rc;
    *out_bytes = 0;
    if (S > 0 && T > 0 && max_rows > 0) *out_bytes = attention_workspace(attention_plan(cache->dim, cache->heads, group, S, max_rows, max_len), cache->dim, cache->heads, group, T);
    return EVOSPEC_OK;
}

int evospec_kv_attention(const evospec_kv_cache* cache, const void* q, long long q_stride, int type, int T, int group,
                         const int32_t* page_table, int width, const int32_t* lens, const int32_t* row_off, int S, int max_rows,
                         int max_len, const uint64_t* tree, float scale, void* out, float* lse, void* workspace,
                         size_t workspace_bytes, void* stream) {
    int rc = check_attention(cache, group, S, T, max_rows, max_len);
    if (rc) return rc;
    if (type != EVOSPEC_BF16 && type != EVOSPEC_FP16) return EVOSPEC_BAD_TYPE;
    if ((rc = check_rows(width, S, max_rows, T))) return rc;
    if (!(scale > 0.f) || !std::isfinite(scale) || (tree && max_rows > 64)) return EVOSPEC_BAD_SHAPE;
    if ((rc = check_stride(q_stride, (long long)cache->heads * group * cache->dim, type))) return rc;
    if (S == 0 || T == 0 || max_rows == 0) return EVOSPEC_OK;
    if (!q || !page_table || !lens || !row_off || !out) return EVOSPEC_NULL_POINTER;
    if ((rc = check_buffers(cache))) return rc;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16)) return EVOSPEC_MISALIGNED;
    const AttnPlan p = attention_plan(cache->dim, cache->heads, group, S, max_rows, max_len);
    const size_t need = attention_workspace(p, cache->dim, cache->heads, group, T);
    if (need && !workspace) return EVOSPEC_NULL_POINTER;
    if (workspace_bytes < need) return EVOSPEC_WORKSPACE_TOO_SMALL;
    AttnArgs a{};
    a.c = cache_of(cache);
    a.r = Rows{page_table, width, lens, row_off, S, T, max_rows};
    a.q = q; a.q_stride = q_stride; a.group = group; a.tree = tree; a.scale = scale; a.out = out; a.lse = lse;
    a.splits = p.splits; a.tiles = p.tiles; a.run = p.run;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = need ? reinterpret_cast<float2*>(static_cast<char*>(workspace) + (size_t)p.splits * T * cache->heads * group * cache->dim * 4) : nullptr;
    return failed(launch_kv_attention(a, p, cache->dim, cache->kind, type, static_cast<hipStream_t>(stream)));
}

int evospec_sample_workspace_bytes(int M, int V, size_t* out_bytes) {
    if (!out_bytes) return EVOSPEC_NULL_POINTER;
    if (!sample_fits(M, V)) return EVOSPEC_BAD_SHAPE;
    *out_bytes = sample_workspace(M, V);
    return EVOSPEC_OK;
}

int evospec_sample(const void* logits, long long stride, int type, int M, int V, const float* u, const float* temperature,
                   const int32_t* top_k, const float* top_p, const float* min_p, const int32_t* ids, int32_t* out_ids,
                   float* out_logprob, void* workspace, size_t workspace_bytes, void* stream) {
    if (type < EVOSPEC_BF16 || type > EVOSPEC_FP32) return EVOSPEC_BAD_TYPE;
    if (!sample_fits(M, V) || stride < V) return EVOSPEC_BAD_SHAPE;
    if (M == 0) return EVOSPEC_OK;
    if (!logits || !u || !out_ids) return EVOSPEC_NULL_POINTER;
    if (!aligned(logits, type_bytes(type)) || !aligned(workspace, 16)) return EVOSPEC_MISALIGNED;
    const size_t need = sample_workspace(M, V);
    if (need && !workspace) return EVOSPEC_NULL_POINTER;
    if (workspace_bytes < need) return EVOSPEC_WORKSPACE_TOO_SMALL;
    const SampleArgs a{logits, stride, M, V, u, temperature, top_k, top_p, min_p, ids, out_ids, out_logprob};
    return failed(launch_sample(a, type, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
