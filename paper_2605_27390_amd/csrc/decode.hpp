// The 8-bit key/value cache and the sampler: layout, host-side arguments and launchers (no HIP code in the types).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "evospec_decode.h"

namespace evospec {

constexpr int kBlock = EVOSPEC_KV_BLOCK;      // tokens that share a scale

// A cache as the kernels take it.
struct Cache {
    uint8_t* data;
    float* scales;
    int pages, heads;
    int shift;                                // log2 of the blocks of a page
};

// The rows of a call: who they belong to.
struct Rows {
    const int32_t* table;
    int width;
    const int32_t* at;                        // starts (write, read) or lens (attention)
    const int32_t* row_off;
    int S, T, max_rows;
};

// Blocks that rows of one sequence can touch, wherever they start.
inline int touched_blocks(int max_rows) { return (max_rows + kBlock - 2) / kBlock + 1; }

hipError_t launch_kv_write(const Cache& c, int dim, int kind, const void* k, long long k_stride, const void* v, long long v_stride,
                           int type, const Rows& r, hipStream_t stream);
hipError_t launch_kv_read(const Cache& c, int dim, int kind, const Rows& r, int type, void* out_k, void* out_v, hipStream_t stream);

// Workgroups go round the 8 dies in turn.  Runs of `run` neighbours, which read the same tokens, go to one die, for its cache: a run for each die
// in a round, and the next round three dies on, so that what repeats every 8 runs does not meet one die.  What is left over is dealt out in
// eighths.  The task of workgroup b of n.
__host__ __device__ inline int dealt_out(int b, int n, int run) {
    const int whole = n / (8 * run) * (8 * run);
    if (b < whole) {
        const int place = b / 8, round = place / run;
        return (round * 8 + ((b + 3 * round) & 7)) * run + place % run;
    }
    const int left = n - whole, die = (b - whole) & 7, most = left / 8, rest = left & 7;
    return whole + die * most + (die < rest ? die : rest) + (b - whole) / 8;
}

// How an attention call is laid out.
struct AttnPlan {
    int row_tiles;                            // tiles of 32 rows of a workgroup
    int tiles;                                // workgroups over the rows of a sequence and head
    int splits;                               // workgroups over its tokens
    bool once;                                // K and V past the caches
    int run;                                  // workgroups in a row for one die
};
AttnPlan attention_plan(int dim, int heads, int group, int S, int max_rows, int max_len);
size_t attention_workspace(const AttnPlan& p, int dim, int heads, int group, int T);

struct AttnArgs {
    Cache c;
    Rows r;
    const void* q;
    long long q_stride;
    int group;
    const uint64_t* tree;
    float scale;
    void* out;
    float* lse;
    float* part_o;                            // [splits][T * heads * group][dim], of splits > 1
    float2* part_ml;                          // [splits][T * heads * group]: reference and sum
    int splits, tiles, run;
};
hipError_t launch_kv_attention(const AttnArgs& a, const AttnPlan& p, int dim, int kind, int type, hipStream_t stream);

struct SampleArgs {
    const void* logits;
    long long stride;
    int M, V;
    const float* u;
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    const int32_t* ids;
    int32_t* out_ids;
    float* out_logprob;
};
int sample_slices(int V);                     // workgroups of 1,024 threads of a row
size_t sample_workspace(int M, int V);
hipError_t launch_sample(const SampleArgs& a, int type, void* workspace, hipStream_t stream);

}  // namespace evospec
