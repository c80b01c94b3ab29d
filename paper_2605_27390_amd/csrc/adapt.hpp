// Adapters, the distillation loss and AdamW: host-side plans, arguments and launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "evospec_adapt.h"

namespace evospec {

// The rows of a call and whose adapter they have.
struct Requests {
    const int32_t* row_off;
    const int32_t* adapter;
    int S, T, n;                              // n adapters
};

// How the products of rows with adapters are laid out: tiles of 16 rows, or 32, the columns of the second product in `slices`.
struct LoraPlan {
    bool wide;                                // 32
    int tiles;                                // workgroups for the rows: every request may begin a tile of its own
    int slices;
    bool deep;                                // a compute unit has one workgroup at most
    bool once;                                // y past the caches
};
LoraPlan lora_plan(int S, int T, int r, int d_down, int d_up);

struct LoraArgs {                             // h = x w_down^T (times factor, backward), y += factor h w_up
    Requests q;
    const void* x;
    long long x_stride;
    const void* w_down;
    int d_down;
    const float* factor;                      // [n] or NULL
    const void* w_up;
    int d_up;
    void* y;                                  // NULL: h alone
    long long y_stride;
    float* h;                                 // [r][T] or NULL
    int r;
    int slices = 1;                           // of y's columns (set by the launch)
};
// back: w_down is [n][d][r] and w_up [n][r][d], else the other way round
hipError_t launch_lora_rows(const LoraArgs& a, const LoraPlan& p, bool back, hipStream_t stream);

struct GradJob {                              // out[rank][c] (or [c][rank]) = factor * sum_rows h[rank][row] x[row][c]
    const float* h;
    const float* factor;
    const void* x;
    long long x_stride;
    int d;
    bool rank_last;                           // of the output
    float* out;                               // [n][...]
};
struct GradArgs {
    Requests q;
    GradJob job[2];
    int r, parts;                             // parts of an adapter's rows
    float* partial;                           // [parts][n r d0 + n r d1] of parts > 1
};
long long lora_grad_groups(int n, int r, int d0, int d1);      // workgroups of a part
int lora_grad_parts(int n, int r, int S, int T, int d0, int d1);
hipError_t launch_lora_grads(const GradArgs& a, hipStream_t stream);

struct KdArgs {
    const void* h;
    const void* W;
    const int32_t* support;
    const float* target;
    const float* weight;
    int E, d, V, K, splits;
    float T;
    int type;
    float* loss;
    void* dh;
    float* draft;
    float* part;                              // [E][splits][2][d] of splits > 1
    float2* part_ml;                          // [E][splits]: reference and sum
};
int kd_splits(int E, int K, int d);
hipError_t launch_kd(const KdArgs& a, hipStream_t stream);

struct AdamwArgs {
    void *m, *v;
    float* scales;
    float* master;
    float decay, rate, beta1, beta1c, beta2, beta2c, root, eps;       // 1 - lr wd, lr / (1 - beta1^t), ..., 1 / sqrt(1 - beta2^t)
    float log_beta1, log_beta2, weight_decay;                        // with a schedule
    uint32_t seed_key, t_key;
    const float* schedule;
    const float* grad_scale;
};
hipError_t launch_adamw(const evospec_adamw_tensor* tensors, int count, int param_type, int grad_type, int kind, const AdamwArgs& a,
                        hipStream_t stream);
hipError_t launch_adamw_moments(const void* m, const void* v, const float* scales, long long blocks, int type, void* out_m, void* out_v,
                                hipStream_t stream);

}  // namespace evospec
