// C ABI of the adapters, the distillation loss and AdamW (declared in include/evospec_adapt.h): argument validation on the host
// and the launches.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>

#include "adapt.hpp"
#include "launch.hpp"

using namespace evospec;

namespace {

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int failed(hipError_t e) { return e == hipSuccess ? EVOSPEC_OK : record_hip_error(e); }
size_t up_to(size_t n) { return (n + 255) & ~(size_t)255; }

int check_lora(const evospec_lora* l, int S, int T) {
    if (!l) return EVOSPEC_NULL_POINTER;
    if (l->n < 1 || l->n > 65535 || l->r < 8 || l->r % 8 || l->r > EVOSPEC_LORA_R_MAX) return EVOSPEC_BAD_SHAPE;
    if (l->d_in < 8 || l->d_in % 8 || l->d_in > (1 << 20) || l->d_out < 8 || l->d_out % 8 || l->d_out > (1 << 20)) return EVOSPEC_BAD_SHAPE;
    return S < 0 || S > (1 << 16) || T < 0 || T >= (1 << 24) ? EVOSPEC_BAD_SHAPE : EVOSPEC_OK;
}
int check_weights(const evospec_lora* l) {
    if (!l->a || !l->b) return EVOSPEC_NULL_POINTER;
    return aligned(l->a, 16) && aligned(l->b, 16) && aligned(l->scale, 4) ? EVOSPEC_OK : EVOSPEC_MISALIGNED;
}
// Rows of d elements in bf16 that lie `stride` apart.
int check_matrix(const void* p, long long stride, int d) {
    if (!p) return EVOSPEC_NULL_POINTER;
    if (stride < d || stride > (1ll << 26)) return EVOSPEC_BAD_SHAPE;
    return stride % 8 == 0 && aligned(p, 16) ? EVOSPEC_OK : EVOSPEC_MISALIGNED;
}
// (a launch takes fewer than 2^32 threads, of 512 here; more than a part of the rows only where workgroups are few)
bool grads_fit(const evospec_lora* l) { return lora_grad_groups(l->n, l->r, l->d_in, l->d_out) < (1ll << 23); }
size_t h_bytes(const evospec_lora* l, int T) { return up_to((size_t)l->r * T * sizeof(float)); }

int check_kd(int E, int K, int d) {
    return E < 0 || E >= (1 << 20) || K < 1 || K > EVOSPEC_KD_K_MAX || d < 8 || d % 8 || d > EVOSPEC_KD_D_MAX ? EVOSPEC_BAD_SHAPE : EVOSPEC_OK;
}
size_t kd_workspace(int E, int K, int d) {
    const int s = E ? kd_splits(E, K, d) : 1;
    return s == 1 ? 0 : up_to((size_t)E * s * 2 * d * sizeof(float)) + (size_t)E * s * sizeof(float2);
}

int check_tensors(const evospec_adamw_tensor* tensors, int count, long long* blocks) {
    if (count < 0) return EVOSPEC_BAD_SHAPE;
    if (count && !tensors) return EVOSPEC_NULL_POINTER;
    long long sum = 0;
    for (int i = 0; i < count; ++i) {
        const long long n = tensors[i].n;
        if (n < 0 || n > (long long)EVOSPEC_ADAMW_BLOCK << 25) return EVOSPEC_BAD_SHAPE;
        sum += (n + EVOSPEC_ADAMW_BLOCK - 1) / EVOSPEC_ADAMW_BLOCK;
    }
    *blocks = sum;
    return EVOSPEC_OK;
}

}  // namespace

extern "C" {

int evospec_lora_forward(const evospec_lora* lora, const void* x, long long x_stride, const int32_t* row_off, const int32_t* adapter,
                         int S, int T, void* y, long long y_stride, float* out_h, void* stream) {
    int rc = check_lora(lora, S, T);
    if (rc) return rc;
    if (T == 0 || (S == 0 && !out_h)) return EVOSPEC_OK;          // (without requests out_h is zeros)
    if ((rc = check_weights(lora))) return rc;
    if ((rc = check_matrix(x, x_stride, lora->d_in)) || (rc = check_matrix(y, y_stride, lora->d_out))) return rc;
    if (!row_off || (!adapter && S)) return EVOSPEC_NULL_POINTER;
    if (!aligned(out_h, 4)) return EVOSPEC_MISALIGNED;
    const LoraArgs rows{{row_off, adapter, S, T, lora->n}, x, x_stride, lora->a, lora->d_in, lora->scale, lora->b, lora->d_out, y, y_stride, out_h, lora->r};
    return failed(launch_lora_rows(rows, lora_plan(S, T, lora->r, lora->d_in, lora->d_out), false, static_cast<hipStream_t>(stream)));
}

int evospec_lora_backward_workspace_bytes(const evospec_lora* lora, int S, int T, size_t* out_bytes) {
    if (!out_bytes) return EVOSPEC_NULL_POINTER;
    const int rc = check_lora(lora, S, T);
    if (rc) return rc;
    if (!grads_fit(lora)) return EVOSPEC_BAD_SHAPE;
    *out_bytes = 0;
    if (S == 0 || T == 0) return EVOSPEC_OK;
    const int parts = lora_grad_parts(lora->n, lora->r, 1, T, lora->d_in, lora->d_out);          // (the most that fewer rows or other requests need)
    *out_bytes = 2 * h_bytes(lora, T) + (parts > 1 ? (size_t)parts * lora->n * lora->r * ((size_t)lora->d_in + lora->d_out) * sizeof(float) : 0);
    return EVOSPEC_OK;
}

int evospec_lora_backward(const evospec_lora* lora, const void* x, long long x_stride, const float* h, const void* dy, long long dy_stride,
                          const int32_t* row_off, const int32_t* adapter, int S, int T, void* dx, long long dx_stride, float* out_da,
                          float* out_db, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_lora(lora, S, T);
    if (rc) return rc;
    if (!grads_fit(lora)) return EVOSPEC_BAD_SHAPE;
    const bool rows = S > 0 && T > 0;                            // (without any the gradients are zeros)
    if ((rc = check_weights(lora))) return rc;
    if (rows && ((rc = check_matrix(x, x_stride, lora->d_in)) || (rc = check_matrix(dy, dy_stride, lora->d_out)) ||
                 (dx && (rc = check_matrix(dx, dx_stride, lora->d_in)))))
        return rc;
    if (!out_da || !out_db || (rows && (!row_off || !adapter || !workspace))) return EVOSPEC_NULL_POINTER;
    if (!aligned(out_da, 16) || !aligned(out_db, 16) || !aligned(workspace, 16) || !aligned(h, 4)) return EVOSPEC_MISALIGNED;
    size_t need = 0;
    evospec_lora_backward_workspace_bytes(lora, S, T, &need);
    if (workspace_bytes < need) return EVOSPEC_WORKSPACE_TOO_SMALL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    Requests q{row_off, adapter, S, T, lora->n};
    if (!rows) q.S = 0;
    char* ws = static_cast<char*>(workspace);
    float* g = reinterpret_cast<float*>(ws);
    float* again = reinterpret_cast<float*>(ws + (rows ? h_bytes(lora, T) : 0));
    if (rows) {
        const LoraPlan p = lora_plan(S, T, lora->r, lora->d_out, lora->d_in);
        if (!h) {
            const LoraArgs down{q, x, x_stride, lora->a, lora->d_in, nullptr, nullptr, 0, nullptr, 0, again, lora->r};
            if ((rc = failed(launch_lora_rows(down, p, false, st)))) return rc;
        }
        const LoraArgs back{q, dy, dy_stride, lora->b, lora->d_out, lora->scale, lora->a, lora->d_in, dx, dx_stride, g, lora->r};
        if ((rc = failed(launch_lora_rows(back, p, true, st)))) return rc;
    }
    GradArgs a{};
    a.q = q;
    a.job[0] = GradJob{g, nullptr, x, x_stride, lora->d_in, false, out_da};
    a.job[1] = GradJob{h ? h : again, lora->scale, dy, dy_stride, lora->d_out, true, out_db};
    a.r = lora->r;
    a.parts = rows ? lora_grad_parts(lora->n, lora->r, S, T, lora->d_in, lora->d_out) : 1;
    a.partial = reinterpret_cast<float*>(ws + (rows ? 2 * h_bytes(lora, T) : 0));
    return failed(launch_lora_grads(a, st));
}

int evospec_kd_loss_workspace_bytes(int E, int K, int d, size_t* out_bytes) {
    if (!out_bytes) return EVOSPEC_NULL_POINTER;
    const int rc = check_kd(E, K, d);
    if (rc) return rc;
    *out_bytes = kd_workspace(E, K, d);
    return EVOSPEC_OK;
}

int evospec_kd_loss(const void* h, int E, int d, const void* W_lm, int V, const int32_t* support, const float* target, const float* weight,
                    int K, float T, int type, float* out_loss, void* out_dh, float* out_draft, void* workspace, size_t workspace_bytes,
                    void* stream) {
    const int rc = check_kd(E, K, d);
    if (rc) return rc;
    if (type != EVOSPEC_BF16 && type != EVOSPEC_FP32) return EVOSPEC_BAD_TYPE;
    if (V < 1 || !(T >= FLT_MIN) || !std::isfinite(T)) return EVOSPEC_BAD_SHAPE;        // (1 / T is finite)
    if (E == 0) return EVOSPEC_OK;
    if (!h || !W_lm || !support || !target || !out_loss || !out_dh || !out_draft) return EVOSPEC_NULL_POINTER;
    if (!aligned(h, 16) || !aligned(W_lm, 16) || !aligned(out_dh, 16) || !aligned(workspace, 16)) return EVOSPEC_MISALIGNED;
    const size_t need = kd_workspace(E, K, d);
    if (need && !workspace) return EVOSPEC_NULL_POINTER;
    if (workspace_bytes < need) return EVOSPEC_WORKSPACE_TOO_SMALL;
    KdArgs a{};
    a.h = h; a.W = W_lm; a.support = support; a.target = target; a.weight = weight;
    a.E = E; a.d = d; a.V = V; a.K = K; a.splits = kd_splits(E, K, d); a.T = T; a.type = type;
    a.loss = out_loss; a.dh = out_dh; a.draft = out_draft;
    a.part = static_cast<float*>(workspace);
    if (need) a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + up_to((size_t)E * a.splits * 2 * d * sizeof(float)));
    return failed(launch_kd(a, static_cast<hipStream_t>(stream)));
}

int evospec_adamw_blocks(const evospec_adamw_tensor* tensors, int count, long long* out_blocks) {
    if (!out_blocks) return EVOSPEC_NULL_POINTER;
    return check_tensors(tensors, count, out_blocks);
}

int evospec_adamw_step(const evospec_adamw_tensor* tensors, int count, int param_type, int grad_type, int kind, void* m, void* v,
                       float* scales, float* master, double lr, double beta1, double beta2, double eps, double weight_decay, long long t,
                       uint32_t seed, const float* schedule, const float* grad_scale, void* stream) {
    long long blocks = 0;
    const int rc = check_tensors(tensors, count, &blocks);
    if (rc) return rc;
    if (param_type < EVOSPEC_BF16 || param_type > EVOSPEC_FP32 || (grad_type != param_type && grad_type != EVOSPEC_FP32) ||
        (kind != EVOSPEC_MOMENTS_FP32 && kind != EVOSPEC_MOMENTS_8BIT))
        return EVOSPEC_BAD_TYPE;
    // (eps as the kernel has it: below the normal numbers its reciprocal is infinite, and an update of nothing, 0 x infinity, NaN)
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !((float)eps >= FLT_MIN) || !std::isfinite((float)eps) || !std::isfinite(lr) ||
        !std::isfinite(weight_decay) || t < 1)
        return EVOSPEC_BAD_SHAPE;
    if (blocks == 0) return EVOSPEC_OK;
    const bool small = kind == EVOSPEC_MOMENTS_8BIT;
    if (!m || !v || (small && !scales)) return EVOSPEC_NULL_POINTER;
    if (!aligned(m, 16) || !aligned(v, 16) || !aligned(scales, 8) || !aligned(master, 16) || !aligned(schedule, 4) || !aligned(grad_scale, 4))
        return EVOSPEC_MISALIGNED;
    for (int i = 0; i < count; ++i) {
        if (tensors[i].n == 0) continue;
        if (!tensors[i].param || !tensors[i].grad) return EVOSPEC_NULL_POINTER;
        if (!aligned(tensors[i].param, 16) || !aligned(tensors[i].grad, 16)) return EVOSPEC_MISALIGNED;
    }
    AdamwArgs a{};
    a.m = m; a.v = v; a.scales = scales; a.master = master; a.schedule = schedule; a.grad_scale = grad_scale;
    a.decay = (float)(1.0 - lr * weight_decay);
    a.rate = (float)(lr / -std::expm1((double)t * std::log(beta1)));
    a.root = (float)(1.0 / std::sqrt(-std::expm1((double)t * std::log(beta2))));
    a.beta1 = (float)beta1; a.beta1c = (float)(1.0 - beta1); a.beta2 = (float)beta2; a.beta2c = (float)(1.0 - beta2);
    a.eps = (float)eps;
    a.log_beta1 = (float)std::log(beta1); a.log_beta2 = (float)std::log(beta2); a.weight_decay = (float)weight_decay;
    a.seed_key = seed * 0x85ebca6bu;
    a.t_key = (uint32_t)t * 0xc2b2ae35u;
    return failed(launch_adamw(tensors, count, param_type, grad_type, kind, a, static_cast<hipStream_t>(stream)));
}

int evospec_adamw_moments(const void* m, const void* v, const float* scales, long long blocks, int type, void* out_m, void* out_v,
                          void* stream) {
    if (type != EVOSPEC_BF16 && type != EVOSPEC_FP32) return EVOSPEC_BAD_TYPE;
    if (blocks < 0 || blocks > (1ll << 40)) return EVOSPEC_BAD_SHAPE;
    if (blocks == 0) return EVOSPEC_OK;
    if (!m || !v || !scales || !out_m || !out_v) return EVOSPEC_NULL_POINTER;
    if (!aligned(m, 16) || !aligned(v, 16) || !aligned(scales, 8) || !aligned(out_m, 16) || !aligned(out_v, 16)) return EVOSPEC_MISALIGNED;
    return failed(launch_adamw_moments(m, v, scales, blocks, type, out_m, out_v, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
