// Launchers of what stands around a layer's products: the norm of rows (layer_norm.hip), the gradient of an activation
// (activation_grad.hip) and the AdamW step (adamw.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace halo {

// ---- norm of rows ----
struct NormFwd {
    const void* X; int64_t ld_x;
    const void* weight;                  // null: 1
    const void* bias;                    // null: 0
    void* Y; int64_t ld_y;
    float* mean;                         // either may be null
    float* rstd;
    int64_t rows; int cols;
    int rms, f32, weight_f32;
    float eps;
};
struct NormBwd {
    const void* E; int64_t ld_e;
    const void* X; int64_t ld_x;
    const float* mean;                   // null: 0
    const float* rstd;
    const void* weight;                  // null: 1
    const void* base; int64_t ld_base;   // null: 0
    void* EX; int64_t ld_ex;             // null: not wanted
    float* GW;                           // null: not wanted
    float* GB;
    float* part;                         // norm_bwd_workspace_floats
    int64_t rows; int cols;
    int rms, f32, weight_f32;
};
constexpr int64_t kMaxNormCols = 32768;
size_t norm_bwd_workspace_floats(int64_t rows, int64_t cols, int f32);
hipError_t launch_norm_fwd(const NormFwd& a, hipStream_t s);
hipError_t launch_norm_bwd(const NormBwd& a, hipStream_t s);

// ---- gradient of an activation ----
struct ActGrad {
    const void* E; int64_t ld_e;
    const void* Z; int64_t ld_z;         // null: act none
    void* EZ; int64_t ld_ez;             // null: not wanted
    float* GB;                           // null: not wanted
    float* part;                         // act_grad_workspace_floats
    int64_t rows, cols;
    int act, f32;
};
size_t act_grad_workspace_floats(int64_t rows, int64_t cols);
hipError_t launch_act_grad(const ActGrad& a, hipStream_t s);

// out[c] = the sum of part[p * pitch + c] over the parts p, always in the same order.  A second vector in the same launch: out2 from part2.
// Either of the two may be null.
hipError_t launch_sum_parts(const float* part, float* out, const float* part2, float* out2, int64_t parts, int64_t cols, int64_t pitch,
                            hipStream_t s);

// ---- AdamW ----
struct AdamwTensor {
    void* param;
    const void* grad;
    void* m;
    void* v;
    float* master;
    float* m_scale;
    float* v_scale;
    int64_t size;
    int32_t number;                      // the tensor's place in the caller's list
};
struct AdamwStep {
    float beta1, rest1, beta2, rest2;    // rest = 1 - beta
    float decay, rate, root;             // 1 - lr weight_decay, lr / (1 - beta1^step), 1 / sqrt(1 - beta2^step)
    float eps, grad_scale;
    uint32_t key0, key1;
    uint64_t offset;                     // of the random numbers: without a step_ptr, the step's is in it
    // where one of the pointers is not null: what the numbers above are computed from
    const int64_t* step_ptr;
    const float* lr_ptr;
    const float* grad_scale_ptr;
    int64_t step;
    double lr, log_beta1, log_beta2, weight_decay;      // logarithms to base 2
};
// param: 0 fp32, 1 bf16, 2 bf16 with a master copy.
hipError_t launch_adamw(const AdamwStep& step, const AdamwTensor* tensors, int count, int param, int grad_f32, int state8, hipStream_t s);
void adamw_numbers(double step, double lr, double beta1, double beta2, double weight_decay, float* decay, float* rate, float* root);

}  // namespace halo
