// Launchers of the gradient norm, the AdamW step and its 8-bit moments (see adamw.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rdcn {

constexpr int ADAMW_BLOCK = 256;  // elements that share a pair of exponents in the 8-bit moments

struct AdamwTensor {
    void* param;
    float* master;     // or NULL
    const void* grad;
    void* m;           // float, or uint8 codes
    void* v;
    uint8_t* exps;     // 8-bit moments: ceil(n / 256) exponents of m, then as many of v
    int64_t n;
    float decay;       // 1 - lr * weight_decay (host lr)
    float weight_decay;
    uint32_t flags;    // ADAMW_*, and from bit ADAMW_ORDINAL on the tensor's place in the caller's list
};
enum { ADAMW_PARAM_BF16 = 1, ADAMW_GRAD_BF16 = 2, ADAMW_8BIT = 4, ADAMW_ORDINAL = 8 };

struct AdamwScalars {
    float beta1, beta2, c1, c2, eps;  // c = 1 - beta, rounded once from double
    float step_size, rsqrt_grown2;    // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    double lr, logb1, logb2;          // for a step or rate on the device: beta^t = exp(t log beta)
    int64_t step;
    const float* device_lr;           // or NULL
    const int64_t* device_step;       // or NULL
    const float* clip;                // or NULL
    float grad_scale;
    bool stochastic, carry;
    uint32_t seed;
};

// Both take any number of tensors; `t` is read before the call returns.
hipError_t launch_adamw(const AdamwTensor* t, int count, const AdamwScalars& a, hipStream_t s);

// Doubles of scratch that launch_grad_norm needs.
int64_t grad_norm_partials(const AdamwTensor* t, int count);
// out[0] = grad_scale * the 2-norm of all gradients, out[1] = the clip factor for it.
hipError_t launch_grad_norm(const AdamwTensor* t, int count, float grad_scale, float max_norm, double* part, float* out,
                            hipStream_t s);

// out (bf16) = the values that 8-bit moments stand for.
hipError_t launch_adamw_values(int64_t n, const uint8_t* codes, const uint8_t* exps, bool is_signed, void* out,
                               hipStream_t s);

}  // namespace rdcn
