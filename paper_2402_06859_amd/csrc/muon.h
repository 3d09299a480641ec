// Launcher of the Muon step: momentum, its orthogonalised update by Newton-Schulz products, and the weights (see muon.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace rdcn {

constexpr int64_t MUON_SIDE_MAX = 1 << 20, MUON_SHORT_MAX = 1 << 14;  // a matrix's longer and shorter side
constexpr int MUON_STEPS_MAX = 16;

struct MuonTensor {
    void* param;
    float* master;    // or NULL
    const void* grad;
    float* m;
    int64_t rows, cols;
    double weight_decay, scale;
    uint32_t flags;   // MUON_*, and from bit MUON_ORDINAL on the tensor's place in the caller's list
};
enum { MUON_PARAM_BF16 = 1, MUON_GRAD_BF16 = 2, MUON_ORDINAL = 8 };

struct MuonScalars {
    float mu, c1;               // momentum, 1 - momentum rounded once from double
    bool nesterov, stochastic;
    float grad_scale;
    double lr;
    const float* device_lr;     // or NULL, and so on
    const int64_t* device_step;
    const float* clip;
    uint32_t seed;
    double a, b, c;             // X <- a X + b A X + c A A X, A = X X^T
    int steps;
};

// Bounds of what an iteration from singular values in [0, 1] holds, and the powers of two that its matrices are kept
// in f16 times; false if it leaves the range that f16 pairs can hold.
struct MuonScales {
    float gram[MUON_STEPS_MAX], poly[MUON_STEPS_MAX], half[MUON_STEPS_MAX], power[MUON_STEPS_MAX], x[MUON_STEPS_MAX + 1];
};
bool muon_scales(double a, double b, double c, int steps, MuonScales* out);

size_t muon_scratch(const MuonTensor* t, int count);
// `t` is read before the call returns.
hipError_t launch_muon(const MuonTensor* t, int count, const MuonScalars& a, const MuonScales& q, void* scratch, hipStream_t s);

}  // namespace rdcn
