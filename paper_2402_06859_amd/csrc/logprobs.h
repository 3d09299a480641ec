// Launchers of the kernels around the products of the log probabilities (see logprobs.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gemm.h"

namespace rdcn {

constexpr int CHOICE_TOP_MAX = 32;

// Results of a row from its tiles' ChoiceStats and its groups (see gemm.h).
struct ChoiceRows {
    int64_t rows, dim, classes, tiles;
    const ChoiceStat* stat;   // [rows][tiles]
    const float* zlabel;      // [rows]
    const void* labels;       // or NULL
    bool ids64;               // labels and top_ids are 64-bit
    float* logprob;           // each of these may be NULL
    float* entropy;
    float* lse;
    float4* stats;            // [rows]: what the gradient needs of a row
    int* err;
    // top > 0:
    int top;
    ChoiceGroups g;
    const uint2* groups;      // [rows][g.count]
    const void* x;
    const void* w;
    const float* offset;      // or NULL
    float logit_scale;
    void* top_ids;            // [rows][top]
    float* top_logprob;       // or NULL
};
hipError_t launch_choice_rows(const ChoiceRows& a, bool bf16, hipStream_t s);

// row[m] (ChoiceRow) from stats and the upstream gradients, and kept [rows, dim] = x with zeros in rows without gradient, `copies` times.
struct ChoicePrepare {
    int64_t rows, dim, classes;
    const float4* stats;
    const void* labels;
    bool ids64;
    const float* grad_logprob;  // or NULL
    const float* grad_entropy;  // or NULL
    float logit_scale;
    const void* x;
    void* kept;
    int copies;
    ChoiceRow* row;
    int* err;
};
hipError_t launch_choice_prepare(const ChoicePrepare& a, bool bf16, hipStream_t s);

// out [rows][ld], `width` columns (whole vectors) of classes from `first` on: the gradient in the logits, from kept [rows][kept_ld]
// (f16 times SOFT_E_SCALE, or float) and the tiles' maxima; without `prepared` (k_choice_prepare ran for p) the
// first classes' launch makes p's copies of x too, and p.row is not used.
struct ChoiceNormalize {
    ChoicePrepare p;
    bool prepared;
    int64_t tiles, tile, first, width, ld, kept_ld;
    const ChoiceStat* stat;
    const void* kept;
    void* out;
    void* out_lo;  // or NULL; bf16: what rounding leaves of out
};
hipError_t launch_choice_normalize(const ChoiceNormalize& a, bool bf16, hipStream_t s);

}  // namespace rdcn
