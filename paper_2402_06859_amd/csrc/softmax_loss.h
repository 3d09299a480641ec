// Launchers of the softmax loss kernels around its products (see softmax_loss.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gemm.h"

namespace rdcn {

// lse, loss and (optional) what the rows' gradients need from the logits product's partials
// softpart [tiles][rows] and zlabel [rows]. A label outside [0, classes) gives loss 0 and a row
// of zeros; one at or past `classes` also sets the index bit of *err. A row's factor = scale * (row_weight or 1).
struct SoftRows {
    int64_t rows, tiles, classes;
    const float2* softpart;
    const float* zlabel;
    const void* labels;
    bool labels64;
    const float* row_weight;
    float scale;
    float* loss;
    float* lse;
    SoftRow* row;  // may be NULL (no gradient)
    int* err;
    // with row: kept [rows, dim] = x, with zeros in the rows that have no label
    const void* x;
    void* kept;
    int64_t dim;
};
hipError_t launch_soft_rows(const SoftRows& a, bool bf16, hipStream_t s);

// e [rows][ld] (f16 times SOFT_E_SCALE, or float with T float): exponentials relative to their tile's
// maximum -> the loss's gradient in the logits, in place (storage type).
struct SoftNorm {
    int64_t rows, classes, ld;
    int tile;  // columns of a tile
    const float2* softpart;
    const SoftRow* row;
    const void* labels;
    bool labels64;
    void* e;
};
hipError_t launch_soft_normalize(const SoftNorm& a, bool bf16, hipStream_t s);
// launch_soft_rows (with row) and launch_soft_normalize in one, where soft_row_at_once says so.
bool soft_row_at_once(int64_t rows, int64_t tiles, int64_t ld);
hipError_t launch_soft_row(const SoftRows& a, const SoftNorm& n, bool bf16, hipStream_t s);

// Sums over planes: over `splits` planes of part (n floats each, in plane order), added to acc if it is not NULL;
// written to acc_out (float) or, if that is NULL, to out (storage type). n is a multiple of 4. Two go in one launch if they are split alike.
struct SoftSum {
    const float* part;
    int splits;
    int64_t n;
    const float* acc;
    float* acc_out;
    void* out;
};
hipError_t launch_soft_reduce(const SoftSum* sums, int count, bool bf16, hipStream_t s);

}  // namespace rdcn
