// Softmax loss over a large set of classes: what stands around its products.
//
//   z[m, v] = s (x[m] . w[v]) + offset[v],  lse[m] = log sum_v exp(z[m, v]),  loss[m] = lse[m] - z[m, y[m]]
//   G[m, v] = f[m] (exp(z[m, v] - lse[m]) - [v = y[m]]),  grad_x = G w,  grad_w = G^T x
//
// The logits product (gemm.hip, EPI_SOFT_FWD) leaves one (maximum, sum of exponentials) pair per row
// and column tile; the pairs of a row are joined here: the sum of exponentials over two
// ranges with maxima a and b is S_a exp(a - c) + S_b exp(b - c) for c = max(a, b).
//
// A row stays (maximum, sum) to the end: a difference from lse, rounded to float, is off by |lse| 2^-24 and loses log(sum)
// itself where all logits are far from 0 (an offset of -10^9 on every class). And the pairs leave the label out, which joins
// them last: with R the sum over the other classes and e the label's exponential, 1 - p = R / (R + e) and loss = log(1 + R / e)
// keep their digits where p is near 1, which neither p - 1 nor lse - z[y] would, and so do the other classes' p.
#include "device_common.h"
#include "gemm.h"
#include "softmax_loss.h"

namespace rdcn {

namespace {

constexpr int ERR_BIT_INDEX = 1;
constexpr float NEG_INF = -__builtin_huge_valf();

__device__ __forceinline__ int64_t label_of(const void* labels, bool l64, int64_t m) {
    return l64 ? ((const int64_t*)labels)[m] : (int64_t)((const int32_t*)labels)[m];
}

// Joins N more ranges to (mx, sum): one maximum, then N + 1 exponentials that do not wait for each other. A range
// without any visible class has (-inf, 0) and adds nothing.
template <int N>
__device__ __forceinline__ void join(float& mx, float& sum, const float2 (&p)[N]) {
    float c = mx;
#pragma unroll
    for (int k = 0; k < N; ++k) c = fmaxf(c, p[k].x);
    const float top = c == NEG_INF ? 0.f : c;
    float s = sum * __expf(mx - top);
#pragma unroll
    for (int k = 0; k < N; ++k) s += p[k].y * __expf(p[k].x - top);
    mx = c;
    sum = s;
}

// A row without a label, or of weight 0, may hold anything (padding behind a sequence, infinities, NaN): its
// gradient factor is 0, but 0 times such a value would still reach grad_w's sum over the rows. So the product
// for grad_w reads a copy of x with zeros there, made by the workgroups from `first` on.
__device__ __forceinline__ bool row_counts(const SoftRows& a, int64_t m) {
    const int64_t y = label_of(a.labels, a.labels64, m);
    return y >= 0 && y < a.classes && !(a.row_weight && a.row_weight[m] == 0.f);
}
template <typename T>
__device__ __forceinline__ void copy_kept_rows(const SoftRows& a, int64_t first) {
    constexpr int W = st<T>::vec;
    const int64_t per = a.dim / W, n = a.rows * per, step = (gridDim.x - first) * 256ll;
    for (int64_t i = (blockIdx.x - first) * 256ll + threadIdx.x; i < n; i += step) {
        u32x4_t v = {0u, 0u, 0u, 0u};
        if (row_counts(a, i / per)) v = *(const u32x4_t*)((const T*)a.x + i * W);
        *(u32x4_t*)((T*)a.kept + i * W) = v;
    }
}

// Row m's gradient from the maximum and sum over the classes other than its label; `write`: it, loss and lse go out.
__device__ __forceinline__ SoftRow finish_row(const SoftRows& a, int64_t m, float others, float rest, bool write) {
    const int64_t y = label_of(a.labels, a.labels64, m);
    const bool kept = y >= 0 && y < a.classes;
    const float f = a.row && kept ? a.scale * (a.row_weight ? a.row_weight[m] : 1.f) : 0.f;
    const float z = kept ? a.zlabel[m] : NEG_INF;
    const bool seen = z != NEG_INF;  // the row's label has a probability
    const bool alone = others == NEG_INF && rest == 0.f, none = alone && !seen;  // (a row of NaN has such a maximum, but that sum)
    const float mx = fmaxf(others, z), own = seen ? expf(z - mx) : 0.f;
    if (!alone) rest *= expf(others - mx);
    const float sum = rest + own;
    SoftRow r{};
    r.max = mx;
    if (f != 0.f && !none) {
        r.c = f / sum;
        r.label = seen ? -f * (rest / sum) : 0.f;
    }
    if (write) {
        if (y >= a.classes) atomicOr(a.err, ERR_BIT_INDEX);
        a.lse[m] = none ? NEG_INF : mx + logf(sum);
        // a label whose own class is masked has probability 0: its loss is +inf, also where every class is
        float loss = 0.f;
        if (kept) loss = !seen ? -NEG_INF : rest < own ? log1pf(rest / own) : (mx - z) + logf(sum);
        a.loss[m] = loss;
        if (a.row) a.row[m] = r;
    }
    return r;
}

// 256 threads as rpb rows x (256 / rpb) lanes that stride over the tiles. Few rows take many
// lanes each (one request over 50000 classes has 782 pairs to join), many rows one lane or few.
template <typename T>
__global__ __launch_bounds__(256) void k_soft_rows(SoftRows a, int rpb) {
    __shared__ float2 sh[256];
    const int64_t nrow = (a.rows + rpb - 1) / rpb;
    if (blockIdx.x >= nrow) {
        copy_kept_rows<T>(a, nrow);
        return;
    }
    const int r = threadIdx.x % rpb, part = threadIdx.x / rpb, parts = 256 / rpb;  // (rpb a power of two)
    const int64_t m = (int64_t)blockIdx.x * rpb + r;
    float mx = NEG_INF, sum = 0.f;
    if (m < a.rows)
        for (int64_t t = part; t < a.tiles; t += 8 * parts) {
            float2 p[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                p[k] = t + k * parts < a.tiles ? a.softpart[(t + k * parts) * a.rows + m] : make_float2(NEG_INF, 0.f);
            join(mx, sum, p);
        }
    sh[threadIdx.x] = make_float2(mx, sum);
    for (int o = parts / 2; o > 0; o >>= 1) {
        __syncthreads();
        if (part < o) {
            const float2 p[1] = {sh[threadIdx.x + o * rpb]};
            join(mx, sum, p);
            sh[threadIdx.x] = make_float2(mx, sum);
        }
    }
    if (part != 0 || m >= a.rows) return;
    (void)finish_row(a, m, mx, sum, true);
}

// Columns first, first + step, .. (vectors) of row m of E -> G. Reads and writes each element once (2 + 2 bytes, 4 + 4
// in float); the factor exp(tile's maximum - row's) f / S is one exponential per vector, not per element. The label's
// own element is the row's.
template <typename T>
__device__ __forceinline__ void normalize_row(const SoftNorm& a, int64_t m, const SoftRow& r, int64_t y, int64_t first,
                                              int64_t step) {
    constexpr int W = st<T>::vec;
    for (int64_t n = first * W; n < a.ld; n += step * W) {
        const float top = a.softpart[n / a.tile * a.rows + m].x;
        float v[W];
        if constexpr (sizeof(T) == 2) unpack_f16x8(*(const u32x4_t*)((const _Float16*)a.e + m * a.ld + n), v);
        else st<T>::unpack(*(const u32x4_t*)((const float*)a.e + m * a.ld + n), v);
        const float unit = sizeof(T) == 2 ? 1.f / SOFT_E_SCALE : 1.f;
        const float c = r.c == 0.f || top == NEG_INF ? 0.f : r.c * unit * expf(top - r.max);
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] = c == 0.f ? 0.f : c * v[e];
        if (y >= n && y < n + W) {
#pragma unroll
            for (int e = 0; e < W; ++e)
                if (y - n == e) v[e] = r.label;
        }
        *(u32x4_t*)((T*)a.e + m * a.ld + n) = st<T>::pack(v);
    }
}

// One workgroup per (row, stretch of columns).
template <typename T>
__global__ __launch_bounds__(256) void k_soft_normalize(SoftNorm a) {
    const int64_t m = blockIdx.y + (int64_t)blockIdx.z * 65535;
    if (m >= a.rows) return;
    normalize_row<T>(a, m, a.row[m], label_of(a.labels, a.labels64, m), blockIdx.x * 256ll + threadIdx.x,
                     gridDim.x * 256ll);
}

// The join, G's row and the kept row of x in one workgroup per row: a launch less where its pairs are few.
template <typename T>
__global__ __launch_bounds__(256) void k_soft_row(SoftRows a, SoftNorm b) {
    __shared__ float2 sh[4];
    const int64_t m = blockIdx.x;
    float mx = NEG_INF, sum = 0.f;
    for (int64_t t = threadIdx.x; t < a.tiles; t += 256) {
        const float2 p[1] = {a.softpart[t * a.rows + m]};
        join(mx, sum, p);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const float2 p[1] = {make_float2(__shfl_xor(mx, o), __shfl_xor(sum, o))};
        join(mx, sum, p);
    }
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = make_float2(mx, sum);
    __syncthreads();
    const float2 p[4] = {sh[0], sh[1], sh[2], sh[3]};
    mx = NEG_INF;
    sum = 0.f;
    join(mx, sum, p);
    const SoftRow r = finish_row(a, m, mx, sum, threadIdx.x == 0);
    const int64_t y = label_of(a.labels, a.labels64, m);
    normalize_row<T>(b, m, r, y, threadIdx.x, 256);
    constexpr int W = st<T>::vec;
    const bool kept = row_counts(a, m);
    for (int64_t i = threadIdx.x; i < a.dim / W; i += 256) {
        u32x4_t v = {0u, 0u, 0u, 0u};
        if (kept) v = *(const u32x4_t*)((const T*)a.x + m * a.dim + i * W);
        *(u32x4_t*)((T*)a.kept + m * a.dim + i * W) = v;
    }
}

// Row y of the grid takes sum y. LANES > 1: that many groups of a workgroup's threads take every LANES-th plane of the same outputs, and their sums are
// added in group order (few outputs with many planes: a serial chain of loads otherwise).
template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_soft_reduce(SoftSum s0, SoftSum s1) {
    const SoftSum& q = blockIdx.y ? s1 : s0;
    const float* const part = q.part;
    const float* const acc = q.acc;
    float* const acc_out = q.acc_out;
    T* const out = (T*)q.out;
    const int splits = q.splits;
    const int64_t n = q.n;
    constexpr int PER = 256 / LANES;  // threads of a group
    __shared__ f32x4_t sh[LANES > 1 ? 256 : 1];
    const int lane = threadIdx.x / PER;
    for (int64_t i0 = (int64_t)blockIdx.x * PER * 4; i0 < n; i0 += (int64_t)gridDim.x * PER * 4) {
        const int64_t i = i0 + threadIdx.x % PER * 4;
        f32x4_t v = {0.f, 0.f, 0.f, 0.f};
        if (i < n) {
#pragma unroll 4
            for (int z = lane; z < splits; z += LANES) v += *(const f32x4_t*)(part + z * n + i);
        }
        if constexpr (LANES > 1) {
            __syncthreads();
            sh[threadIdx.x] = v;
            __syncthreads();
            if (lane != 0) continue;
#pragma unroll
            for (int k = 1; k < LANES; ++k) v += sh[threadIdx.x + k * PER];
        }
        if (i >= n) continue;
        if (acc) v += *(const f32x4_t*)(acc + i);
        if (acc_out) {
            *(f32x4_t*)(acc_out + i) = v;
        } else if constexpr (sizeof(T) == 4) {
            *(f32x4_t*)(out + i) = v;
        } else {
            *(uint2*)(out + i) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
        }
    }
}

dim3 blocks_for(int64_t items, int64_t most) {
    const int64_t b = (items + 255) / 256;
    return dim3((unsigned)(b < 1 ? 1 : b > most ? most : b));
}

}  // namespace

hipError_t launch_soft_rows(const SoftRows& a, bool bf16, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    int rpb = 1;  // about 256 workgroups or more, as long as there are that many rows
    while (rpb < 64 && a.rows / (2 * rpb) >= 256) rpb *= 2;
    const unsigned nrow = (unsigned)((a.rows + rpb - 1) / rpb);
    const unsigned ncopy = a.row ? blocks_for(a.rows * a.dim / (bf16 ? 8 : 4), 4096).x : 0;
    if (bf16) hipLaunchKernelGGL(k_soft_rows<bf16_t>, dim3(nrow + ncopy), dim3(256), 0, s, a, rpb);
    else hipLaunchKernelGGL(k_soft_rows<float>, dim3(nrow + ncopy), dim3(256), 0, s, a, rpb);
    return hipGetLastError();
}

bool soft_row_at_once(int64_t rows, int64_t tiles, int64_t ld) {
    // a workgroup per row has to fill the chip, unless rows are short; pairs of one row lie far apart (us, at once / apart:
    // 157 pairs of 512 rows 8.4 / 11, 500 of 4096 132 / 105)
    return tiles <= 192 && (rows >= 256 || ld <= 8192) && rows < 1 << 24;  // (a grid has less than 2^32 threads)
}

hipError_t launch_soft_row(const SoftRows& a, const SoftNorm& n, bool bf16, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    if (bf16) hipLaunchKernelGGL(k_soft_row<bf16_t>, dim3((unsigned)a.rows), dim3(256), 0, s, a, n);
    else hipLaunchKernelGGL(k_soft_row<float>, dim3((unsigned)a.rows), dim3(256), 0, s, a, n);
    return hipGetLastError();
}

hipError_t launch_soft_normalize(const SoftNorm& a, bool bf16, hipStream_t s) {
    if (a.rows == 0 || a.ld == 0) return hipSuccess;
    const int64_t per = a.ld / (bf16 ? 8 : 4);
    const int64_t y = a.rows < 65535 ? a.rows : 65535, z = (a.rows + 65534) / 65535;
    const dim3 grid(blocks_for((per + 3) / 4, 64).x, (unsigned)y, (unsigned)z);
    if (bf16) hipLaunchKernelGGL(k_soft_normalize<bf16_t>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(k_soft_normalize<float>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_soft_reduce(const SoftSum* sums, int count, bool bf16, hipStream_t s) {
    if (count < 1 || count > 2) return hipErrorInvalidValue;
    auto lanes = [](const SoftSum& q) { return q.splits > 8 && q.n / 4 <= 256 * 256 ? 8 : 1; };
    for (int i = 0; i < count; ++i) {
        const SoftSum s0 = sums[i];
        // One of eight groups and one of none: up to 16 planes one launch without groups is ahead of a launch each (float
        // 512 x 160 x 5000, 16 planes and 1: the gradient takes 55.3 us against 57.9); a chain of 64 loads isn't.
        const bool alike = i + 1 < count && lanes(sums[i + 1]) == lanes(s0);
        const bool both = i + 1 < count && (alike || (s0.splits <= 16 && sums[i + 1].splits <= 16));
        const int groups = both && !alike ? 1 : lanes(s0);
        const SoftSum s1 = both ? sums[++i] : s0;
        const int64_t n = s0.n > s1.n ? s0.n : s1.n;
        if (n == 0) continue;
        const dim3 grid(blocks_for(n / 4 * groups, 4096).x, both ? 2 : 1);
        if (groups == 8) {
            if (bf16) hipLaunchKernelGGL((k_soft_reduce<bf16_t, 8>), grid, dim3(256), 0, s, s0, s1);
            else hipLaunchKernelGGL((k_soft_reduce<float, 8>), grid, dim3(256), 0, s, s0, s1);
        } else {
            if (bf16) hipLaunchKernelGGL((k_soft_reduce<bf16_t, 1>), grid, dim3(256), 0, s, s0, s1);
            else hipLaunchKernelGGL((k_soft_reduce<float, 1>), grid, dim3(256), 0, s, s0, s1);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace rdcn
