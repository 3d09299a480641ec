// GEMM launcher interface (see gemm.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rdcn {

enum GemmEpi {
    EPI_STORE = 0,      // c[m, n] (storage type, or f16 with c_f16) = scale * acc; c2 as c2_kind says
    EPI_STORE_F32 = 1,  // c[m, n] (float) = scale * acc
    EPI_PARTIAL = 2,    // c[z, m, n] (float) = scale * acc   (split-K partials, z = split)
    EPI_CROSS = 3,      // t = scale*acc + bias[n]; c = x0 * t + xl; t_out = t   (storage type;
                        // xl2: lo plane of a hi + lo bf16 x_l; xl_f16: x_l held as f16;
                        // c_f16: c written as f16; c2 as c2_kind says)
    EPI_RESID = 4,      // c (float) = gin + scale * acc
    EPI_RESID_X0 = 5,   // c (float) += gin + scale * acc
    // MLP layers (bf16 storage, A K-contiguous):
    EPI_MLP_FWD = 6,    // c = ReLU(scale*acc + bias[n]) * (rowv ? sigmoid(rowv[m]) : 1);
                        // with c2: an f16 copy of c (c2_kind C2_F16, err needed)
    EPI_MLP_BWD = 7,    // v = scale*acc + (colv ? rowv[m] * colv[n] : 0);
                        // act == NULL: c = v;
                        // else c = v * [act[m, n] > 0] * (rowg ? sigmoid(rowg[m]) : 1), and with
                        // rowpart: rowpart[(n0 / BN) * M + m] = sum over the tile's columns of v * act
    // Softmax loss (both operands K-contiguous), z = scale*acc + offset[n], -inf where offset[n] is:
    EPI_SOFT_FWD = 8,   // softpart[t * M + m] over the classes of column tile t (gemm_soft_tiles) other than the row's
                        // label = (max, sum of exp(z - max)); zlabel[m] = z at the label, if it is one of the tile's columns; with c:
                        // c = exp(z - max) (f16 times SOFT_E_SCALE, or float), zero at the label and in the pad of a row
    EPI_SOFT_GRAD = 9,  // c = r.c * exp(z - r.max) for r = softrow[m], r.label at the row's label (storage type), zero
                        // where r.c is 0 or z is -inf and in the pad of a row
    // Log probabilities (both operands K-contiguous), z as above:
    EPI_CHOICE_FWD = 10,  // stat[m * tiles + t] = ChoiceStat of the classes of column tile t (gemm_soft_tiles); zlabel[m] = z at
                          // the label; with groups: groups[m * ngroups + u] of the classes of group u (gemm_choice_groups);
                          // with c: c = exp(z - max of the tile) (f16 times SOFT_E_SCALE, or float), zero in the pad of a row
    EPI_CHOICE_GRAD = 11  // c = exp(d) (r.a + r.b d) for d = z - r.max, r = choicerow[m], r.label at the row's label (storage
                          // type; with c2: hi in c, lo in c2), zero where r.a and r.b are 0 or z is -inf and in the pad of a row
};

// exp(z - max) of a tile's row is held in f16 times this (a power of two): values down to
// 2^-29 of the row's largest in the tile keep all 11 bits, down to 2^-39 they are not zero.
constexpr float SOFT_E_SCALE = 32768.f;

// A row of the softmax loss. With f its gradient factor, max its largest logit and S its sum of exp(z - max): c = f / S, and
// label = -f (S - the label's own exponential) / S, the gradient in the label's logit: f (p - 1), which a subtraction of 1
// from p, or a log-sum-exp rounded to float, would leave few digits of where p is near 1.
struct SoftRow {
    float max, c, label, unused;
};

// A row's logits over some classes. With max the largest of them and d = z - max: rest = the sum of exp(d) over all but one
// class of that size (-1 where no class is visible), mean = the sum of exp(d) d. Nothing here is a difference of near values: rest keeps
// its digits where one class has nearly all of the probability, and so do 1 - p = rest / (1 + rest) and the entropy.
struct ChoiceStat {
    float max, rest, mean, unused;
};
// A row of the gradient: see EPI_CHOICE_GRAD.
struct ChoiceRow {
    float max, a, b, label;
};
// The classes of a group: the `columns / span` runs of four that begin at base + pitch k + 4 g, base = u / (pitch / 4) * span
// and g = u % (pitch / 4) for group u: what one lane of a product's block holds of a row. In memory: x = the largest logit's float bits, y =
// a bound that no other class of the group exceeds, with the largest one's place in its low 4 bits.
struct ChoiceGroups {
    int64_t count;
    int span, pitch, size;  // size: classes of a group, 8 or 16
};

// What an optional second output plane c2 receives (same row stride as c).
enum GemmC2 {
    C2_LO = 0,    // c is bf16 hi = bf16(v), c2 the lo part bf16(v - hi): the pair carries ~16 bits
    C2_BF16 = 1,  // a bf16 copy of v (c holds v as f16)
    C2_F16 = 2    // an f16 copy of v (c holds v in the storage type)
};

// Bit of the device error word set when a value written as f16 is beyond its range.
constexpr int ERR_BIT_F16_RANGE = 2;

struct GemmArgs {
    int64_t M, N, K;
    const void* a;      // A(m, k) = a[m*lda + k], or a[k*lda + m] when a_kstrided
    const void* a2;     // optional second A plane: C = (A + A2) B^T as two passes over K (no split-K)
    int64_t lda;
    const void* b;      // B(n, k) = b[n*ldb + k], or b[k*ldb + n] when b_kstrided
    int64_t ldb;
    bool a_kstrided, b_kstrided;
    bool rem_last;      // K is no multiple of 8: a K-contiguous A holds zeros behind K up to one (the row strides
                        // and whatever else is vectorised along K stay multiples of 8)
    bool ops_f16;       // A and B hold f16 values (f16 MFMAs; both K-contiguous, not EPI_MLP_BWD)
    int epi;
    float scale;
    void* c;            // output (see GemmEpi)
    void* c2;           // optional second output plane (see GemmC2)
    int c2_kind;
    bool c_f16;         // EPI_STORE / EPI_CROSS: c is written as f16
    int* err;           // device error word (needed with c_f16 or c2_kind == C2_F16)
    int64_t ldc;
    // cross / residual epilogue operands, row stride ldx
    const void* bias;
    const void* x0;
    const void* xl;
    const void* xl2;    // optional lo plane of x_l
    bool xl_f16;        // x_l is f16
    void* t_out;
    const void* gin;
    bool gin_f32;
    int64_t ldx;
    // MLP epilogue operands (act has row stride ldx)
    const float* rowv;
    const void* colv;
    const float* rowg;
    const void* act;
    float* rowpart;
    // softmax loss epilogues
    const SoftRow* softrow;  // [M]
    const float* offset;  // [N] or NULL
    const void* labels;   // [M] int32 or int64; column n stands for class label0 + n
    bool labels64;
    int64_t label0;
    float* zlabel;        // [M]
    float2* softpart;     // [gemm_soft_tiles][M]
    // log probability epilogues (and offset .. zlabel above)
    ChoiceStat* stat;     // [M][tiles]
    int64_t tiles;
    uint2* groups;        // [M][ngroups] or NULL
    int64_t ngroups;
    const ChoiceRow* choicerow;  // [M]
    int group_m;        // set from GemmPlan::group_m by launch_gemm
};

struct GemmPlan {
    int bm = 128, bn = 128;
    int splits = 1;
    int stages = 3;  // LDS ring depth (2 lets two workgroups share a CU)
    int group_m = 0; // > 1: tiles walked in groups of group_m tile rows, column by column
};

// split_blocks: with split-K allowed, the workgroup count the K split aims for when
// the output tiles alone are fewer than 256 (a product that runs beside other
// kernels does better with fewer, longer splits). fused_out: the epilogue reads and writes 10
// bytes or more per output (the cross layer's and the residual gradient's).
GemmPlan plan_gemm(int64_t M, int64_t N, int64_t K, bool bf16, bool allow_split, int split_blocks = 384,
                   bool fused_out = false);
// Float products of 16-byte aligned rows (operands' bases and strides): 64 x 64 blocks through LDS.
constexpr int F32_LDS_STAGES = 103;  // marks such a plan (other float plans leave GemmPlan::stages as it is)
inline GemmPlan plan_f32_lds() {
    GemmPlan p;
    p.bm = p.bn = 64;
    p.stages = F32_LDS_STAGES;
    return p;
}
// Logits of few rows (EPI_CHOICE_*), over at most 2^27 classes: streamed 16 x 64 blocks, or 64 x 128 or 64 x 256 ones.
constexpr int FEW_ROWS_STAGES = 104;  // marks such a plan
inline GemmPlan plan_few_rows(int bm, int bn) {
    GemmPlan p;
    p.bm = bm;
    p.bn = bn;
    p.stages = FEW_ROWS_STAGES;
    return p;
}
// Whether launch_gemm takes streamed blocks for a product of two K-contiguous operands under plan p.
bool gemm_streams(int64_t M, int64_t N, int64_t K, const GemmPlan& p);
// Whether a product's grid is one that can be launched: less than 2^32 threads along x.
bool gemm_fits_grid(int64_t M, int64_t N, const GemmPlan& p, bool bf16);
// plan_gemm (K may be split) for one long product at a time on the whole chip, whose partial sums the caller reduces.
GemmPlan plan_gemm_long(int64_t M, int64_t N, int64_t K, bool bf16);
hipError_t launch_gemm(const GemmArgs& g, const GemmPlan& p, bool bf16, hipStream_t s);
// Column tiles of an MLP GEMM under plan p (the rowpart partials per row).
inline int64_t gemm_tiles_n(int64_t N, const GemmPlan& p) { return (N + p.bn - 1) / p.bn; }
// Column tiles of a softmax loss product (EPI_SOFT_FWD) and the columns of one, as launch_gemm's blocks have them.
int64_t gemm_soft_tiles(int64_t M, int64_t N, int64_t K, const GemmPlan& p, bool bf16, int* columns);
ChoiceGroups gemm_choice_groups(int64_t M, int64_t N, int64_t K, const GemmPlan& p, bool bf16);
// Two products in one launch, with plain epilogues: x with A K-contiguous and B K-strided, y with both K-strided. gemm_pairs:
// their plans are of 64 x 64 blocks, and so few of them that a launch each would leave the chip part empty.
bool gemm_pairs(const GemmArgs& x, const GemmPlan& px, const GemmArgs& y, const GemmPlan& py, bool bf16);
hipError_t launch_gemm_pair(const GemmArgs& x, const GemmPlan& px, const GemmArgs& y, const GemmPlan& py, bool bf16,
                            hipStream_t s);
hipError_t launch_splitk_reduce(const float* part, int splits, int64_t MN, float* out, hipStream_t s);
// dst = f16(src) for n bf16 values (n % 8 == 0, 16-byte aligned); sets ERR_BIT_F16_RANGE
// in err when a value is beyond the f16 range.
hipError_t launch_bf16_to_f16(const void* src, void* dst, int64_t n, int* err, hipStream_t s);

}  // namespace rdcn
