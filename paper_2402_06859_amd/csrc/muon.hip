// The Muon step over many matrices at once: a momentum, its update made (nearly) orthogonal by Newton-Schulz products, and the weights.
//
//   M' = mu M + (1 - mu) g,  U = mu M' + (1 - mu) g (or M'),  X = U / |U|
//   X <- (a I + b A + c A^2) X,  A = X X^T        `steps` times
//   p' = p (1 - lr wd) - lr scale X
//
// Products on the Gram matrix. Every X of the iteration is a polynomial of A = X0 X0^T times X0, so the steps run on m x m matrices, m
// the shorter side (for a tall matrix A = X^T X and X times the polynomial):
//   T = a I + b A + c A^2,   P <- T P,   A <- T A T = T (T A)
// and X = P X0 once. All of them are symmetric: only the blocks on and under the diagonal are computed, and stored twice. For sides m <=
// n, five steps take (17 + 3 n/m) m^3 operations against 5 (3 n/m + 1) m^3 with X itself. A error in a small direction of A grows by
// up to a^2 (12) a step, while X's own would grow by a with the direction: so X and A are made anew after two steps, and every three from
// then on (6 n/m + 14 m^3 for five steps). The error of X over spectra from even to falling by 10^6 (relative, five steps, 30 x 80 to 1000 x
// 1000): 2e-7 to 5e-5, float products of X itself 2e-7 to 7e-5; of ordinary ones (i^-1/2) 1e-6 and 1e-6, falling by 10^3 1e-5 and 2e-6. Never
// restarted it reached 4e-4.
//
// Operands. Every matrix stands as a pair of f16, hi + lo of a power of two times its values (22 bits), and a product is three of f16 matrix
// instructions: hi hi + hi lo + lo hi, sums in float. (One f16 each would leave 3e-3 to 5e-1 of X in error, bf16 more; float
// matrix instructions run at a sixteenth of the rate.) The powers keep all values below f16's range: |A| <= 1 for X of norm 1, and what
// follows is bounded by the polynomial's largest value on the singular values' range (muon_scales). Matrices are padded with zeros to
// multiples of 64: zero rows stay zero rows of X, and no load needs a bound.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "device_common.h"
#include "mfma_tiles.h"
#include "muon.h"

namespace rdcn {

namespace {

constexpr int PAD = 64;              // sides are padded to multiples of this
constexpr int PARTS = 512;           // most partial sums of a matrix's norm, each of at least PART elements
constexpr int PART = 8192;
constexpr int SPLIT_ROWS = 64, SPLIT_COLS = 128;
constexpr int PER_LAUNCH = 24;       // matrices, or products, of one launch: their descriptors are kernel arguments
constexpr int NAMES = 5;             // m x m matrices in scratch
enum { GRAM = 0, HALF = 1, FREE = 2 };  // A, T A, and three for T and P in turn

int64_t padded(int64_t n) { return (n + PAD - 1) / PAD * PAD; }

struct Matrix {
    const void* grad;
    float* m;
    void* param;
    float* master;
    uint16_t* x;      // [2][rp][cp]: hi, lo
    double* part;     // [parts]
    int64_t rows, cols;
    int32_t rp, cp, parts;
    int32_t per;      // elements of a part
    uint32_t flags;
    float weight_decay;
    double scale;
};

struct Elements {  // the momentum and the split of many matrices
    Matrix t[PER_LAUNCH];
    uint32_t first[PER_LAUNCH + 1];  // first workgroup of each
    int count;
    MuonScalars a;
    float scale;  // of x
};
static_assert(sizeof(Elements) <= 4096, "kernel arguments");

// The entry that workgroup b belongs to: one load for all of them, lane by lane (a search would wait for each in turn).
__device__ __forceinline__ int entry_of(const uint32_t* first, int count, uint32_t b) {
    const int lane = threadIdx.x & 63;
    const bool begun = lane < count && first[lane < PER_LAUNCH ? lane : PER_LAUNCH] <= b;
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(begun)) - 1);
}

// Sum of 256 doubles over a workgroup, in a fixed order, for every thread.
__device__ __forceinline__ double block_sum(double x) {
    __shared__ double sh[4];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
    __syncthreads();
    return ((sh[0] + sh[1]) + sh[2]) + sh[3];
}

// The factor of the gradients, or false where the clip factor is not finite: such a step changes nothing.
__device__ __forceinline__ bool gradient_scale(const MuonScalars& a, float& gs) {
    gs = a.grad_scale;
    if (!a.clip) return true;
    const float c = *a.clip;
    gs *= c;
    return fabsf(c) < __builtin_huge_valf();
}

// Elements from <= e < to of v[8], as a pair.
__device__ __forceinline__ void store_pair(uint16_t* c, int64_t plane, const float* v, int from, int to) {
    if (to <= 0 || from >= 8) return;
    bool ovf = false;
    float hi[8], lo[8];
    const u32x4_t h = pack_f16x8(v, ovf);
    unpack_f16x8(h, hi);
#pragma unroll
    for (int e = 0; e < 8; ++e) lo[e] = v[e] - hi[e];
    const u32x4_t l = pack_f16x8(lo, ovf);
    if (from <= 0 && to >= 8) {
        *(u32x4_t*)c = h;
        *(u32x4_t*)(c + plane) = l;
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (e < from || e >= to) continue;
        c[e] = (uint16_t)(h[e / 2] >> (16 * (e & 1)));
        c[plane + e] = (uint16_t)(l[e / 2] >> (16 * (e & 1)));
    }
}

// Eight values of an array from element i on, `left` of which exist (eight: a vector, whatever its alignment: rows of an odd length).
typedef u32x4_t u32x4_a4_t __attribute__((aligned(4)));
typedef u32x4_t u32x4_a2_t __attribute__((aligned(2)));
__device__ __forceinline__ void load_f32(const float* p, int64_t i, int left, float* v) {
    if (left == 8) {
        st<float>::unpack(*(const u32x4_a4_t*)(p + i), v);
        st<float>::unpack(*(const u32x4_a4_t*)(p + i + 4), v + 4);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < left ? p[i + e] : 0.f;
    }
}
__device__ __forceinline__ void load_bf16(const bf16_t* p, int64_t i, int left, float* v) {
    if (left == 8) {
        st<bf16_t>::unpack(*(const u32x4_a2_t*)(p + i), v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < left ? bf16_to_f32(p[i + e]) : 0.f;
    }
}
__device__ __forceinline__ void load_grad(const Matrix& t, int64_t i, int left, float* v) {
    if (t.flags & MUON_GRAD_BF16) load_bf16((const bf16_t*)t.grad, i, left, v);
    else load_f32((const float*)t.grad, i, left, v);
}
__device__ __forceinline__ float update_of(const MuonScalars& a, float m, float g) {
#pragma clang fp contract(off)
    return a.nesterov ? m * a.mu + g * a.c1 : m;
}

// M' of elements from <= k < to (from a multiple of 8) by a workgroup, and its threads' shares of |U|^2, in 64 bits: the squares of
// floats cannot overflow there, or vanish.
__device__ __forceinline__ double momentum_range(const Matrix& t, const MuonScalars& a, float gs, bool taken, int64_t from, int64_t to) {
#pragma clang fp contract(off)
    double s[2] = {0.0, 0.0};
    for (int64_t k = from + threadIdx.x * 8; k < to; k += 2048) {
        const int left = to - k < 8 ? (int)(to - k) : 8;
        float g[8], m[8];
        load_grad(t, k, left, g);
        load_f32(t.m, k, left, m);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = g[e] * gs;
            m[e] = m[e] * a.mu + x * a.c1;
            const double u = (double)update_of(a, m[e], x);
            s[e & 1] = fma(u, u, s[e & 1]);
        }
        if (!taken) continue;
        if (left == 8) {
            *(u32x4_t*)(t.m + k) = st<float>::pack(m);
            *(u32x4_t*)(t.m + k + 4) = st<float>::pack(m + 4);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) t.m[k + e] = m[e];
        }
    }
    return s[0] + s[1];
}

// X's elements (r, c) .. (r, c + 7), 0 outside the matrix.
__device__ __forceinline__ void x_elements(const Matrix& t, const MuonScalars& a, float gs, bool taken, double inv, int64_t r, int64_t c,
                                           float (&v)[8]) {
#pragma clang fp contract(off)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
    if (!taken || r >= t.rows || c >= t.cols) return;
    const int64_t k = r * t.cols + c;
    const int left = t.cols - c < 8 ? (int)(t.cols - c) : 8;
    float g[8] = {}, m[8];
    if (a.nesterov) load_grad(t, k, left, g);  // (else U is the momentum itself)
    load_f32(t.m, k, left, m);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? (float)((double)update_of(a, m[e], g[e] * gs) * inv) : 0.f;
}

__global__ __launch_bounds__(256) void k_muon_momentum(Elements b) {
    float gs;
    const bool taken = gradient_scale(b.a, gs);
    const int i = entry_of(b.first, b.count, blockIdx.x);
    const Matrix& t = b.t[i];
    const int64_t n = t.rows * t.cols, from = (int64_t)(blockIdx.x - b.first[i]) * t.per;
    const double sum = block_sum(momentum_range(t, b.a, gs, taken, from, from + t.per < n ? from + t.per : n));
    if (threadIdx.x == 0) t.part[blockIdx.x - b.first[i]] = sum;
}

// X = U / |U| as a pair of f16, padded with zeros; a workgroup per SPLIT_ROWS x SPLIT_COLS block, eight columns a thread.
__global__ __launch_bounds__(256) void k_muon_split(Elements b) {
    float gs;
    const bool taken = gradient_scale(b.a, gs);
    const int i = entry_of(b.first, b.count, blockIdx.x);
    const Matrix& t = b.t[i];
    double s = 0.0;
    for (int k = threadIdx.x; k < t.parts; k += 256) s += t.part[k];
    s = block_sum(s);
    // (a norm of 0: X is 0, and only the decay moves the weights)
    const double inv = s == 0.0 ? 0.0 : (double)b.scale / sqrt(s);
    const int block = (int)(blockIdx.x - b.first[i]), across = (t.cp + SPLIT_COLS - 1) / SPLIT_COLS;
    const int r0 = block / across * SPLIT_ROWS, c = block % across * SPLIT_COLS + (threadIdx.x % (SPLIT_COLS / 8)) * 8;
    if (c >= t.cp) return;
    const int64_t plane = (int64_t)t.rp * t.cp;
    for (int r = r0 + threadIdx.x / (SPLIT_COLS / 8); r < r0 + SPLIT_ROWS && r < t.rp; r += 256 / (SPLIT_COLS / 8)) {
        float v[8];
        x_elements(t, b.a, gs, taken, inv, r, c, v);
        store_pair(t.x + (int64_t)r * t.cp + c, plane, v, 0, 8);
    }
}

// One product C[m, n] = sum_k A(m, k) B(n, k) of pairs; all sides multiples of PAD.
struct Product {
    const uint16_t *a, *b;   // hi; lo is `ap` (`bp`) elements behind it
    const uint16_t* aux;     // POLY: the Gram matrix, laid out as c
    uint16_t* c;             // pair
    int64_t ap, bp;          // (c's planes and aux's are M * N apart)
    int32_t lda, ldb;
    int32_t M, N, K;
    int32_t tall;
};
struct Destination {         // STEP: where the update goes
    void* param;
    float* master;
    int64_t rows, cols;
    double scale;
    float weight_decay;
    uint32_t flags;
};
enum { PAIR = 0, POLY = 1, STEP = 2 };

struct StepFactors {
    float decay, size;
    uint32_t key;
};
__device__ __forceinline__ bool step_factors(const MuonScalars& a, const Destination& d, StepFactors& f) {
    float gs;
    if (!gradient_scale(a, gs)) return false;
    const double lr = a.device_lr ? (double)*a.device_lr : a.lr;
    f.decay = (float)(1.0 - lr * (double)d.weight_decay);
    f.size = (float)(lr * d.scale);
    uint32_t seed = a.seed;
    if (a.device_step) {  // a step that is replayed draws anew
        const int64_t t = *a.device_step;
        seed += (uint32_t)(t < 1 ? 1 : t) * 0x85EBCA6Bu;
    }
    f.key = seed + 0x9E3779B9u * ((d.flags >> MUON_ORDINAL) + 1u);
    return true;
}

// p' of the elements (m, n) .. (m, n + 7) that the matrix has, v their X.
__device__ __forceinline__ void step_elements(const MuonScalars& a, const Destination& d, const StepFactors& f, int64_t m, int64_t n,
                                              const float* v) {
#pragma clang fp contract(off)
    if (m >= d.rows || n >= d.cols) return;
    const int64_t at = m * d.cols + n;
    const int left = d.cols - n < 8 ? (int)(d.cols - n) : 8;
    const bool pbf = d.flags & MUON_PARAM_BF16;
    float p[8];
    if (d.master) load_f32(d.master, at, left, p);
    else if (pbf) load_bf16((const bf16_t*)d.param, at, left, p);
    else load_f32((const float*)d.param, at, left, p);
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = p[e] * f.decay - v[e] * f.size;
    if (d.master || !pbf) {
        float* const q = (d.master ? d.master : (float*)d.param) + at;
        if (left == 8) {
            *(u32x4_a4_t*)q = st<float>::pack(p);
            *(u32x4_a4_t*)(q + 4) = st<float>::pack(p + 4);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) q[e] = p[e];
        }
    }
    if (!pbf) return;
    uint32_t r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (a.stochastic && !d.master) {
            const uint32_t h = fmix32((uint32_t)(at + e) ^ f.key);
            r[e] = (__float_as_uint(p[e]) + ((h * 0x85EBCA6Bu) >> 16)) >> 16;
            r[e] = p[e] == p[e] ? r[e] : 0x7FC0u;  // (a NaN's bits could carry into its sign)
        } else {
            r[e] = f32_to_bf16(p[e]);
        }
    }
    bf16_t* const q = (bf16_t*)d.param + at;
    if (left == 8) {
        *(u32x4_a2_t*)q = u32x4_t{r[0] | r[1] << 16, r[2] | r[3] << 16, r[4] | r[5] << 16, r[6] | r[7] << 16};
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) q[e] = (bf16_t)r[e];
    }
}

struct Products {
    Product p[PER_LAUNCH];
    uint32_t first[PER_LAUNCH + 1];
    int count;
    float scale;             // of the sum: what the operands were held times, undone
    float out;               // what c is held times
    float pa, pb, pc;        // POLY: pa I + pb aux + pc sum, aux as it is held
    float scale2, out2;      // of the products from `second` on
    int second;
    int from;                // quarters: blocks of twice the side in front of this launch's, which are all cut in four; else -1
    Destination d[PER_LAUNCH];
    MuonScalars s;
};
static_assert(sizeof(Products) <= 4096, "kernel arguments");

// A barrier for what is in LDS alone: __syncthreads() also waits until the stores to memory have arrived, some 0.7 us.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// BM x BM blocks of WM x WN waves, each of 32 x 32 tiles; K in stages of KB through a ring of ST in LDS, filled by direct
// global-to-LDS loads. One barrier a stage, before its last substep's multiplies, whose fragments are then in registers: behind it the
// slot just read is filled again and the next stage's first fragments are read, every read and load between two multiplies.
template <int BM, int WM, int WN, int KW, bool AKS, bool BKS, int KB, int ST, bool SYM, int EPI>
__device__ __forceinline__ void product_block(const Products& b, int i, int t, int quarter, bf16_t* smem) {
    constexpr int NW = WM * WN * KW, THREADS = 64 * NW, NI = BM * KB / (512 * NW), LOADS = 4 * NI;
    constexpr int TM = BM / WM / 32, TN = BM / WN / 32, NS = KB / 16 / KW, CH = 64, CP = BM + 4;
    constexpr int EO = BM * KB, STAGE = 4 * EO;  // a stage: A hi, A lo, B hi, B lo
    constexpr int MU = 3 * TM * TN, FR = 2 * (TM + TN);  // multiplies and fragments of a substep
    constexpr int SUMS = TM * TN == 1 ? 3 : 1;           // one tile a wave: a sum for each of the three products, so that none waits
    static_assert(NS % 2 == 0, "the fragment buffers alternate");
    static_assert(KW * CH * CP * 4 <= ST * STAGE * 2, "the staged sums fit the ring");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, kw = wave / (WM * WN);
    const int wm = wave / WN % WM, wn = wave % WN;
    const Product p = b.p[i];  // (a copy: the loads' asm would have the arguments read again in every step)
    // Groups of GROUP tile rows, walked column by column: the blocks that run together on an XCD share their panels in its L2.
    const bool quarters = BM == 128 && quarter >= 0;
    const int GROUP = BM == 256 || quarters ? 4 : 8, side = quarters ? 2 * BM : BM;
    const int tiles_m = (p.M + side - 1) / side, tiles_n = (p.N + side - 1) / side;
    int tm, tn;
    if constexpr (SYM) {
        // on and under the diagonal: in front of group g lie GROUP^2 g (g - 1) / 2 + g GROUP (GROUP + 1) / 2 tiles; it has
        // GROUP g whole columns, then a triangle
        auto before = [&](int g) { return GROUP * GROUP * (g * (g - 1) / 2) + g * (GROUP * (GROUP + 1) / 2); };
        int g = (int)(sqrtf(2.f * (float)t) / (float)GROUP);
        while (before(g) > t) --g;
        while (before(g + 1) <= t) ++g;
        const int rows = tiles_m - g * GROUP < GROUP ? tiles_m - g * GROUP : GROUP, r = t - before(g), whole = rows * g * GROUP;
        if (r < whole) {
            tn = r / rows;
            tm = g * GROUP + r - tn * rows;
        } else {
            int row = 0, q = r - whole;
            while (q > row) q -= ++row;
            tm = g * GROUP + row;
            tn = g * GROUP + q;
        }
    } else {
        const int per = GROUP * tiles_n, g = t / per, r = t - g * per;
        const int rows = tiles_m - g * GROUP < GROUP ? tiles_m - g * GROUP : GROUP;
        tn = r / rows;
        tm = g * GROUP + r - tn * rows;
    }
    if (quarters) {
        tm = 2 * tm + (quarter >> 1);
        tn = 2 * tn + (quarter & 1);
        if ((SYM && tn > tm) || tm * BM >= p.M || tn * BM >= p.N) return;
    }
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BM;

    uint32_t aoff[NI], boff[NI];
    stage_offsets<BM, AKS, NW, KB>(p.lda, p.M, m0, m0, wave, lane, aoff);
    stage_offsets<BM, BKS, NW, KB>(p.ldb, p.N, n0, n0, wave, lane, boff);
    const int nk = p.K / KB;
    const uint32_t ring = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_addr(smem));
    const uint32_t mine = (uint32_t)__builtin_amdgcn_readfirstlane(wave * NI) * 1024u;
    struct Source {
        const void* at[4];  // A hi, A lo, B hi, B lo
    };
    auto source = [&](int kt) __attribute__((always_inline)) {
        const int64_t k0 = (int64_t)kt * KB;
        const uint16_t* const x = p.a + (AKS ? k0 * p.lda + m0 : m0 * p.lda + k0);
        const uint16_t* const y = p.b + (BKS ? k0 * p.ldb + n0 : n0 * p.ldb + k0);
        return Source{{uniform_ptr(x), uniform_ptr(x + p.ap), uniform_ptr(y), uniform_ptr(y + p.bp)}};
    };
    auto load = [&](int j, const Source& src, uint32_t off) __attribute__((always_inline)) {  // load j of a stage
        const int o = j / NI, u = j % NI;
        dma16_s(o < 2 ? aoff[u] : boff[u], src.at[o], ring + off + o * (EO * 2u) + mine + 1024u * u);
    };
    f32x16_t acc[SUMS][TM][TN];
#pragma unroll
    for (int z = 0; z < SUMS; ++z)
#pragma unroll
        for (int x = 0; x < TM; ++x)
#pragma unroll
            for (int y = 0; y < TN; ++y)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[z][x][y][e] = 0.f;
    uint32_t fa = frag_base<BM, AKS, KB>(smem, wm * (BM / WM), lane);
    uint32_t fb = frag_base<BM, BKS, KB>(smem + 2 * EO, wn * (BM / WN), lane);
    // (the substeps of wave group kw: NS from kw NS on)
    if constexpr (!AKS) fa ^= (uint32_t)(kw * NS * 32);
    else fa += (uint32_t)(kw * NS * 16 * BM * 2);
    if constexpr (!BKS) fb ^= (uint32_t)(kw * NS * 32);
    else fb += (uint32_t)(kw * NS * 16 * BM * 2);
    bf16x8_t af[2][2][TM], bf[2][2][TN];  // [buffer][hi, lo]
    auto frag = [&](int f, uint32_t off, int buf, int s) __attribute__((always_inline)) {
        const int q = f / (TM + TN), g = f % (TM + TN);  // hi first
        if (g < TN) bf[buf][q][g] = frag_at<BM, BKS, KB>(fb, off + q * (EO * 2u), g, s);
        else af[buf][q][g - TN] = frag_at<BM, AKS, KB>(fa, off + q * (EO * 2u), g - TN, s);
    };
    // the small products first
    auto mul = [&](int u, int buf) __attribute__((always_inline)) {
        const int k = u / (TM * TN), x = u % (TM * TN) / TN, y = u % TN;
        f32x16_t& c = acc[SUMS == 3 ? k : 0][x][y];
        c = mfma32x32x16<true>(bf[buf][k == 0][y], af[buf][k == 1][x], c);
    };
    // what the epilogue needs of the arguments, read before the loop: behind it each would be waited for
    const int64_t plane = (int64_t)p.M * p.N;
    float scale = i >= b.second ? b.scale2 : b.scale, out = i >= b.second ? b.out2 : b.out;
    float pa = b.pa, pb = b.pb, pc = b.pc;
    asm volatile("" : "+s"(scale), "+s"(out), "+s"(pa), "+s"(pb), "+s"(pc));
    const bool diagonal = SYM && tm == tn;
    StepFactors f;
    if constexpr (EPI == STEP) {
        if (!step_factors(b.s, b.d[i], f)) return;
    }
    // QUARTIC's block of the Gram matrix, where a thread has little of it: on its way before the operands
    constexpr int AHEAD = EPI == POLY && BM == 64 ? CH * (BM / 8) / THREADS : 0;
    u32x4_t ahead[AHEAD + 1][2];
    if constexpr (AHEAD > 0) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {  // (sides are multiples of 64: the block is whole)
            const int q = tid + u * THREADS;
            const uint16_t* const at = p.aux + (m0 + q / (BM / 8)) * p.N + n0 + q % (BM / 8) * 8;
            ahead[u][0] = *(const u32x4_t*)at;
            ahead[u][1] = *(const u32x4_t*)(at + (int64_t)p.M * p.N);
        }
    }
    constexpr uint32_t SB = STAGE * 2u;
    for (int u = 0; u < ST && u < nk; ++u) {
        const Source src = source(u);
#pragma unroll
        for (int j = 0; j < LOADS; ++j) load(j, src, u * SB);
    }
    if (nk >= ST) wait_vmcnt(LOADS * (ST - 1));  // the first stage has landed
    else wait_vmcnt(0);
    __builtin_amdgcn_s_barrier();
#pragma unroll
    for (int f = 0; f < FR; ++f) frag(f, 0, 0, 0);
    constexpr int RPM = MU > 4 ? (FR + MU - 3) / (MU - 2) : 2;  // fragments read behind a multiply
    uint32_t cur = 0;
    auto step = [&](int kt, auto refill_c) __attribute__((always_inline)) {
        constexpr bool REFILL = decltype(refill_c)::value;
        const uint32_t nxt = cur == (ST - 1) * SB ? 0 : cur + SB;
        asm volatile("" : "+v"(fa), "+v"(fb));  // (addresses are formed here, not kept for every fragment)
        const Source src = REFILL ? source(kt + ST) : Source{};
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const bool last = s == NS - 1;
            if (last) {
                wait_lgkm0();                               // this wave's last reads of `cur` are done,
                wait_vmcnt(REFILL ? LOADS * (ST - 2) : 0);  // and its loads of `nxt` have landed
                __builtin_amdgcn_s_barrier();
            }
#pragma unroll
            for (int u = 0; u < MU; ++u) {
                __builtin_amdgcn_sched_barrier(0);
                mul(u, s & 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int f = u * RPM; f < (u + 1) * RPM && f < FR; ++f)
                    frag(f, last ? nxt : cur, (s + 1) & 1, last ? 0 : s + 1);
                if (last && REFILL) {
#pragma unroll
                    for (int j = u * LOADS / MU; j < (u + 1) * LOADS / MU; ++j) load(j, src, cur);
                }
            }
        }
        cur = nxt;
    };
    int kt = 0;
#pragma unroll 1
    for (; kt + ST < nk; ++kt) step(kt, std::true_type{});
#pragma unroll 1
    for (; kt < nk; ++kt) step(kt, std::false_type{});

    float* const cs = (float*)smem;
    // 64 rows at a time through LDS. Lane holds C[m = 32 x + lane % 32][n = 32 y + 8 q + 4 (lane / 32) + e] in acc[4 q + e].
#pragma unroll
    for (int h = 0; h < BM / CH; ++h) {
        lds_barrier();
#pragma unroll
        for (int x = 0; x < TM; ++x) {
            const int row = wm * (BM / WM) + x * 32 + (lane & 31) - h * CH;
            if (row < 0 || row >= CH) continue;
#pragma unroll
            for (int y = 0; y < TN; ++y)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    f32x4_t v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[e] = acc[0][x][y][4 * q + e];
                        if constexpr (SUMS == 3) v[e] = (v[e] + acc[1][x][y][4 * q + e]) + acc[2][x][y][4 * q + e];
                    }
                    *(f32x4_t*)(cs + (kw * CH + row) * CP + wn * (BM / WN) + y * 32 + 8 * q + 4 * (lane >> 5)) = v;
                }
        }
        lds_barrier();
#pragma unroll(AHEAD > 0 ? AHEAD : 1)
        for (int u = 0; u < CH * (BM / 8) / THREADS; ++u) {
            const int q = tid + u * THREADS, r = q / (BM / 8), c = q % (BM / 8) * 8;
            const int64_t m = m0 + h * CH + r, n = n0 + c;
            if (m >= p.M || n >= p.N) continue;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = cs[r * CP + c + e];
#pragma unroll
                for (int g = 1; g < KW; ++g) v[e] += cs[(g * CH + r) * CP + c + e];  // (the wave groups' sums)
                v[e] *= scale;
            }
            if constexpr (EPI == STEP) {
                step_elements(b.s, b.d[i], f, m, n, v);
                continue;
            }
            if constexpr (EPI == POLY) {
                float hi[8], lo[8];
                if constexpr (AHEAD > 0) {
                    unpack_f16x8(ahead[u][0], hi);
                    unpack_f16x8(ahead[u][1], lo);
                } else {
                    unpack_f16x8(*(const u32x4_t*)(p.aux + m * p.N + n), hi);
                    unpack_f16x8(*(const u32x4_t*)(p.aux + plane + m * p.N + n), lo);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = fmaf(pc, v[e], fmaf(pb, hi[e] + lo[e], m == n + e ? pa : 0.f));
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] *= out;
                if (SYM) cs[r * CP + c + e] = v[e];
            }
            // (a block on the diagonal is its lower half, twice: the matrix is symmetric to the bit)
            store_pair(p.c + m * p.N + n, plane, v, 0, diagonal ? (int)(m - n) + 1 : 8);
        }
        if constexpr (SYM) {  // the block above the diagonal: rows n, columns m
            lds_barrier();
            for (int q = tid; q < BM * (CH / 8); q += THREADS) {
                const int r = q / (CH / 8), c = q % (CH / 8) * 8;
                const int64_t n = n0 + r, m = m0 + h * CH + c;
                if (m >= p.M || n >= p.N) continue;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = cs[(c + e) * CP + r];
                store_pair(p.c + n * p.N + m, plane, v, diagonal ? (int)(n - m) + 1 : 0, 8);
            }
        }
    }
}

// Which operands' rows are K-strided, and what becomes of the sums.
//   SQUARE, QUARTIC  products of symmetric matrices (symmetric too), QUARTIC with the polynomial in its epilogue
//   GRAM             X X^T, or X^T X of a tall matrix
//   NEXT, LAST       P X, or X P of a tall matrix: the next X, or the weights' step
enum { SQUARE = 0, QUARTIC = 1, OF_X = 2, NEXT = 3, LAST = 4 };

template <int BM, int WM, int WN, int KW, int KB, int ST, int KIND>
__global__ __launch_bounds__(64 * WM * WN * KW) void k_muon_product(Products b) {
    __shared__ __attribute__((aligned(1024))) bf16_t smem[ST * 4 * BM * KB];
    int block = xcd_remap(blockIdx.x, gridDim.x), quarter = -1;
    if (BM == 128 && b.from >= 0) {
        quarter = block & 3;
        block = b.from + (block >> 2);
    }
    const int i = entry_of(b.first, b.count, (uint32_t)block), t = block - (int)b.first[i];
    if constexpr (KIND == SQUARE) product_block<BM, WM, WN, KW, false, false, KB, ST, true, PAIR>(b, i, t, quarter, smem);
    else if constexpr (KIND == QUARTIC) product_block<BM, WM, WN, KW, false, false, KB, ST, true, POLY>(b, i, t, quarter, smem);
    else if constexpr (KIND == OF_X) {
        if (b.p[i].tall) product_block<BM, WM, WN, KW, true, true, KB, ST, true, PAIR>(b, i, t, quarter, smem);
        else product_block<BM, WM, WN, KW, false, false, KB, ST, true, PAIR>(b, i, t, quarter, smem);
    } else {
        constexpr int EPI = KIND == LAST ? STEP : PAIR;
        if (b.p[i].tall) product_block<BM, WM, WN, KW, false, false, KB, ST, false, EPI>(b, i, t, quarter, smem);
        else product_block<BM, WM, WN, KW, false, true, KB, ST, false, EPI>(b, i, t, quarter, smem);
    }
}

// The whole step of matrices whose shorter side is at most 64, a workgroup each: the 64 x 64 matrices stay in LDS, and X (in scratch, a
// pair, the shorter side's index first) is passed through by 64 columns at a time. A launch for each product would cost
// such a matrix 19 starts and ends of kernels of some 5 us.
constexpr int SMALL = 64, SMALL_LENGTH = 1024;
struct Small {
    Matrix t[PER_LAUNCH];
    MuonScalars a;
    MuonScales q;
};
static_assert(sizeof(Small) <= 4096, "kernel arguments");

// Whether X and A are made anew after step k.
__host__ __device__ inline bool anew_after(int k, int steps) { return k < steps - 1 && (k == 1 || (k > 1 && (k - 1) % 3 == 0)); }

// S: 64, or 32 for a shorter side of at most that (half of every sum, a quarter of the elements). Tiles of 16 x 16: what bounds a product here is the way from
// the sums through the pairs to the next product's fragments, so the elements are spread over all lanes (four of 32 x 160, 32 x 32 tiles of 64 x 64: 34 us,
// this 22; 64 x 64 24 and 22).
template <int S>
__global__ __launch_bounds__(256) void k_muon_small(Small b) {
    constexpr int E = SMALL * SMALL, CP = SMALL + 4;  // elements of a plane
    constexpr int TS = S / 32;                        // a wave's tiles, down, and in a square matrix across (a block of X: two)
    __shared__ __attribute__((aligned(1024))) bf16_t squares[4][2 * E];  // A, T A, T, P
    __shared__ __attribute__((aligned(1024))) bf16_t xk[2 * E];          // a block of X, K-contiguous along the longer side
    __shared__ __attribute__((aligned(1024))) bf16_t xs[2 * E];          // the same, K-strided along the shorter
    __shared__ __attribute__((aligned(16))) float cs[SMALL * CP];
    const Matrix t = b.t[blockIdx.x];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int down = (wave >> 1) * 16 * TS, along = (wave & 1) * 16 * TS, across = (wave & 1) * 32;  // the wave's first row, and column of either kind
    const bool tall = t.rows > t.cols;
    const int64_t length = tall ? t.rp : t.cp;  // of the longer side, padded
    float gs;
    const bool taken = gradient_scale(b.a, gs);
    const double sum = block_sum(momentum_range(t, b.a, gs, taken, 0, t.rows * t.cols));
    const double inv = sum == 0.0 ? 0.0 : (double)b.q.x[0] / sqrt(sum);

    // c = (add: c +) x y^T for pairs x (K-contiguous) and y, this wave's tiles of it, from column n0 on
    auto product = [&](const bf16_t* x, const bf16_t* y, auto strided, auto depth, bool add, int n0, auto& c) __attribute__((always_inline)) {
        constexpr bool KS = decltype(strided)::value;
        constexpr int TN = sizeof(c[0]) / sizeof(c[0][0]);
#pragma unroll
        for (int ks = 0; ks < decltype(depth)::value; ks += 32) {
            bf16x8_t xh[TS], xl[TS];
#pragma unroll
            for (int u = 0; u < TS; ++u) {
                xh[u] = load_frag<SMALL, false, SMALL>(x, down + 16 * u, ks, lane);
                xl[u] = load_frag<SMALL, false, SMALL>(x + E, down + 16 * u, ks, lane);
            }
#pragma unroll
            for (int w = 0; w < TN; ++w) {
                const bf16x8_t yh = load_frag<SMALL, KS, SMALL>(y, n0 + 16 * w, ks, lane);
                const bf16x8_t yl = load_frag<SMALL, KS, SMALL>(y + E, n0 + 16 * w, ks, lane);
#pragma unroll
                for (int u = 0; u < TS; ++u) {
                    if (ks == 0 && !add) {
#pragma unroll
                        for (int z = 0; z < 3; ++z) c[u][w][z] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                    }
                    c[u][w][0] = mfma16x16x32<true>(yl, xh[u], c[u][w][0]);
                    c[u][w][1] = mfma16x16x32<true>(yh, xl[u], c[u][w][1]);
                    c[u][w][2] = mfma16x16x32<true>(yh, xh[u], c[u][w][2]);
                }
            }
        }
    };
    const std::integral_constant<int, S> side{};
    const std::integral_constant<int, SMALL> block{};
    // f(row, column, values) for the four elements of each tile that a lane has
    auto each = [&](auto& c, int n0, auto f) __attribute__((always_inline)) {
        constexpr int TN = sizeof(c[0]) / sizeof(c[0][0]);
#pragma unroll
        for (int u = 0; u < TS; ++u)
#pragma unroll
            for (int w = 0; w < TN; ++w)
                f(down + 16 * u + (lane & 15), n0 + 16 * w + 4 * (lane >> 4), (c[u][w][0] + c[u][w][1]) + c[u][w][2]);
    };
    auto at = [](int r, int k) { return r * SMALL + (((k >> 3) ^ kc_swz<SMALL>(r)) * 8) + (k & 7); };  // K-contiguous
    auto strided_at = [](int k, int r) { return k * SMALL + (((r >> 4) ^ kstr_swz<SMALL>(k)) * 16) + (r & 15); };
    auto put4 = [&](bf16_t* x, int off, int64_t plane, const f32x4_t& v) __attribute__((always_inline)) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const _Float16 hi = (_Float16)v[e], lo = (_Float16)(v[e] - (float)hi);
            h[e] = __builtin_bit_cast(uint16_t, hi);
            l[e] = __builtin_bit_cast(uint16_t, lo);
        }
        *(uint2*)(x + off) = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
        *(uint2*)(x + off + plane) = make_uint2(l[0] | l[1] << 16, l[2] | l[3] << 16);
    };
    auto store = [&](bf16_t* x, auto& c, int n0, float scale) __attribute__((always_inline)) {
        each(c, n0, [&](int m, int n, const f32x4_t& v) __attribute__((always_inline)) { put4(x, at(m, n), E, v * scale); });
    };
    auto half_value = [](bf16_t x) { return (float)__builtin_bit_cast(_Float16, x); };

    // X0, and A from it
    f32x4_t gram[TS][TS][3], c[TS][TS][3], cx[TS][2][3];
    const int row = tid >> 2, first = (tid & 3) * 16;  // a thread's 16 values of a block's row
    for (int64_t l0 = 0; l0 < length; l0 += SMALL) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int k = first + 8 * u;
            float v[8];
            if (!tall) {
                x_elements(t, b.a, gs, taken, inv, row, l0 + k, v);
                store_pair(xk + at(row, k), E, v, 0, 8);
            } else {
                x_elements(t, b.a, gs, taken, inv, l0 + row, k, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const _Float16 hi = (_Float16)v[e], lo = (_Float16)(v[e] - (float)hi);
                    xk[at(k + e, row)] = __builtin_bit_cast(uint16_t, hi);
                    xk[E + at(k + e, row)] = __builtin_bit_cast(uint16_t, lo);
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u) {  // (hi and lo, two pieces each)
            const int k = first + 8 * (u & 1);
            *(u32x4_t*)(t.x + (u >> 1) * SMALL * length + row * length + l0 + k) = *(const u32x4_t*)(xk + (u >> 1) * E + at(row, k));
        }
        product(xk, xk, std::false_type{}, block, l0 > 0, along, gram);
    }
    bf16_t* const A = squares[0];
    bf16_t* const TA = squares[1];
    bf16_t *T = squares[2], *P = squares[3];
    store(A, gram, along, b.q.gram[0] / (b.q.x[0] * b.q.x[0]));
    __syncthreads();

    // a block of X as a K-strided operand, its loads ahead of the block in front
    u32x4_t ahead[4];
    auto fetch = [&](int64_t l0) {
#pragma unroll
        for (int u = 0; u < 4; ++u) ahead[u] = *(const u32x4_t*)(t.x + (u >> 1) * SMALL * length + row * length + l0 + first + 8 * (u & 1));
    };
    auto take_block = [&](int64_t l0) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u) *(u32x4_t*)(xs + (u >> 1) * E + strided_at(row, first + 8 * (u & 1))) = ahead[u];
        __syncthreads();
        if (l0 + SMALL < length) fetch(l0 + SMALL);
    };
    bool power = false;  // whether P stands (else it is I)
    float sx = b.q.x[0], sp = 1.f;
    const int steps = b.a.steps;
    for (int k = 0; k < steps; ++k) {
        const bool last = k == steps - 1, anew = anew_after(k, steps);
        const float sg = b.q.gram[k], st_ = b.q.poly[k];
        product(A, A, std::false_type{}, side, false, along, c);
        {
            const float pa = (float)b.a.a, pb = (float)b.a.b / sg, pc = (float)b.a.c / (sg * sg);
            each(c, along, [&](int m, int n, const f32x4_t& v) __attribute__((always_inline)) {
                f32x4_t p;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = half_value(A[at(m, n + e)]) + half_value(A[E + at(m, n + e)]);
                    p[e] = fmaf(pc, v[e], fmaf(pb, x, m == n + e ? pa : 0.f)) * st_;
                }
                put4(T, at(m, n), E, p);
            });
        }
        __syncthreads();
        if (!last && !anew) {
            product(T, A, std::false_type{}, side, false, along, c);
            store(TA, c, along, b.q.half[k] / (st_ * sg));
        }
        if (power) {
            product(T, P, std::false_type{}, side, false, along, c);
            __syncthreads();
            store(P, c, along, b.q.power[k] / (st_ * sp));
            sp = b.q.power[k];
            __syncthreads();
        }
        if (!last && !anew) {
            __syncthreads();
            product(T, TA, std::false_type{}, side, false, along, c);
            store(A, c, along, b.q.gram[k + 1] / (st_ * b.q.half[k]));
            __syncthreads();
        }
        if (!power) {
            bf16_t* const x = T;
            T = P;
            P = x;
            sp = st_;
            power = true;
        }
        if (!anew) continue;
        const float sn = b.q.x[k + 1];
        __syncthreads();
        fetch(0);
        for (int64_t l0 = 0; l0 < length; l0 += SMALL) {
            take_block(l0);
            product(P, xs, std::true_type{}, side, false, across, cx);
            each(cx, across, [&](int m, int n, const f32x4_t& v) __attribute__((always_inline)) {
                put4(xk, at(m, n), E, v * (sn / (sx * sp)));
                put4(t.x, (int)(m * length + l0) + n, SMALL * length, v * (sn / (sx * sp)));
            });
            __syncthreads();
            product(xk, xk, std::false_type{}, block, l0 > 0, along, gram);
        }
        sx = sn;
        power = false;
        __syncthreads();
        store(A, gram, along, b.q.gram[k + 1] / (sx * sx));
        __syncthreads();
    }
    StepFactors f;
    Destination d{t.param, t.master, t.rows, t.cols, t.scale, t.weight_decay, t.flags};
    if (!step_factors(b.a, d, f)) return;
    __syncthreads();
    fetch(0);
    for (int64_t l0 = 0; l0 < length; l0 += SMALL) {
        take_block(l0);
        product(P, xs, std::true_type{}, side, false, across, cx);
        each(cx, across, [&](int m, int n, const f32x4_t& v) __attribute__((always_inline)) { *(f32x4_t*)(cs + m * CP + n) = v * (1.f / (sx * sp)); });
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int k = first + 8 * u;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = tall ? cs[(k + e) * CP + row] : cs[row * CP + k + e];
            if (tall) step_elements(b.a, d, f, l0 + row, k, v);
            else step_elements(b.a, d, f, row, l0 + k, v);
        }
    }
}

// What the host knows of a matrix's scratch.
struct Layout {
    int64_t rp, cp, mp;
    bool tall;
    size_t x[2], square[NAMES], part, total;
    int64_t parts, per;
};
Layout layout(const MuonTensor& t, size_t at) {
    Layout l;
    l.rp = padded(t.rows);
    l.cp = padded(t.cols);
    l.tall = t.rows > t.cols;
    l.mp = l.tall ? l.cp : l.rp;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += (size_t)((bytes + 255) / 256 * 256);
        return here;
    };
    for (size_t& x : l.x) x = take(l.rp * l.cp * 4);
    for (size_t& q : l.square) q = take(l.mp * l.mp * 4);
    const int64_t n = t.rows * t.cols;
    l.per = std::max<int64_t>(PART, ((n + PARTS - 1) / PARTS + 2047) / 2048 * 2048);
    l.parts = (n + l.per - 1) / l.per;
    l.part = take(l.parts * 8);
    l.total = at;
    return l;
}

template <int KIND>
int64_t blocks_of(const Product& p, int side) {
    const int64_t tm = (p.M + side - 1) / side, tn = (p.N + side - 1) / side;
    return KIND <= OF_X ? tm * (tm + 1) / 2 : tm * tn;
}

// How a launch's products are cut: whichever is through first. `slots` blocks run at once; a K step of 64 takes them `full` us where
// all slots are taken, and base + slope * their share where fewer are. Fitted to times of all five plans, and of the large one with a tail, for each kind
// of product of twenty lists, 12 of 160 x 640 up to those of two layers of 4096 x 10624: the plans chosen make a list's step 0.7% slower than the best ones would on average, 3% at worst.
// (us of a squaring, in the order below: 2048^2 54 / 53 / 57 / 45 / 114; six of 1000^2 35 / 41 / 37 / 29 / 68; 4096^2 259 / 261 / 266 / 234 / 216, two of
// them 524 / 571 / 472 / 449 / 552 and 419 with a tail; and of the product with X of 4096^2 503 / 586 / 350 / 366 / 299.)
enum { SMALL_TWO, SMALL_DEEP, MIDDLE_TWO, MIDDLE_DEEP, LARGE };
struct Plan {
    int id, side, slots;
    double full, base, slope;
};
constexpr Plan PLANS[] = {{SMALL_TWO, 64, 512, 0.96, 0.52, 0.38},  // 64 KiB of LDS: two blocks a CU
                          {SMALL_DEEP, 64, 256, 0.52, 0.42, 0.02},  // a ring of four stages, one block a CU
                          {MIDDLE_TWO, 128, 512, 2.87, 1.32, 1.33},
                          {MIDDLE_DEEP, 128, 256, 1.54, 0.92, 0.61},  // stages of 64, eight waves in two groups along K
                          {LARGE, 256, 256, 4.59, 2.7, 1.82}};
constexpr double TAIL = 24.0;  // us, for a second launch

struct Share {  // blocks of a plan's side, and their K steps of 64
    double blocks = 0.0, steps = 0.0, longest = 0.0;
    void add(double n, double k) {
        blocks += n;
        steps += n * k;
        if (n > 0.0) longest = std::max(longest, k);
    }
};
double time_of(const Plan& q, const Share& x) {
    if (x.blocks == 0.0) return 0.0;
    const double rounds = std::floor(x.blocks / q.slots), rest = x.blocks / q.slots - rounds;
    return std::max(x.longest * (q.base + q.slope * std::min(1.0, x.blocks / q.slots)),  // (beside others, short ones too)
                    x.steps / x.blocks * (rounds * q.full + (rest > 0.0 ? q.base + q.slope * rest : 0.0)));
}

template <int KIND>
hipError_t launch_blocks(const Plan& plan, Products& b, uint32_t n, hipStream_t s) {
    // (the weights' step has more to do behind its sums: eight waves, 512 x 4352 eight times 105 -> 91 us; elsewhere four are as fast or faster)
    constexpr int MIDDLE_WN = KIND == LAST ? 4 : 2;
    switch (plan.id) {
        case LARGE: hipLaunchKernelGGL((k_muon_product<256, 2, 4, 1, 32, 2, KIND>), dim3(n), dim3(512), 0, s, b); break;
        case MIDDLE_TWO: hipLaunchKernelGGL((k_muon_product<128, 2, MIDDLE_WN, 1, 32, 2, KIND>), dim3(n), dim3(128 * MIDDLE_WN), 0, s, b); break;
        case MIDDLE_DEEP: hipLaunchKernelGGL((k_muon_product<128, 2, 2, 2, 64, 2, KIND>), dim3(n), dim3(512), 0, s, b); break;
        case SMALL_DEEP: hipLaunchKernelGGL((k_muon_product<64, 2, 2, 2, 64, 4, KIND>), dim3(n), dim3(512), 0, s, b); break;
        default: hipLaunchKernelGGL((k_muon_product<64, 2, 2, 2, 64, 2, KIND>), dim3(n), dim3(512), 0, s, b); break;
    }
    return hipGetLastError();
}

template <int KIND>
hipError_t launch_products(Products& b, hipStream_t s) {
    if (b.count == 0) return hipSuccess;
    const Plan* head = nullptr;
    const Plan* tail = nullptr;
    double least = 0.0;
    for (const Plan& q : PLANS) {
        Share x;
        for (int i = 0; i < b.count; ++i) x.add((double)blocks_of<KIND>(b.p[i], q.side), b.p[i].K / 64.0);
        const double us = time_of(q, x);
        if (!head || us < least) {
            head = &q;
            least = us;
        }
    }
    // Whole rounds of the largest blocks, which take the fewest loads, and what is left of them in a launch of its own, in quarters, so that the
    // last round is not one of a few blocks (two of 4096 x 10624 and two of 2048 x 10624: 344 blocks on 256 CUs, 552 -> 474 us a squaring, the step 15.8 -> 14.2 ms)
    const Plan& large = PLANS[LARGE];
    int64_t blocks = 0;
    for (int i = 0; i < b.count; ++i) blocks += blocks_of<KIND>(b.p[i], large.side);
    const int64_t whole = blocks / large.slots * large.slots;
    if (whole > 0 && whole < blocks) {
        Share x, y;
        int64_t free = whole;
        for (int i = 0; i < b.count; ++i) {
            const int64_t n = blocks_of<KIND>(b.p[i], large.side), m = std::min(n, free);
            free -= m;
            x.add((double)m, b.p[i].K / 64.0);
            y.add(4.0 * (double)(n - m), b.p[i].K / 64.0);
        }
        for (int id : {MIDDLE_TWO, MIDDLE_DEEP}) {
            const double us = time_of(large, x) + time_of(PLANS[id], y) + TAIL;
            if (us < least) {
                head = &large;
                tail = &PLANS[id];
                least = us;
            }
        }
    }
    uint32_t n = 0;
    for (int i = 0; i < b.count; ++i) {
        b.first[i] = n;
        n += (uint32_t)blocks_of<KIND>(b.p[i], head->side);
    }
    b.first[b.count] = n;
    b.from = -1;
    hipError_t e = launch_blocks<KIND>(*head, b, tail ? (uint32_t)whole : n, s);
    if (e != hipSuccess || !tail) return e;
    b.from = (int)whole;
    return launch_blocks<KIND>(*tail, b, 4 * (n - (uint32_t)whole), s);
}

}  // namespace

bool muon_scales(double a, double b, double c, int steps, MuonScales* out) {
    // the largest power of two that keeps values up to `bound` within half of f16's range
    auto power = [](double bound) { return std::exp2(std::floor(std::log2(32768.0 / std::max(bound, 1.0 / 32768.0)))); };
    auto poly = [&](double l) { return a + b * l + c * l * l; };
    double most = 1.0, p = 1.0;  // the largest eigenvalue of A, and of P
    out->x[0] = 32768.f;
    for (int k = 0; k < steps; ++k) {
        double t = 0.0, next = 0.0, half = 0.0;
        for (int i = 0; i <= 4096; ++i) {
            const double l = most * i / 4096.0, v = std::fabs(poly(l));
            t = std::max(t, v);
            half = std::max(half, l * v);
            next = std::max(next, l * v * v);
        }
        // between the samples, and for rounding
        t *= 1.01; half *= 1.01; next *= 1.01;
        if (k == 2 || (k > 2 && (k - 2) % 3 == 0)) p = 1.0;
        p *= t;
        if (!(p < 1e6) || !(next < 64.0)) return false;
        out->gram[k] = (float)power(most);
        out->poly[k] = (float)power(t);
        out->half[k] = (float)power(half);
        out->power[k] = (float)power(p);
        most = next;
        out->x[k + 1] = (float)power(std::sqrt(next));
    }
    return true;
}

namespace {

// The launches of up to PER_LAUNCH / 2 matrices.
void fill(Matrix& m, const MuonTensor& t, const Layout& l, char* sc) {
    m.grad = t.grad; m.m = t.m; m.param = t.param; m.master = t.master;
    m.x = (uint16_t*)(sc + l.x[0]);
    m.part = (double*)(sc + l.part);
    m.rows = t.rows; m.cols = t.cols;
    m.rp = (int32_t)l.rp; m.cp = (int32_t)l.cp;
    m.parts = (int32_t)l.parts; m.per = (int32_t)l.per;
    m.flags = t.flags;
    m.weight_decay = (float)t.weight_decay; m.scale = t.scale;
}

// Matrices that one workgroup is through with sooner than many are with theirs, launch by launch.
bool is_small(const MuonTensor& t) { return std::min(t.rows, t.cols) <= SMALL && std::max(t.rows, t.cols) <= SMALL_LENGTH; }

hipError_t run_batch(const MuonTensor* t, const Layout* l, int count, const MuonScalars& a, const MuonScales& q, char* sc,
                     hipStream_t s) {
    hipError_t e;
    if (std::all_of(t, t + count, is_small)) {  // (beside larger ones they cost nothing in those's launches)
        Small b;
        b.a = a;
        b.q = q;
        for (int i = 0; i < count; ++i) fill(b.t[i], t[i], l[i], sc);
        if (std::all_of(t, t + count, [](const MuonTensor& x) { return std::min(x.rows, x.cols) <= 32; }))
            hipLaunchKernelGGL(k_muon_small<32>, dim3((unsigned)count), dim3(256), 0, s, b);
        else hipLaunchKernelGGL(k_muon_small<64>, dim3((unsigned)count), dim3(256), 0, s, b);
        return hipGetLastError();
    }
    {
        Elements b;
        b.a = a;
        b.count = count;
        b.scale = q.x[0];
        uint32_t n = 0;
        for (int i = 0; i < count; ++i) {
            fill(b.t[i], t[i], l[i], sc);
            b.first[i] = n;
            n += (uint32_t)l[i].parts;
        }
        b.first[count] = n;
        hipLaunchKernelGGL(k_muon_momentum, dim3(n), dim3(256), 0, s, b);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        n = 0;
        for (int i = 0; i < count; ++i) {
            b.first[i] = n;
            n += (uint32_t)((l[i].rp + SPLIT_ROWS - 1) / SPLIT_ROWS * ((l[i].cp + SPLIT_COLS - 1) / SPLIT_COLS));
        }
        b.first[count] = n;
        hipLaunchKernelGGL(k_muon_split, dim3(n), dim3(256), 0, s, b);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    Products b;
    b.s = a;
    auto square = [&](int i, int name) { return (uint16_t*)(sc + l[i].square[name]); };
    auto begin = [&]() {
        b.count = 0;
        b.second = PER_LAUNCH;
    };
    // C = A B of two symmetric matrices
    auto add = [&](int i, int x, int y, int c) {
        Product& p = b.p[b.count++];
        p = Product{};
        p.a = square(i, x); p.b = square(i, y); p.c = square(i, c);
        p.ap = p.bp = l[i].mp * l[i].mp;
        p.lda = p.ldb = p.M = p.N = p.K = (int32_t)l[i].mp;
    };
    // A from X
    auto gram = [&](int x, float sx, float sa) {
        begin();
        b.scale = 1.f / (sx * sx);
        b.out = sa;
        for (int i = 0; i < count; ++i) {
            Product& p = b.p[b.count++];
            p = Product{};
            p.tall = l[i].tall;
            p.a = p.b = (uint16_t*)(sc + l[i].x[x]);
            p.ap = p.bp = l[i].rp * l[i].cp;
            p.lda = p.ldb = (int32_t)l[i].cp;
            p.M = p.N = (int32_t)l[i].mp;
            p.K = (int32_t)(l[i].tall ? l[i].rp : l[i].cp);
            p.c = square(i, GRAM);
        }
        return launch_products<OF_X>(b, s);
    };
    // P X (X P of a tall matrix): the next X, or the weights' step
    auto apply = [&](int x, int pw, float sx, float sp, float out, bool step) {
        begin();
        b.scale = 1.f / (sx * sp);
        b.out = out;
        for (int i = 0; i < count; ++i) {
            const bool tall = l[i].tall;
            const uint16_t* const xs = (uint16_t*)(sc + l[i].x[x]);
            const int64_t xp = l[i].rp * l[i].cp, pp = l[i].mp * l[i].mp;
            b.d[b.count] = Destination{t[i].param, t[i].master, t[i].rows, t[i].cols, t[i].scale, (float)t[i].weight_decay, t[i].flags};
            Product& p = b.p[b.count++];
            p = Product{};
            p.tall = tall;
            p.a = tall ? xs : square(i, pw); p.ap = tall ? xp : pp;
            p.b = tall ? square(i, pw) : xs; p.bp = tall ? pp : xp;
            p.lda = (int32_t)(tall ? l[i].cp : l[i].mp);
            p.ldb = (int32_t)(tall ? l[i].mp : l[i].cp);
            p.M = (int32_t)l[i].rp; p.N = (int32_t)l[i].cp; p.K = (int32_t)l[i].mp;
            p.c = (uint16_t*)(sc + l[i].x[1 - x]);
        }
        return step ? launch_products<LAST>(b, s) : launch_products<NEXT>(b, s);
    };

    int x = 0, power = -1;  // the X that stands, and the name of P (none yet: I)
    float sx = q.x[0], sp = 1.f;
    if ((e = gram(x, sx, q.gram[0])) != hipSuccess) return e;
    for (int k = 0; k < a.steps; ++k) {
        const bool last = k == a.steps - 1, anew = anew_after(k, a.steps);
        int poly = FREE;
        while (poly == power) ++poly;
        begin();
        for (int i = 0; i < count; ++i) {
            add(i, GRAM, GRAM, poly);
            b.p[i].aux = square(i, GRAM);
        }
        b.scale = 1.f / (q.gram[k] * q.gram[k]);
        b.out = q.poly[k];
        b.pa = (float)a.a; b.pb = (float)(a.b / q.gram[k]); b.pc = (float)a.c;
        if ((e = launch_products<QUARTIC>(b, s)) != hipSuccess) return e;
        // T A (where another A follows) and T P beside it
        begin();
        if (!last && !anew)
            for (int i = 0; i < count; ++i) add(i, poly, GRAM, HALF);
        b.scale = 1.f / (q.poly[k] * q.gram[k]);
        b.out = q.half[k];
        int next = poly;
        if (power >= 0) {
            b.second = b.count;
            b.scale2 = 1.f / (q.poly[k] * sp);
            b.out2 = q.power[k];
            next = FREE;
            while (next == poly || next == power) ++next;
            for (int i = 0; i < count; ++i) add(i, poly, power, next);
        }
        if (b.count && (e = launch_products<SQUARE>(b, s)) != hipSuccess) return e;
        sp = power >= 0 ? q.power[k] : q.poly[k];
        power = next;
        if (anew) {
            if ((e = apply(x, power, sx, sp, q.x[k + 1], false)) != hipSuccess) return e;
            x = 1 - x;
            sx = q.x[k + 1];
            power = -1;
            if ((e = gram(x, sx, q.gram[k + 1])) != hipSuccess) return e;
        } else if (!last) {
            begin();
            for (int i = 0; i < count; ++i) add(i, poly, HALF, GRAM);
            b.scale = 1.f / (q.poly[k] * q.half[k]);
            b.out = q.gram[k + 1];
            if ((e = launch_products<SQUARE>(b, s)) != hipSuccess) return e;
        }
    }
    return apply(x, power, sx, sp, 1.f, true);
}

// The matrices of one run of launches, from t[i] on: up to PER_LAUNCH / 2 of them, with grids that can be launched. Their
// scratch lies at the beginning of the caller's: runs follow each other on one stream.
struct Run {
    MuonTensor t[PER_LAUNCH / 2];
    Layout l[PER_LAUNCH / 2];
    int count;
    size_t total;
};
int next_run(const MuonTensor* t, int i, int count, Run* r) {
    r->count = 0;
    r->total = 0;
    int64_t blocks = 0;
    for (; i < count && r->count < PER_LAUNCH / 2; ++i) {
        if (t[i].rows <= 0 || t[i].cols <= 0) continue;
        const int64_t n = padded(t[i].rows) / 64 * (padded(t[i].cols) / 64);
        if (r->count > 0 && blocks + n > (int64_t)1 << 22) break;
        blocks += n;
        r->t[r->count++] = t[i];
    }
    // those with the longest sums first: a launch's last blocks are then short ones
    std::sort(r->t, r->t + r->count, [](const MuonTensor& x, const MuonTensor& y) {
        const int64_t a = std::min(x.rows, x.cols), b = std::min(y.rows, y.cols);
        return a != b ? a > b : x.flags < y.flags;
    });
    for (int k = 0; k < r->count; ++k) {
        r->l[k] = layout(r->t[k], r->total);
        r->total = r->l[k].total;
    }
    return i;
}

}  // namespace

size_t muon_scratch(const MuonTensor* t, int count) {
    size_t most = 0;
    Run r;
    for (int i = 0; i < count;) {
        i = next_run(t, i, count, &r);
        most = std::max(most, r.total);
    }
    return most;
}

hipError_t launch_muon(const MuonTensor* t, int count, const MuonScalars& a, const MuonScales& q, void* scratch, hipStream_t s) {
    Run r;
    for (int i = 0; i < count;) {
        i = next_run(t, i, count, &r);
        if (r.count == 0) break;
        const hipError_t e = run_batch(r.t, r.l, r.count, a, q, (char*)scratch, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace rdcn
