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
// then on (6 n/m + 14 m^3 for five steps). The error of X over ranges of spectra (relative, five steps): restarted 2e-6 to 4e-5, never
// 2e-6 to 4e-4, float products of X itself 2e-6 to 1e-5.
//
// Operands. Every matrix stands as a pair of f16, hi + lo of a power of two times its values (22 bits), and a product is three of f16 matrix
// instructions: hi hi + hi lo + lo hi, sums in float. (One f16 each would leave 3e-3 to 5e-1 of X in error, bf16 more; float
// matrix instructions run at a sixteenth of the rate.) The powers keep all values below f16's range: |A| <= 1 for X of norm 1, and what
// follows is bounded by the polynomial's largest value on the singular values' range (muon_scales). Matrices are padded with zeros to
// multiples of 64: zero rows stay zero rows of X, and no load needs a bound.
#include <algorithm>
#include <cmath>

#include "device_common.h"
#include "mfma_tiles.h"
#include "muon.h"

namespace rdcn {

namespace {

constexpr int PAD = 64;              // sides are padded to multiples of this
constexpr int PARTS = 1024;          // most partial sums of a matrix's norm
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

__device__ __forceinline__ int entry_of(const uint32_t* first, int count, uint32_t b) {
    int i = 0;
    while (i + 1 < count && first[i + 1] <= b) ++i;
    return i;
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

__device__ __forceinline__ float grad_at(const Matrix& t, int64_t i) {
    return t.flags & MUON_GRAD_BF16 ? bf16_to_f32(((const bf16_t*)t.grad)[i]) : ((const float*)t.grad)[i];
}
__device__ __forceinline__ float update_of(const MuonScalars& a, float m, float g) {
#pragma clang fp contract(off)
    return a.nesterov ? m * a.mu + g * a.c1 : m;
}

// M' and the partial sums of |U|^2, in 64 bits: the squares of floats cannot overflow there, or vanish.
__global__ __launch_bounds__(256) void k_muon_momentum(Elements b) {
#pragma clang fp contract(off)
    float gs;
    const bool taken = gradient_scale(b.a, gs);
    const int i = entry_of(b.first, b.count, blockIdx.x);
    const Matrix& t = b.t[i];
    const int64_t n = t.rows * t.cols, from = (int64_t)(blockIdx.x - b.first[i]) * t.per;
    const int64_t to = from + t.per < n ? from + t.per : n;
    double s = 0.0;
    for (int64_t k = from + threadIdx.x; k < to; k += 256) {
        const float g = grad_at(t, k) * gs, m = t.m[k] * b.a.mu + g * b.a.c1;
        if (taken) t.m[k] = m;
        const double u = (double)update_of(b.a, m, g);
        s = fma(u, u, s);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) t.part[blockIdx.x - b.first[i]] = s;
}

// X = U / |U| as a pair of f16, padded with zeros; a workgroup per 64 x 64 block.
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
    const int block = (int)(blockIdx.x - b.first[i]), tiles = t.cp / 64;
    const int r0 = block / tiles * 64, c = block % tiles * 64 + (threadIdx.x & 63);
    const int64_t plane = (int64_t)t.rp * t.cp;
    for (int r = r0 + (threadIdx.x >> 6); r < r0 + 64; r += 4) {
        float v = 0.f;
        if (taken && r < t.rows && c < t.cols) {
            const int64_t k = (int64_t)r * t.cols + c;
            v = (float)((double)update_of(b.a, t.m[k], grad_at(t, k) * gs) * inv);
        }
        const _Float16 hi = (_Float16)v, lo = (_Float16)(v - (float)hi);
        t.x[(int64_t)r * t.cp + c] = __builtin_bit_cast(uint16_t, hi);
        t.x[plane + (int64_t)r * t.cp + c] = __builtin_bit_cast(uint16_t, lo);
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
    int32_t matrix;          // STEP: its place in the launch's matrices
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

struct Products {
    Product p[PER_LAUNCH];
    uint32_t first[PER_LAUNCH + 1];
    int count;
    float scale;             // of the sum: what the operands were held times, undone
    float out;               // what c is held times
    float pa, pb, pc;        // POLY: pa I + pb aux + pc sum, aux as it is held
    float scale2, out2;      // of the products from `second` on
    int second;
    Destination d[PER_LAUNCH];
    MuonScalars s;
};
static_assert(sizeof(Products) <= 4096, "kernel arguments");

template <int BM, int BN, bool AKS, bool BKS, int KB, int ST, bool SYM, int EPI>
__global__ __launch_bounds__(256) void k_muon_product(Products b) {
    constexpr int NW = 4, NIA = BM * KB / (512 * NW), NIB = BN * KB / (512 * NW), LOADS = 2 * (NIA + NIB);
    constexpr int TM = BM / 64, TN = BN / 64, CP = BN + 4;
    constexpr int EA = BM * KB, EB = BN * KB, STAGE = 2 * (EA + EB);  // a stage: A hi, A lo, B hi, B lo
    static_assert(BM * CP * 4 <= ST * STAGE * 2, "the block's staged sums fit the ring");
    __shared__ __attribute__((aligned(1024))) bf16_t smem[ST * STAGE];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
    const int block = xcd_remap(blockIdx.x, gridDim.x);
    const int i = entry_of(b.first, b.count, (uint32_t)block);
    const Product& p = b.p[i];
    const int t = block - (int)b.first[i], tiles_n = (p.N + BN - 1) / BN;
    int tm, tn;
    if constexpr (SYM) {  // t = tm (tm + 1) / 2 + tn, tn <= tm
        tm = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
        while (tm * (tm + 1) / 2 > t) --tm;
        while ((tm + 1) * (tm + 2) / 2 <= t) ++tm;
        tn = t - tm * (tm + 1) / 2;
    } else {
        tm = t / tiles_n;
        tn = t % tiles_n;
    }
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;

    uint32_t aoff[NIA], boff[NIB];
    stage_offsets<BM, AKS, NW, KB>(p.lda, p.M, m0, m0, wave, lane, aoff);
    stage_offsets<BN, BKS, NW, KB>(p.ldb, p.N, n0, n0, wave, lane, boff);
    const int nk = p.K / KB;
    auto issue = [&](int kt) __attribute__((always_inline)) {
        const int64_t k0 = (int64_t)(kt < nk ? kt : nk - 1) * KB;  // (past the last stage it is read again)
        const uint16_t* const a = p.a + (AKS ? k0 * p.lda + m0 : m0 * p.lda + k0);
        const uint16_t* const bb = p.b + (BKS ? k0 * p.ldb + n0 : n0 * p.ldb + k0);
        const uint32_t base = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_addr(smem + kt % ST * STAGE));
        const uint32_t wa = (uint32_t)__builtin_amdgcn_readfirstlane(wave * NIA) * 1024u;
        const uint32_t wb = (uint32_t)__builtin_amdgcn_readfirstlane(wave * NIB) * 1024u;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const void* const sa = uniform_ptr(a + q * p.ap);
            const void* const sb = uniform_ptr(bb + q * p.bp);
#pragma unroll
            for (int j = 0; j < NIA; ++j) dma16_s(aoff[j], sa, base + q * EA * 2u + wa + 1024u * j);
#pragma unroll
            for (int j = 0; j < NIB; ++j) dma16_s(boff[j], sb, base + 4u * EA + q * EB * 2u + wb + 1024u * j);
        }
    };
    f32x16_t acc[TM][TN];
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int y = 0; y < TN; ++y)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[x][y][e] = 0.f;
#pragma unroll
    for (int u = 0; u < ST - 1; ++u) issue(u);
    const uint32_t fa = frag_base<BM, AKS, KB>(smem, wm * (BM / 2), lane);
    const uint32_t fb = frag_base<BN, BKS, KB>(smem + 2 * EA, wn * (BN / 2), lane);
    for (int kt = 0; kt < nk; ++kt) {
        wait_vmcnt(LOADS * (ST - 2));
        __builtin_amdgcn_s_barrier();
        issue(kt + ST - 1);
        const uint32_t off = (uint32_t)(kt % ST) * (STAGE * 2u);
#pragma unroll
        for (int s = 0; s < KB / 16; ++s) {
            bf16x8_t ah[TM], al[TM], bh[TN], bl[TN];
#pragma unroll
            for (int x = 0; x < TM; ++x) {
                ah[x] = frag_at<BM, AKS, KB>(fa, off, x, s);
                al[x] = frag_at<BM, AKS, KB>(fa, off + EA * 2u, x, s);
            }
#pragma unroll
            for (int y = 0; y < TN; ++y) {
                bh[y] = frag_at<BN, BKS, KB>(fb, off, y, s);
                bl[y] = frag_at<BN, BKS, KB>(fb, off + EB * 2u, y, s);
            }
#pragma unroll
            for (int x = 0; x < TM; ++x)
#pragma unroll
                for (int y = 0; y < TN; ++y) {
                    acc[x][y] = mfma32x32x16<true>(bl[y], ah[x], acc[x][y]);
                    acc[x][y] = mfma32x32x16<true>(bh[y], al[x], acc[x][y]);
                    acc[x][y] = mfma32x32x16<true>(bh[y], ah[x], acc[x][y]);
                }
        }
    }
    wait_vmcnt(0);  // the loads that were issued past the end have landed
    __syncthreads();
    // lane holds C[m = 32 x + lane % 32][n = 32 y + 8 q + 4 (lane / 32) + e] in acc[4 q + e]
    float* const cs = (float*)smem;
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int y = 0; y < TN; ++y)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(f32x4_t*)(cs + (wm * (BM / 2) + x * 32 + (lane & 31)) * CP + wn * (BN / 2) + y * 32 + 8 * q + 4 * (lane >> 5)) =
                    f32x4_t{acc[x][y][4 * q], acc[x][y][4 * q + 1], acc[x][y][4 * q + 2], acc[x][y][4 * q + 3]};
    __syncthreads();
    if constexpr (EPI == STEP) {
        const Destination& d = b.d[p.matrix];
        float gs;
        if (!gradient_scale(b.s, gs)) return;
        const double lr = b.s.device_lr ? (double)*b.s.device_lr : b.s.lr;
        const float decay = (float)(1.0 - lr * (double)d.weight_decay), size = (float)(lr * d.scale);
        uint32_t seed = b.s.seed;
        if (b.s.device_step) {  // a step that is replayed draws anew
            int64_t st = *b.s.device_step;
            seed += (uint32_t)(st < 1 ? 1 : st) * 0x85EBCA6Bu;
        }
        const uint32_t key = seed + 0x9E3779B9u * ((d.flags >> MUON_ORDINAL) + 1u);
        const bool pbf = d.flags & MUON_PARAM_BF16;
        for (int q = tid; q < BM * BN; q += 256) {
#pragma clang fp contract(off)
            const int64_t m = m0 + q / BN, n = n0 + q % BN;
            if (m >= d.rows || n >= d.cols) continue;
            const int64_t at = m * d.cols + n;
            float v = d.master ? d.master[at] : pbf ? bf16_to_f32(((const bf16_t*)d.param)[at]) : ((const float*)d.param)[at];
            v = v * decay - (cs[q / BN * CP + q % BN] * b.scale) * size;
            if (d.master) d.master[at] = v;
            if (!pbf) {
                ((float*)d.param)[at] = v;
            } else if (b.s.stochastic && !d.master) {
                const uint32_t h = fmix32((uint32_t)at ^ key);
                const uint32_t r = (__float_as_uint(v) + ((h * 0x85EBCA6Bu) >> 16)) >> 16;
                ((bf16_t*)d.param)[at] = (bf16_t)(v == v ? r : 0x7FC0u);  // (a NaN's bits could carry into its sign)
            } else {
                ((bf16_t*)d.param)[at] = (bf16_t)f32_to_bf16(v);
            }
        }
    } else {
        const int64_t plane = (int64_t)p.M * p.N;
        const float scale = i >= b.second ? b.scale2 : b.scale, out = i >= b.second ? b.out2 : b.out;
        const bool diagonal = SYM && tm == tn;
        auto put = [&](int64_t at, const float* v) __attribute__((always_inline)) {
            bool ovf = false;
            float hi[8], lo[8];
            const u32x4_t h = pack_f16x8(v, ovf);
            unpack_f16x8(h, hi);
#pragma unroll
            for (int e = 0; e < 8; ++e) lo[e] = v[e] - hi[e];
            *(u32x4_t*)(p.c + at) = h;
            *(u32x4_t*)(p.c + plane + at) = pack_f16x8(lo, ovf);
        };
        for (int q = tid; q < BM * (BN / 8); q += 256) {
            const int r = q / (BN / 8), c = q % (BN / 8) * 8;
            const int64_t m = m0 + r, n = n0 + c;
            if (m >= p.M || n >= p.N) continue;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // (a block on the diagonal is its lower half, twice: the matrix is symmetric to the bit)
                const float x = diagonal && c + e > r ? cs[(c + e) * CP + r] : cs[r * CP + c + e];
                v[e] = x * scale;
            }
            if constexpr (EPI == POLY) {
                float h[8], l[8];
                unpack_f16x8(*(const u32x4_t*)(p.aux + m * p.N + n), h);
                unpack_f16x8(*(const u32x4_t*)(p.aux + plane + m * p.N + n), l);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = fmaf(b.pc, v[e], fmaf(b.pb, h[e] + l[e], m == n + e ? b.pa : 0.f));
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] *= out;
                if (SYM && !diagonal) cs[r * CP + c + e] = v[e];
            }
            put(m * p.N + n, v);
        }
        if (SYM && !diagonal) {  // the block above the diagonal: rows n, columns m
            __syncthreads();
            for (int q = tid; q < BN * (BM / 8); q += 256) {
                const int r = q / (BM / 8), c = q % (BM / 8) * 8;
                const int64_t n = n0 + r, m = m0 + c;
                if (m >= p.M || n >= p.N) continue;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = cs[(c + e) * CP + r];
                put(n * p.N + m, v);
            }
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
    l.per = std::max<int64_t>(2048, (n + PARTS - 1) / PARTS);
    l.parts = (n + l.per - 1) / l.per;
    l.part = take(l.parts * 8);
    l.total = at;
    return l;
}

template <bool SYM, int EPI, bool AKS, bool BKS>
hipError_t launch_products(Products& b, hipStream_t s) {
    uint32_t n = 0;
    for (int i = 0; i < b.count; ++i) {
        b.first[i] = n;
        const int64_t tm = b.p[i].M / 64, tn = b.p[i].N / 64;
        n += (uint32_t)(SYM ? tm * (tm + 1) / 2 : tm * tn);
    }
    b.first[b.count] = n;
    if (n == 0) return hipSuccess;
    hipLaunchKernelGGL((k_muon_product<64, 64, AKS, BKS, 64, 3, SYM, EPI>), dim3(n), dim3(256), 0, s, b);
    return hipGetLastError();
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
hipError_t run_batch(const MuonTensor* t, const Layout* l, int count, const MuonScalars& a, const MuonScales& q, char* sc,
                     hipStream_t s) {
    hipError_t e;
    {
        Elements b;
        b.a = a;
        b.count = count;
        b.scale = q.x[0];
        uint32_t n = 0;
        for (int i = 0; i < count; ++i) {
            Matrix& m = b.t[i];
            m.grad = t[i].grad; m.m = t[i].m; m.param = t[i].param; m.master = t[i].master;
            m.x = (uint16_t*)(sc + l[i].x[0]);
            m.part = (double*)(sc + l[i].part);
            m.rows = t[i].rows; m.cols = t[i].cols;
            m.rp = (int32_t)l[i].rp; m.cp = (int32_t)l[i].cp;
            m.parts = (int32_t)l[i].parts; m.per = (int32_t)l[i].per;
            m.flags = t[i].flags;
            m.weight_decay = (float)t[i].weight_decay; m.scale = t[i].scale;
            b.first[i] = n;
            n += (uint32_t)l[i].parts;
        }
        b.first[count] = n;
        hipLaunchKernelGGL(k_muon_momentum, dim3(n), dim3(256), 0, s, b);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        n = 0;
        for (int i = 0; i < count; ++i) {
            b.first[i] = n;
            n += (uint32_t)((l[i].rp / 64) * (l[i].cp / 64));
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
    auto gram = [&](int x, float sx, float sa) -> hipError_t {
        for (int tall = 0; tall < 2; ++tall) {
            begin();
            b.scale = 1.f / (sx * sx);
            b.out = sa;
            for (int i = 0; i < count; ++i) {
                if (l[i].tall != (tall == 1)) continue;
                Product& p = b.p[b.count++];
                p = Product{};
                p.a = p.b = (uint16_t*)(sc + l[i].x[x]);
                p.ap = p.bp = l[i].rp * l[i].cp;
                p.lda = p.ldb = (int32_t)l[i].cp;
                p.M = p.N = (int32_t)l[i].mp;
                p.K = (int32_t)(tall ? l[i].rp : l[i].cp);
                p.c = square(i, GRAM);
            }
            const hipError_t r = tall ? launch_products<true, PAIR, true, true>(b, s) : launch_products<true, PAIR, false, false>(b, s);
            if (r != hipSuccess) return r;
        }
        return hipSuccess;
    };
    // P X (X P of a tall matrix): the next X, or the weights' step
    auto apply = [&](int x, int pw, float sx, float sp, float out, bool step) -> hipError_t {
        for (int tall = 0; tall < 2; ++tall) {
            begin();
            b.scale = 1.f / (sx * sp);
            b.out = out;
            for (int i = 0; i < count; ++i) {
                if (l[i].tall != (tall == 1)) continue;
                Product& p = b.p[b.count];
                p = Product{};
                const uint16_t* const xs = (uint16_t*)(sc + l[i].x[x]);
                const int64_t xp = l[i].rp * l[i].cp, pp = l[i].mp * l[i].mp;
                p.a = tall ? xs : square(i, pw); p.ap = tall ? xp : pp;
                p.b = tall ? square(i, pw) : xs; p.bp = tall ? pp : xp;
                p.lda = (int32_t)(tall ? l[i].cp : l[i].mp);
                p.ldb = (int32_t)(tall ? l[i].mp : l[i].cp);
                p.M = (int32_t)l[i].rp; p.N = (int32_t)l[i].cp; p.K = (int32_t)l[i].mp;
                p.c = (uint16_t*)(sc + l[i].x[1 - x]);
                p.matrix = b.count;
                b.d[b.count++] = Destination{t[i].param, t[i].master, t[i].rows, t[i].cols, t[i].scale,
                                             (float)t[i].weight_decay, t[i].flags};
            }
            hipError_t r;
            if (step) r = tall ? launch_products<false, STEP, false, false>(b, s) : launch_products<false, STEP, false, true>(b, s);
            else r = tall ? launch_products<false, PAIR, false, false>(b, s) : launch_products<false, PAIR, false, true>(b, s);
            if (r != hipSuccess) return r;
        }
        return hipSuccess;
    };

    int x = 0, power = -1;  // the X that stands, and the name of P (none yet: I)
    float sx = q.x[0], sp = 1.f;
    if ((e = gram(x, sx, q.gram[0])) != hipSuccess) return e;
    for (int k = 0; k < a.steps; ++k) {
        const bool last = k == a.steps - 1, anew = !last && (k == 1 || (k > 1 && (k - 1) % 3 == 0));
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
        if ((e = launch_products<true, POLY, false, false>(b, s)) != hipSuccess) return e;
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
        if (b.count && (e = launch_products<true, PAIR, false, false>(b, s)) != hipSuccess) return e;
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
            if ((e = launch_products<true, PAIR, false, false>(b, s)) != hipSuccess) return e;
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
        r->t[r->count] = t[i];
        r->l[r->count] = layout(t[i], r->total);
        r->total = r->l[r->count++].total;
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
