// Log probabilities of given classes, with the entropy and the most probable classes of each row, and their gradient: what
// stands around the products.
//
//   z[m, v] = s (x[m] . w[v]) + offset[v],  d = z - max_v z,  rest = sum over all classes but one largest of exp(d)
//   lse = max + log1p(rest),   log p[v] = d[v] - log1p(rest)
//   tau = sum_v p[v] d[v],     H = -sum_v p[v] log p[v] = log1p(rest) - tau
//   L's gradient for g = dL/dlog p[y] and h = dL/dH:  dL/dz[v] = g ([v = y] - p[v]) - h p[v] (d[v] - tau)
//
// The logits product (gemm.hip, EPI_CHOICE_FWD) leaves a ChoiceStat (max, rest, sum of exp(d) d) per row and column tile, which are
// joined here: for maxima a >= b and t = b - a, rest = rest_a + exp(t) (1 + rest_b) and mean = mean_a + exp(t) (mean_b + t (1 +
// rest_b)). All terms of a sum have one sign, so that a row whose probability is nearly all on one class keeps the digits of 1 - p and
// of its entropy.
//
// Most probable classes. The product leaves the largest logit of each group of 8 or 16 classes, its place, and a bound on the
// others': 1/16 or less of the logits' own bytes. The `top` largest logits lie in the `top` groups with the largest maxima, and
// beside those maxima only classes of groups whose bound reaches the least of them can be among them. So SLACK more groups
// than wanted are taken, the candidates' logits are computed again as sums in 64 bits, and these decide: ties go to the lowest class.
// The slack covers what a float sum may mistake at the border, and equal logits in groups whose classes interleave (up to 4).
#include "device_common.h"
#include "logprobs.h"

namespace rdcn {

namespace {

constexpr int ERR_BIT_INDEX = 1;
constexpr float NEG_INF = -__builtin_huge_valf();
constexpr int SLACK = 4, GROUPS_MAX = CHOICE_TOP_MAX + SLACK, CANDIDATES_MAX = GROUPS_MAX * 16;

__device__ __forceinline__ int64_t id_of(const void* ids, bool i64, int64_t m) {
    return i64 ? ((const int64_t*)ids)[m] : (int64_t)((const int32_t*)ids)[m];
}

// a and b become their join; one without any visible class has max -inf and rest -1.
__device__ __forceinline__ ChoiceStat join(const ChoiceStat& p, const ChoiceStat& q) {
    const bool swap = q.max > p.max;
    const ChoiceStat a = swap ? q : p, b = swap ? p : q;
    // (a range of NaN alone has such a maximum, but not that rest)
    if (b.max == NEG_INF) return ChoiceStat{a.max, b.rest == -1.f ? a.rest : a.rest + b.rest, a.mean, 0.f};
    const float t = b.max - a.max, e = expf(t), all = 1.f + b.rest;
    return ChoiceStat{a.max, fmaf(e, all, a.rest), e == 0.f ? a.mean : fmaf(e, fmaf(t, all, b.mean), a.mean), 0.f};
}
__device__ __forceinline__ ChoiceStat shuffled(const ChoiceStat& p, int o) {
    return ChoiceStat{__shfl_xor(p.max, o), __shfl_xor(p.rest, o), __shfl_xor(p.mean, o), 0.f};
}

// (value, id) a ahead of b in the order of the answer: larger first, then the lower id.
__device__ __forceinline__ bool ahead(float a, int64_t ia, float b, int64_t ib) { return a > b || (a == b && ia < ib); }

__device__ __forceinline__ float key_of(uint2 g) {  // a group's largest logit; NaN counts as not visible
    const float v = __uint_as_float(g.x);
    return v == v ? v : NEG_INF;
}

// One workgroup per row.
template <typename T>
__global__ __launch_bounds__(256) void k_choice_rows(ChoiceRows a) {
    __shared__ ChoiceStat wave_stat[4];
    __shared__ float wave_key[4];
    __shared__ int64_t wave_group[4];
    __shared__ int64_t chosen[GROUPS_MAX];
    __shared__ float chosen_key[GROUPS_MAX];
    __shared__ int count;
    __shared__ int64_t cand[CANDIDATES_MAX];
    __shared__ double cand_z[CANDIDATES_MAX];
    __shared__ double best;
    const int64_t m = blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (m >= a.rows) return;

    ChoiceStat r{NEG_INF, -1.f, 0.f, 0.f};
    for (int64_t t = tid; t < a.tiles; t += 256) r = join(r, a.stat[m * a.tiles + t]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) r = join(r, shuffled(r, o));
    if (lane == 0) wave_stat[wave] = r;
    __syncthreads();
    r = join(join(wave_stat[0], wave_stat[1]), join(wave_stat[2], wave_stat[3]));
    const bool none = r.max == NEG_INF && r.rest == -1.f;  // every class is masked
    const float log_all = none ? 0.f : log1pf(r.rest), tau = none ? 0.f : r.mean / (1.f + r.rest);
    if (tid == 0) {
        int64_t y = -1;
        if (a.labels) {
            y = id_of(a.labels, a.ids64, m);
            if (y >= a.classes) {
                atomicOr(a.err, ERR_BIT_INDEX);
                y = -1;
            }
        }
        float dy = NEG_INF;
        if (y >= 0 && a.zlabel[m] != NEG_INF) dy = a.zlabel[m] - r.max;
        if (a.logprob) a.logprob[m] = y >= 0 ? dy - log_all : 0.f;
        if (a.lse) a.lse[m] = none ? NEG_INF : r.max + log_all;
        if (a.entropy) a.entropy[m] = log_all - tau;
        if (a.stats) a.stats[m] = make_float4(r.max, r.rest, tau, dy);
    }
    if (a.top == 0) return;

    // the top + SLACK groups of the largest maxima, one at a time: each thread holds the best of its own that is
    // behind the last one taken
    const uint2* const groups = a.groups + m * a.g.count;
    const int want = (int)(a.g.count < a.top + SLACK ? a.g.count : a.top + SLACK);
    float last = __builtin_huge_valf(), mine = NEG_INF;
    int64_t last_at = -1, mine_at = a.g.count;
    auto rescan = [&]() {
        mine = NEG_INF;
        mine_at = a.g.count;
        for (int64_t u = tid; u < a.g.count; u += 256) {
            const float k = key_of(groups[u]);
            if (ahead(last, last_at, k, u) && ahead(k, u, mine, mine_at)) mine = k, mine_at = u;
        }
    };
    rescan();
    for (int i = 0; i < want; ++i) {
        float k = mine;
        int64_t at = mine_at;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const float ok = __shfl_xor(k, o);
            const int64_t oat = __shfl_xor(at, o);
            if (ahead(ok, oat, k, at)) k = ok, at = oat;
        }
        if (lane == 0) wave_key[wave] = k, wave_group[wave] = at;
        __syncthreads();
        k = wave_key[0], at = wave_group[0];
#pragma unroll
        for (int v = 1; v < 4; ++v)
            if (ahead(wave_key[v], wave_group[v], k, at)) k = wave_key[v], at = wave_group[v];
        if (tid == 0) chosen[i] = at, chosen_key[i] = k;
        last = k, last_at = at;
        if (at == mine_at) rescan();
        __syncthreads();
    }

    // their candidates: the largest class, and all where another may be as large as the last group's
    if (tid == 0) count = 0;
    __syncthreads();
    const float least = want < a.g.count ? chosen_key[want - 1] : NEG_INF;
    if (tid < want) {
        const int64_t u = chosen[tid];
        const uint2 g = groups[u];
        const int per = a.g.pitch / 4;
        const int64_t base = u / per * a.g.span + u % per * 4;
        auto cls = [&](int k) { return base + (int64_t)(k / 4) * a.g.pitch + k % 4; };
        const bool all = !(__uint_as_float(g.y & ~15u) < least);
        for (int k = 0; k < a.g.size; ++k)
            if ((all || k == (int)(g.y & 15u)) && cls(k) < a.classes) cand[atomicAdd(&count, 1)] = cls(k);
    }
    __syncthreads();
    const int n = count;
    for (int c = wave; c < n; c += 4) {
        const int64_t v = cand[c];
        const T* const x = (const T*)a.x + m * a.dim;
        const T* const w = (const T*)a.w + v * a.dim;
        double z = 0.0;
        constexpr int W = st<T>::vec;
        for (int64_t k = lane * W; k < a.dim; k += 64 * W) {
            float p[W], q[W];
            st<T>::unpack(*(const u32x4_t*)(x + k), p);
            st<T>::unpack(*(const u32x4_t*)(w + k), q);
#pragma unroll
            for (int e = 0; e < W; ++e) z = fma((double)p[e], (double)q[e], z);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o);
        const float off = a.offset ? a.offset[v] : 0.f;
        z = off == NEG_INF ? -__builtin_huge_val() : z * (double)a.logit_scale + (double)off;
        if (lane == 0) cand_z[c] = z == z ? z : -__builtin_huge_val();
    }
    __syncthreads();
    // ranks
    auto rank = [&](int c) {
        int k = 0;
        for (int i = 0; i < n; ++i) k += cand_z[i] > cand_z[c] || (cand_z[i] == cand_z[c] && cand[i] < cand[c]);
        return k;
    };
    int ranks[(CANDIDATES_MAX + 255) / 256];
#pragma unroll
    for (int i = 0; i < (CANDIDATES_MAX + 255) / 256; ++i) {
        const int c = tid + 256 * i;
        ranks[i] = c < n ? rank(c) : a.top;
        if (ranks[i] == 0) best = cand_z[c];
    }
    __syncthreads();
    auto put = [&](int k, int64_t id, float v) {
        if (a.ids64) ((int64_t*)a.top_ids)[m * a.top + k] = id;
        else ((int32_t*)a.top_ids)[m * a.top + k] = (int32_t)id;
        if (a.top_logprob) a.top_logprob[m * a.top + k] = v;
    };
#pragma unroll
    for (int i = 0; i < (CANDIDATES_MAX + 255) / 256; ++i) {
        if (ranks[i] >= a.top) continue;
        const int c = tid + 256 * i;
        const bool seen = cand_z[c] != -__builtin_huge_val();
        put(ranks[i], seen ? cand[c] : -1, seen ? (float)(cand_z[c] - best) - log_all : NEG_INF);
    }
    for (int k = n + tid; k < a.top; k += 256) put(k, -1, NEG_INF);  // fewer classes than wanted
}

// Whether row m has a gradient at all. Rows without one (no label, or both upstream gradients 0) may hold anything in x: 0 times
// an infinity would still reach grad_w's sum over the rows, whose product therefore reads a copy with zeros there.
__device__ __forceinline__ bool upstream(const ChoicePrepare& a, int64_t m, int64_t& y, float& g, float& h) {
    y = a.labels ? id_of(a.labels, a.ids64, m) : -1;
    const bool counts = !a.labels || (y >= 0 && y < a.classes);
    g = counts && a.labels && a.grad_logprob ? a.grad_logprob[m] : 0.f;
    h = counts && a.grad_entropy ? a.grad_entropy[m] : 0.f;
    return g != 0.f || h != 0.f;
}

template <typename T>
__global__ __launch_bounds__(256) void k_choice_prepare(ChoicePrepare a) {
    constexpr int W = st<T>::vec;
    const int64_t per = a.dim / W, n = a.rows * per, step = gridDim.x * 256ll, t = blockIdx.x * 256ll + threadIdx.x;
    int64_t y;
    float g, h;
    for (int64_t m = t; m < a.rows; m += step) {
        ChoiceRow r{};
        const bool any = upstream(a, m, y, g, h);
        if (y >= a.classes) atomicOr(a.err, ERR_BIT_INDEX);
        const float4 q = a.stats[m];  // max, rest, tau, label's d
        r.max = q.x;
        if (any && !(q.x == NEG_INF && q.y == -1.f)) {
            const float all = 1.f + q.y, inv = a.logit_scale / all;
            r.a = -inv * (g - h * q.z);
            r.b = -inv * h;
            if (y >= 0 && q.w != NEG_INF) {
                // 1 - p: the largest class's own share is left out of rest, another's is in it
                const float e = expf(q.w), others = q.w == 0.f ? q.y : q.y + (1.f - e);
                r.label = a.logit_scale * (g * (others / all) - h * (e / all) * (q.w - q.z));
            }
        }
        a.row[m] = r;
    }
    for (int64_t i = t; i < n; i += step) {
        u32x4_t v = {0u, 0u, 0u, 0u};
        if (upstream(a, i / per, y, g, h)) v = *(const u32x4_t*)((const T*)a.x + i * W);
        *(u32x4_t*)((T*)a.kept + i * W) = v;
    }
}

}  // namespace

hipError_t launch_choice_rows(const ChoiceRows& a, bool bf16, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    const int64_t x = a.rows < 1 << 20 ? a.rows : 1 << 20;  // (less than 2^32 threads along x)
    const dim3 grid((unsigned)x, (unsigned)((a.rows + x - 1) / x));
    if (bf16) hipLaunchKernelGGL(k_choice_rows<bf16_t>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(k_choice_rows<float>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_choice_prepare(const ChoicePrepare& a, bool bf16, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    const int64_t b = (a.rows * a.dim / (bf16 ? 8 : 4) + 255) / 256;
    const dim3 grid((unsigned)(b > 4096 ? 4096 : b));
    if (bf16) hipLaunchKernelGGL(k_choice_prepare<bf16_t>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(k_choice_prepare<float>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace rdcn
