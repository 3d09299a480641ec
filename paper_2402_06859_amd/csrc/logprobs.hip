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
constexpr int LISTED = 512;  // groups among which the largest are ranked

__device__ __forceinline__ int64_t id_of(const void* ids, bool i64, int64_t m) {
    return i64 ? ((const int64_t*)ids)[m] : (int64_t)((const int32_t*)ids)[m];
}

// a and b become their join; one without any visible class has max -inf and rest -1.
__device__ __forceinline__ ChoiceStat join(const ChoiceStat& p, const ChoiceStat& q) {
    const bool swap = q.max > p.max;
    const ChoiceStat a = swap ? q : p, b = swap ? p : q;
    // (a range that holds NaN may have such a maximum too, but not that rest)
    if (b.max == NEG_INF) return ChoiceStat{a.max, b.rest == -1.f ? a.rest : a.rest + b.rest, a.mean, 0.f};
    const float t = b.max - a.max, e = expf(t), all = 1.f + b.rest;
    return ChoiceStat{a.max, fmaf(e, all, a.rest), e == 0.f ? a.mean : fmaf(e, fmaf(t, all, b.mean), a.mean), 0.f};
}
// The join of a wave's: the largest maximum first, then sums of what each adds to it (a tree of joins has three times the instructions).
__device__ __forceinline__ ChoiceStat wave_join(const ChoiceStat& p) {
    float top = p.max;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const uint64_t at_top = __ballot(p.max == top);
    const float t = p.max - top, e = expf(t), all = 1.f + p.rest;
    float rest = e * all, mean = e == 0.f ? 0.f : e * fmaf(t, all, p.mean);
    if (p.max == NEG_INF) rest = p.rest == -1.f ? 0.f : p.rest, mean = 0.f;
    if ((int)(threadIdx.x & 63) == __ffsll((unsigned long long)at_top) - 1) rest = p.rest, mean = p.mean;  // (the one whose maximum stands for all)
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        rest += __shfl_xor(rest, o);
        mean += __shfl_xor(mean, o);
    }
    return ChoiceStat{top, rest, mean, 0.f};
}

// (value, id) a ahead of b in the order of the answer: larger first, then the lower id.
__device__ __forceinline__ bool ahead(float a, int ia, float b, int ib) { return a > b || (a == b && ia < ib); }

__device__ __forceinline__ float key_of(uint2 g) {  // a group's largest logit; NaN counts as not visible
    const float v = __uint_as_float(g.x);
    return v == v ? v : NEG_INF;
}

// The rank of item `at` of n (at most 64) in a wave: up to four lanes an item, each against a part of the others. before(j, i): j is ahead of i.
template <typename F>
__device__ __forceinline__ int wave_rank(int n, int& at, bool& writes, F before) {
    const int lane = threadIdx.x & 63, log = n <= 16 ? 2 : n <= 32 ? 1 : 0, part = lane & ((1 << log) - 1);
    at = lane >> log;
    writes = part == 0 && at < n;
    int r = 0;
    if (at < n) {
#pragma unroll 4
        for (int j = part; j < n; j += 1 << log) r += before(j, at);
    }
    const int r1 = __shfl_xor(r, 1);
    if (log > 0) r += r1;
    const int r2 = __shfl_xor(r, 2);
    if (log > 1) r += r2;
    return r;
}

// The groups of the `want` largest maxima, ordered, into chosen; returns how many there are (fewer where fewer hold a visible
// class). Every four threads' largest is ranked among the 64 of them; the want-th of those is no larger than the want-th of all
// groups, so all that reach it are listed, a few more than wanted, and ranked in turn.
struct Chosen {
    int group[GROUPS_MAX];
    float key[GROUPS_MAX];
    uint32_t bound[GROUPS_MAX];
    float keys[64];
    int list[LISTED];
    float list_key[LISTED];
    uint32_t list_bound[LISTED];
    float wave_key[4];
    int count, wave_group[4];
};
__device__ __forceinline__ double lane_double(double x, int lane) {
    const uint64_t b = (uint64_t)__double_as_longlong(x);
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)b, lane), hi = __builtin_amdgcn_readlane((uint32_t)(b >> 32), lane);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}

// `beside` runs where one wave ranks what is listed and the others wait.
template <typename F>
__device__ __forceinline__ int choose_groups(const uint2* groups, int n, int want, Chosen& c, F beside) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int AHEAD = 8;  // loads in flight
    float mine = NEG_INF;
    for (int u0 = tid; u0 < n; u0 += 256 * AHEAD) {
        uint2 g[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) g[i] = groups[u0 + 256 * i < n ? u0 + 256 * i : u0];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) mine = fmaxf(mine, key_of(g[i]));
    }
    float four = fmaxf(mine, __shfl_xor(mine, 1));
    four = fmaxf(four, __shfl_xor(four, 2));
    if (lane % 4 == 0) c.keys[tid / 4] = four;
    if (tid == 0) c.count = 0;
    __syncthreads();
    // the want-th largest of 64, its first 20 bits (what is cut off makes it no larger), bit by bit from the top: each counts the lanes that
    // reach it. (Ranking the lanes against each other takes four times the instructions, and this part is bound by those.)
    const uint32_t raw = __float_as_uint(c.keys[lane]), key = raw ^ ((int)raw < 0 ? 0xFFFFFFFFu : 0x80000000u);
    uint32_t bits = 0;
#pragma unroll
    for (int j = 31; j >= 12; --j) {
        const uint32_t next = bits | 1u << j;
        bits = __popcll(__ballot(key >= next)) >= want ? next : bits;
    }
    const float bar = __uint_as_float(bits & 0x80000000u ? bits ^ 0x80000000u : ~bits);  // (of every wave alike)
    if (!(mine < bar) && mine != NEG_INF) {  // (a bar below all is NaN)
        for (int u0 = tid; u0 < n; u0 += 256 * AHEAD) {
            uint2 g[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) g[i] = groups[u0 + 256 * i < n ? u0 + 256 * i : u0];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const float k = key_of(g[i]);
                if (u0 + 256 * i >= n || k < bar || k == NEG_INF) continue;
                const int at = atomicAdd(&c.count, 1);
                if (at < LISTED) c.list[at] = u0 + 256 * i, c.list_key[at] = k, c.list_bound[at] = g[i].y;
            }
        }
    }
    __syncthreads();
    const int listed = c.count;
    beside();
    if (listed <= LISTED) {  // (the list's order is by chance, its ranks are not)
        if (listed <= 64) {
            if (wave == 0) {
                int i;
                bool writes;
                const int r = wave_rank(listed, i, writes, [&](int j, int i) { return ahead(c.list_key[j], c.list[j], c.list_key[i], c.list[i]); });
                if (writes && r < want) c.group[r] = c.list[i], c.key[r] = c.list_key[i], c.bound[r] = c.list_bound[i];
            }
        } else {
            for (int i = tid; i < listed; i += 256) {
                const float k = c.list_key[i];
                const int u = c.list[i];
                int r = 0;
                for (int j = 0; j < listed; ++j) r += ahead(c.list_key[j], c.list[j], k, u);
                if (r < want) c.group[r] = u, c.key[r] = k, c.bound[r] = c.list_bound[i];
            }
        }
        __syncthreads();
        return listed < want ? listed : want;
    }
    // many equal ones at the bar: one group at a time, each thread holding the best of its own behind the last one taken
    float last = __builtin_huge_valf(), best = NEG_INF;
    int last_at = -1, best_at = n;
    auto rescan = [&]() {
        best = NEG_INF;
        best_at = n;
        for (int u = tid; u < n; u += 256) {
            const float k = key_of(groups[u]);
            if (ahead(last, last_at, k, u) && ahead(k, u, best, best_at)) best = k, best_at = u;
        }
    };
    rescan();
    for (int i = 0; i < want; ++i) {
        float k = best;
        int at = best_at;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const float ok = __shfl_xor(k, o);
            const int oat = __shfl_xor(at, o);
            if (ahead(ok, oat, k, at)) k = ok, at = oat;
        }
        if (lane == 0) c.wave_key[wave] = k, c.wave_group[wave] = at;
        __syncthreads();
        k = c.wave_key[0], at = c.wave_group[0];
#pragma unroll
        for (int v = 1; v < 4; ++v)
            if (ahead(c.wave_key[v], c.wave_group[v], k, at)) k = c.wave_key[v], at = c.wave_group[v];
        if (tid == 0) c.group[i] = at, c.key[i] = k, c.bound[i] = groups[at].y;
        last = k, last_at = at;
        if (at == best_at) rescan();
        __syncthreads();
    }
    return want;
}

// One workgroup per row.
template <typename T, bool LATE>
__global__ __launch_bounds__(256) void k_choice_rows(ChoiceRows a) {
    __shared__ ChoiceStat wave_stat[4];
    __shared__ Chosen chosen;
    __shared__ int count;
    __shared__ int cand[CANDIDATES_MAX];
    __shared__ double cand_z[CANDIDATES_MAX];
    __shared__ double best;
    __shared__ float row_log_all;
    const int64_t m = blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (m >= a.rows) return;

    // One wave joins the tiles, unless they are very many: the others go on to the groups (this kernel is bound by its instructions, and a
    // join has 45 of them). LATE: the second wave, from loads made ahead, while the first one ranks groups.
    const int joiners = !LATE && a.tiles > 1024 ? 256 : 64, joiner = LATE ? 1 : 0;
    const int64_t label = a.labels ? id_of(a.labels, a.ids64, m) : -1;
    const float zlabel = a.labels ? a.zlabel[m] : 0.f;  // (written where the label is in range)
    const bool joins = joiners == 256 || wave == joiner;
    const int64_t from = joiners == 256 ? tid : lane;
    ChoiceStat q[4];
    auto load = [&](int64_t t0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = a.stat[m * a.tiles + (t0 + joiners * i < a.tiles ? t0 + joiners * i : a.tiles - 1)];
    };
    auto joined = [&]() __attribute__((always_inline)) {
        ChoiceStat r{NEG_INF, -1.f, 0.f, 0.f};
        for (int64_t t0 = from; t0 < a.tiles; t0 += 4 * joiners) {
            if (!LATE || t0 != from) load(t0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t0 + joiners * i < a.tiles) r = join(r, q[i]);
        }
        return wave_join(r);
    };
    auto answer = [&](const ChoiceStat& r) __attribute__((always_inline)) {
        const bool none = r.max == NEG_INF && r.rest == -1.f;  // every class is masked
        const float log_all = none ? 0.f : log1pf(r.rest), tau = none ? 0.f : r.mean / (1.f + r.rest);
        if (lane == 0) {
            int64_t y = label;
            if (y >= a.classes) {
                atomicOr(a.err, ERR_BIT_INDEX);
                y = -1;
            }
            float dy = NEG_INF;
            if (y >= 0 && zlabel != NEG_INF) dy = zlabel - r.max;
            if (a.logprob) a.logprob[m] = y >= 0 ? dy - log_all : 0.f;
            if (a.lse) a.lse[m] = none ? NEG_INF : r.max + log_all;
            if (a.entropy) a.entropy[m] = log_all - tau;
            if (a.stats) a.stats[m] = make_float4(r.max, r.rest, tau, dy);
            row_log_all = log_all;
        }
    };
    if (tid == 0) count = 0;
    if (LATE) {
        if (joins) load(from);
    } else {
        if (joins) {
            const ChoiceStat r = joined();
            if (joiners == 64) answer(r);
            else if (lane == 0) wave_stat[wave] = r;
        }
        if (joiners == 256) {
            __syncthreads();
            if (wave == 0) answer(join(join(wave_stat[0], wave_stat[1]), join(wave_stat[2], wave_stat[3])));
        }
        if (a.top == 0) return;
    }

    const uint2* const groups = a.groups + m * a.g.count;
    const int want = (int)(a.g.count < a.top + SLACK ? a.g.count : a.top + SLACK);
    const int got = choose_groups(groups, (int)a.g.count, want, chosen, [&]() {
        if (LATE && joins) answer(joined());
    });
    // the candidates: each group's largest class, and all of its classes where another may be as large as the last group's
    const float least = got == want && want < a.g.count ? chosen.key[want - 1] : NEG_INF;
    const int size_log = 31 - __builtin_clz(a.g.size), per_log = 29 - __builtin_clz(a.g.pitch);  // (powers of two)
    for (int i = tid; i < got << size_log; i += 256) {
        const int u = chosen.group[i >> size_log], k = i & (a.g.size - 1);
        const uint32_t bound = chosen.bound[i >> size_log];
        const int64_t v = (int64_t)(u >> per_log) * a.g.span + (u & ((1 << per_log) - 1)) * 4 + (k >> 2) * a.g.pitch + (k & 3);
        const bool all = !(__uint_as_float(bound & ~15u) < least);
        if ((all || k == (int)(bound & 15u)) && v < a.classes) cand[atomicAdd(&count, 1)] = (int)v;
    }
    __syncthreads();
    const int n = count;
    // their logits, four at a time in a wave
    constexpr int W = st<T>::vec, AT_ONCE = 4;
    static_assert(AT_ONCE == 4, "the exchanges below");
    const T* const x = (const T*)a.x + m * a.dim;
    for (int c0 = wave * AT_ONCE; c0 < n; c0 += 4 * AT_ONCE) {
        const T* w[AT_ONCE];
        double z[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            w[i] = (const T*)a.w + cand[c0 + i < n ? c0 + i : n - 1] * a.dim;
            z[i] = 0.0;
        }
#pragma unroll 2
        for (int64_t k = lane * W; k < a.dim; k += 64 * W) {
            float p[W], q[W];
            u32x4_t raw[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) raw[i] = *(const u32x4_t*)(w[i] + k);
            st<T>::unpack(*(const u32x4_t*)(x + k), p);
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                st<T>::unpack(raw[i], q);
#pragma unroll
                for (int e = 0; e < W; ++e) z[i] = fma((double)p[e], (double)q[e], z[i]);
            }
        }
        // four sums over 64 lanes at once: every exchange halves the values that a lane goes on with
        const bool high = lane & 32, odd = lane & 16;
        double y0 = (high ? z[2] : z[0]) + __shfl_xor(high ? z[0] : z[2], 32);
        const double y1 = (high ? z[3] : z[1]) + __shfl_xor(high ? z[1] : z[3], 32);
        y0 = (odd ? y1 : y0) + __shfl_xor(odd ? y0 : y1, 16);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) y0 += __shfl_xor(y0, o);
        const int at = c0 + (lane >> 4);  // (lanes from 16 i on have the sum of candidate i)
        if ((lane & 15) == 0 && at < n) {
            const float off = a.offset ? a.offset[cand[at]] : 0.f;
            const double v = off == NEG_INF ? -__builtin_huge_val() : y0 * (double)a.logit_scale + (double)off;
            cand_z[at] = v == v ? v : -__builtin_huge_val();
        }
    }
    __syncthreads();
    const float log_all = row_log_all;
    auto put = [&](int k, int64_t id, float v) {
        if (a.ids64) ((int64_t*)a.top_ids)[m * a.top + k] = id;
        else ((int32_t*)a.top_ids)[m * a.top + k] = (int32_t)id;
        if (a.top_logprob) a.top_logprob[m * a.top + k] = v;
    };
    if (n <= 64) {  // one wave ranks them, from its registers
        if (wave > 0) return;
        int i;
        bool writes;
        const int r = wave_rank(n, i, writes, [&](int j, int i) { return cand_z[j] > cand_z[i] || (cand_z[j] == cand_z[i] && cand[j] < cand[i]); });
        const double z = i < n ? cand_z[i] : 0.0, first = lane_double(z, __ffsll((unsigned long long)__ballot(writes && r == 0)) - 1);
        const bool seen = z != -__builtin_huge_val();
        if (writes && r < a.top) put(r, seen ? cand[i] : -1, seen ? (float)(z - first) - log_all : NEG_INF);
        if (lane >= n && lane < a.top) put(lane, -1, NEG_INF);  // fewer visible classes than wanted
        return;
    }
    constexpr int MOST = (CANDIDATES_MAX + 255) / 256;
    int ranks[MOST];
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
        const int c = tid + 256 * i;
        ranks[i] = a.top;
        if (c >= n) continue;
        ranks[i] = 0;
#pragma unroll 4
        for (int j = 0; j < n; ++j) ranks[i] += cand_z[j] > cand_z[c] || (cand_z[j] == cand_z[c] && cand[j] < cand[c]);
        if (ranks[i] == 0) best = cand_z[c];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
        if (ranks[i] >= a.top) continue;
        const int c = tid + 256 * i;
        const bool seen = cand_z[c] != -__builtin_huge_val();
        put(ranks[i], seen ? cand[c] : -1, seen ? (float)(cand_z[c] - best) - log_all : NEG_INF);
    }
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

__device__ __forceinline__ ChoiceRow choice_row(const ChoicePrepare& a, int64_t m, bool any, int64_t y, float g, float h) {
    ChoiceRow r{};
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
    return r;
}

template <typename T>
__global__ __launch_bounds__(256) void k_choice_prepare(ChoicePrepare a) {
    constexpr int W = st<T>::vec;
    const int64_t per = a.dim / W, n = a.rows * per, step = gridDim.x * 256ll, t = blockIdx.x * 256ll + threadIdx.x;
    int64_t y;
    float g, h;
    for (int64_t m = t; m < a.rows; m += step) {
        const bool any = upstream(a, m, y, g, h);
        if (y >= a.classes) atomicOr(a.err, ERR_BIT_INDEX);
        a.row[m] = choice_row(a, m, any, y, g, h);
    }
    for (int64_t i = t; i < n; i += step) {
        u32x4_t v = {0u, 0u, 0u, 0u};
        if (upstream(a, i / per, y, g, h)) v = *(const u32x4_t*)((const T*)a.x + i * W);
        for (int k = 0; k < a.copies; ++k) *(u32x4_t*)((T*)a.kept + k * a.rows * a.dim + i * W) = v;
    }
}

// Columns first .. of row m of the gradient in the logits, from the exponentials that the forward kept: p = e exp(tile's
// maximum - row's) / (1 + rest), and d from e's logarithm. Reads and writes each element once (2 + 2 bytes, 4 + 4 in float). Where
// little is to be written, no k_choice_prepare runs in front: every thread computes its row's factors, and the first piece's workgroups copy x on
// the way (333 x 1001, dim 136: 3.5 + 4.1 us in two launches, 5.1 in one; 4096 x 32000: 101 and 104; 8192 x 131072: 816 and 869).
template <typename T>
__global__ __launch_bounds__(256) void k_choice_normalize(ChoiceNormalize a) {
    constexpr int W = st<T>::vec;
    constexpr float UNIT = sizeof(T) == 2 ? 1.f / SOFT_E_SCALE : 1.f, LN2 = 0.693147181f;
    const int64_t m = blockIdx.y + (int64_t)blockIdx.z * 65535;
    if (m >= a.p.rows) return;
    int64_t y;
    float g, h;
    const bool any = upstream(a.p, m, y, g, h);
    if (!a.prepared && a.first == 0) {
        if (y >= a.p.classes && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.p.err, ERR_BIT_INDEX);
        for (int64_t i = (blockIdx.x * 256ll + threadIdx.x) * W; i < a.p.dim; i += gridDim.x * 256ll * W) {
            u32x4_t v = {0u, 0u, 0u, 0u};
            if (any) v = *(const u32x4_t*)((const T*)a.p.x + m * a.p.dim + i);
            for (int k = 0; k < a.p.copies; ++k) *(u32x4_t*)((T*)a.p.kept + (k * a.p.rows + m) * a.p.dim + i) = v;
        }
    }
    const ChoiceRow r = a.prepared ? a.p.row[m] : choice_row(a.p, m, any, y, g, h);
    const bool none = r.a == 0.f && r.b == 0.f;
    for (int64_t n = (blockIdx.x * 256ll + threadIdx.x) * W; n < a.width; n += gridDim.x * 256ll * W) {
        const int64_t v = a.first + n;  // the class
        const float top = a.stat[m * a.tiles + v / a.tile].max;
        float e[W];
        if constexpr (sizeof(T) == 2) unpack_f16x8(*(const u32x4_t*)((const _Float16*)a.kept + m * a.kept_ld + v), e);
        else st<T>::unpack(*(const u32x4_t*)((const float*)a.kept + m * a.kept_ld + v), e);
        const float gap = top - r.max, f = none || top == NEG_INF ? 0.f : UNIT * expf(gap);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float d = fmaf(__builtin_amdgcn_logf(e[i] * UNIT), LN2, gap);
            e[i] = f == 0.f || e[i] == 0.f ? 0.f : e[i] * f * fmaf(r.b, d, r.a);
        }
        if (y >= v && y < v + W) {
#pragma unroll
            for (int i = 0; i < W; ++i)
                if (y - v == i) e[i] = r.label;
        }
        *(u32x4_t*)((T*)a.out + m * a.ld + n) = st<T>::pack(e);
        if (sizeof(T) == 2 && a.out_lo) {
#pragma unroll
            for (int i = 0; i < W; ++i) e[i] -= st<T>::round(e[i]);
            *(u32x4_t*)((T*)a.out_lo + m * a.ld + n) = st<T>::pack(e);
        }
    }
}

}  // namespace

hipError_t launch_choice_normalize(const ChoiceNormalize& a, bool bf16, hipStream_t s) {
    if (a.p.rows == 0 || a.width == 0) return hipSuccess;
    const int64_t vectors = a.width / (bf16 ? 8 : 4), y = a.p.rows < 65535 ? a.p.rows : 65535;
    int64_t per = (vectors + 1023) / 1024;  // four vectors a thread
    if (per > 64) per = 64;
    const int64_t fill = (1024 + a.p.rows - 1) / a.p.rows;  // (or fewer, down to one, until there are 1024 workgroups)
    if (per < fill) per = fill < (vectors + 255) / 256 ? fill : (vectors + 255) / 256;
    const dim3 grid((unsigned)per, (unsigned)y, (unsigned)((a.p.rows + 65534) / 65535));
    if (bf16) hipLaunchKernelGGL(k_choice_normalize<bf16_t>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(k_choice_normalize<float>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_choice_rows(const ChoiceRows& a, bool bf16, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    const int64_t x = a.rows < 1 << 20 ? a.rows : 1 << 20;  // (less than 2^32 threads along x)
    const dim3 grid((unsigned)x, (unsigned)((a.rows + x - 1) / x));
    // us, join first / late: 64 x 5000 classes 10.6 / 9.5, 1024 x 5000 17.3 / 16.0, 1 x 50000 12.4 / 11.4; 2000 x 5000 23.6 / 24.4, 8192 x 1000 73 / 80 (more
    // rows hide one another's waits); 50 x 100003 in float (1563 tiles) 25.8 / 29.8
    if (a.top > 0 && a.rows <= 1024 && a.tiles <= 1024) {
        if (bf16) hipLaunchKernelGGL((k_choice_rows<bf16_t, true>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((k_choice_rows<float, true>), grid, dim3(256), 0, s, a);
    } else {
        if (bf16) hipLaunchKernelGGL((k_choice_rows<bf16_t, false>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((k_choice_rows<float, false>), grid, dim3(256), 0, s, a);
    }
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
