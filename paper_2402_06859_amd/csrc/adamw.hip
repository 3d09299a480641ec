// AdamW over many tensors at once, with moments in 32 bits or in 8, and the norm of their gradients.
//
//   g' = g * grad_scale * clip          m' = beta1 m + (1 - beta1) g'     v' = beta2 v + (1 - beta2) g' g'
//   p' = p (1 - lr wd) - lr / (1 - beta1^t) * m' / (sqrt(v') / sqrt(1 - beta2^t) + eps)
//
// Every operation above is one rounding to float in this order (no contraction to fused ones): a step
// is the same bits wherever an element stands, and 8-bit codes do not hang on how it was compiled. (With 8-bit
// moments the root and the quotient, which only p' depends on, are within a unit in the last place each.)
//
// 8-bit moments. A block of 256 elements has one exponent, its largest element's. An
// element's code is the upper bits of its float (exponent and 3 mantissa bits, bits 20 and up)
// counted down from the top of the block's exponent: for m a sign and 7 bits, which reach 2^-15
// of the block's binade, for v 8 bits, 2^-31. Code 0 is the value 0; a nonzero v gets at least
// code 1, so that m / sqrt(v) never divides by nothing. With 3 mantissa bits a moving average whose
// step is 1 - beta = 0.1 or 0.001 would stand still under rounding to nearest (half a step is 1/16 to 1/32 of the
// value), so codes are rounded up with the probability of the part that is cut off: the bits below 20
// are added to 20 random bits, a hash of (seed, tensor, element). bf16 weights without a float master
// are rounded the same way, for the same reason. With `carry` a block's exponent goes up by one where that takes an element
// past its last code. Without, the block's largest elements stand still at that code, 1.875 of their binade, as long as no single
// step leaves the binade: v of gradients of one size then stays at 0.03 of its value, of normal ones at half of it. (585 M
// elements, without / with: 1299 / 1298 us.)
#include "adamw.h"
#include "device_common.h"

namespace rdcn {

namespace {

constexpr int EPT = 8;                      // consecutive elements of a thread
constexpr int CHUNK = 256 * EPT;            // elements of a workgroup's step
constexpr int PER_LAUNCH = 48;              // tensors of one launch: their descriptors are kernel arguments

struct Batch {
    AdamwTensor t[PER_LAUNCH];
    uint32_t first[PER_LAUNCH + 1];  // first chunk of each tensor
    int count;
    AdamwScalars a;
};
static_assert(sizeof(Batch) <= 4096, "kernel arguments");

struct NormBatch {
    const void* grad[PER_LAUNCH];
    int64_t n[PER_LAUNCH];
    uint32_t first[PER_LAUNCH + 1];
    uint32_t flags[PER_LAUNCH];
    int count;
    double* part;
};

// The tensor of chunk c: the last one that begins at or before it (tensors of no elements have no chunk). `last` is
// the tensor of an earlier chunk: most often still the one, without a search through the arguments.
__device__ __forceinline__ int tensor_of(const uint32_t* first, int count, uint32_t c, int last) {
    if (c < first[last + 1]) return last;
    int lo = last, hi = count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= c) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ uint32_t fmix32(uint32_t h) {  // MurmurHash3's 32-bit finalizer
    h ^= h >> 16;
    h *= 0x85EBCA6Bu;
    h ^= h >> 13;
    h *= 0xC2B2AE35u;
    return h ^ (h >> 16);
}

// Bits (from bit 20 up) that code 0 of a block whose largest exponent is e counts from.
__device__ __forceinline__ uint32_t code_base(uint32_t e, uint32_t top) {
    const int b = (int)(8 * e + 7) - (int)top;
    return b > 0 ? (uint32_t)b : 0u;
}
__device__ __forceinline__ float decode(uint32_t size, uint32_t base) {
    return size ? __uint_as_float((size + base) << 20) : 0.f;
}
// EPT values at p: all of them (known for the whole workgroup with WHOLE), or the first `left` and zeros.
template <bool WHOLE>
__device__ __forceinline__ void load_f32(const float* p, int left, float* v) {
    if (WHOLE || left == EPT) {
        *(f32x4_t*)v = *(const f32x4_t*)p;
        *(f32x4_t*)(v + 4) = *(const f32x4_t*)(p + 4);
    } else {
#pragma unroll
        for (int e = 0; e < EPT; ++e) v[e] = e < left ? p[e] : 0.f;
    }
}
template <bool WHOLE>
__device__ __forceinline__ void load_bf16(const bf16_t* p, int left, float* v) {
    if (WHOLE || left == EPT) {
        st<bf16_t>::unpack(*(const u32x4_t*)p, v);
    } else {
#pragma unroll
        for (int e = 0; e < EPT; ++e) v[e] = e < left ? bf16_to_f32(p[e]) : 0.f;
    }
}
template <bool WHOLE>
__device__ __forceinline__ void store_f32(float* p, int left, const float* v) {
    if (WHOLE || left == EPT) {
        *(f32x4_t*)p = *(const f32x4_t*)v;
        *(f32x4_t*)(p + 4) = *(const f32x4_t*)(v + 4);
    } else {
#pragma unroll
        for (int e = 0; e < EPT; ++e)
            if (e < left) p[e] = v[e];
    }
}
template <bool WHOLE>
__device__ __forceinline__ void store_u16(bf16_t* p, int left, const uint32_t* r) {  // r < 2^16
    if (WHOLE || left == EPT) {
        *(u32x4_t*)p = u32x4_t{r[0] | r[1] << 16, r[2] | r[3] << 16, r[4] | r[5] << 16, r[6] | r[7] << 16};
    } else {
#pragma unroll
        for (int e = 0; e < EPT; ++e)
            if (e < left) p[e] = (bf16_t)r[e];
    }
}
template <bool WHOLE>
__device__ __forceinline__ void load_codes(const uint8_t* p, int left, uint32_t* c) {
    if (WHOLE || left == EPT) {
        const uint2 w = *(const uint2*)p;
#pragma unroll
        for (int e = 0; e < EPT; ++e) c[e] = ((e < 4 ? w.x : w.y) >> (8 * (e & 3))) & 255u;
    } else {
#pragma unroll
        for (int e = 0; e < EPT; ++e) c[e] = e < left ? p[e] : 0u;
    }
}
template <bool WHOLE>
__device__ __forceinline__ void store_codes(uint8_t* p, int left, const uint32_t* c) {
    if (WHOLE || left == EPT) {
        *(uint2*)p = make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
    } else {
#pragma unroll
        for (int e = 0; e < EPT; ++e)
            if (e < left) p[e] = (uint8_t)c[e];
    }
}

// The largest value over the 32 lanes of a block of 256 elements: exchanges within rows of 16 lanes as part of the
// maximum's own operands, then one of two rows.
__device__ __forceinline__ uint32_t max_of_block(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0xB1, 0xF, 0xF, true));   // lane ^ 1
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x4E, 0xF, 0xF, true));   // lane ^ 2
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x141, 0xF, 0xF, true));  // mirrored in 8
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x140, 0xF, 0xF, true));  // mirrored in 16
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return max(r[0], r[1]);
}

struct StepScalars {
    float gs, step_size, r2, decay;
    uint32_t key;
};

// One thread's EPT elements from `at` on of one tensor.
template <bool EIGHT, bool WHOLE>
__device__ __forceinline__ void adamw_elements(const AdamwTensor& t, const AdamwScalars& a, const StepScalars& k, int64_t at) {
#pragma clang fp contract(off)
    const int left = WHOLE ? EPT : at < t.n ? (int)(t.n - at < EPT ? t.n - at : EPT) : 0;
    const bool pbf = t.flags & ADAMW_PARAM_BF16;
    const int64_t blocks = (t.n + ADAMW_BLOCK - 1) / ADAMW_BLOCK, blk = at / ADAMW_BLOCK;
    float p[EPT], g[EPT], m[EPT], v[EPT];
    if (t.flags & ADAMW_GRAD_BF16) load_bf16<WHOLE>((const bf16_t*)t.grad + at, left, g);
    else load_f32<WHOLE>((const float*)t.grad + at, left, g);
    if (t.master) load_f32<WHOLE>(t.master + at, left, p);
    else if (pbf) load_bf16<WHOLE>((const bf16_t*)t.param + at, left, p);
    else load_f32<WHOLE>((const float*)t.param + at, left, p);
    if constexpr (EIGHT) {
        uint32_t cm[EPT], cv[EPT];
        load_codes<WHOLE>((const uint8_t*)t.m + at, left, cm);
        load_codes<WHOLE>((const uint8_t*)t.v + at, left, cv);
        const uint32_t bm = left ? code_base(t.exps[blk], 127) : 0, bv = left ? code_base(t.exps[blocks + blk], 255) : 0;
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            m[e] = __uint_as_float(__float_as_uint(decode(cm[e] & 127u, bm)) | (cm[e] & 128u) << 24);
            v[e] = decode(cv[e], bv);
        }
    } else {
        load_f32<WHOLE>((const float*)t.m + at, left, m);
        load_f32<WHOLE>((const float*)t.v + at, left, v);
    }
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
        const float x = g[e] * k.gs;
        m[e] = m[e] * a.beta1 + x * a.c1;
        v[e] = v[e] * a.beta2 + (x * x) * a.c2;
        // 8-bit moments: the root and the quotient from the units alone (each within a unit in the last place, far
        // below what the codes' 3 bits carry); the rounded ones cost 24 more operations, and these kernels are bound by those
        const float down = (EIGHT ? __builtin_amdgcn_sqrtf(v[e]) : sqrtf(v[e])) * k.r2 + a.eps;
        const float q = EIGHT ? m[e] * __builtin_amdgcn_rcpf(down) : m[e] / down;
        p[e] = p[e] * k.decay - q * k.step_size;
    }
    uint32_t h[EPT];
    if (a.stochastic && (EIGHT || (pbf && !t.master))) {
#pragma unroll
        for (int e = 0; e < EPT; ++e) h[e] = fmix32(((uint32_t)at ^ k.key) ^ (uint32_t)e);  // (at is a multiple of EPT)
    }
    if (t.master) store_f32<WHOLE>(t.master + at, left, p);
    if (!pbf) {
        store_f32<WHOLE>((float*)t.param + at, left, p);
    } else {
        uint32_t r[EPT];
        if (a.stochastic && !t.master) {
#pragma unroll
            for (int e = 0; e < EPT; ++e) {
                r[e] = (__float_as_uint(p[e]) + ((h[e] * 0x85EBCA6Bu) >> 16)) >> 16;
                r[e] = p[e] == p[e] ? r[e] : 0x7FC0u;  // (a NaN's bits could carry into its sign)
            }
        } else {
#pragma unroll
            for (int e = 0; e < EPT; ++e) r[e] = f32_to_bf16(p[e]);
        }
        store_u16<WHOLE>((bf16_t*)t.param + at, left, r);
    }
    if constexpr (!EIGHT) {
        store_f32<WHOLE>((float*)t.m + at, left, m);
        store_f32<WHOLE>((float*)t.v + at, left, v);
    } else {
        if constexpr (!WHOLE) {  // past the end nothing counts towards the block's largest
#pragma unroll
            for (int e = 0; e < EPT; ++e)
                if (e >= left) m[e] = v[e] = 0.f;
        }
        uint32_t um[EPT], uv[EPT], mm = 0, mv = 0;
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            um[e] = __float_as_uint(m[e]) & 0x7FFFFFFFu;
            uv[e] = __float_as_uint(v[e]) & 0x7FFFFFFFu;
            mm = max(mm, um[e]);
            mv = max(mv, uv[e]);
        }
        uint32_t em = max_of_block(mm) >> 23, ev = max_of_block(mv) >> 23;
        const uint32_t bm = 0u - (code_base(em, 127) << 20), bv = 0u - (code_base(ev, 255) << 20);
        int x[EPT], y[EPT];
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            const uint32_t rm = a.stochastic ? h[e] >> 12 : 0x80000u;
            const uint32_t rv = a.stochastic ? (h[e] * 0x9E3779B1u) >> 12 : 0x80000u;
            // (a value of the block is at most 8 2^20 above its exponent's base + top: the differences fit an int; of a
            // zero and what lies below the reach they are negative or round to 0)
            x[e] = (int)(um[e] + rm + bm) >> 20;
            y[e] = (int)(uv[e] + rv + bv) >> 20;
        }
        if (a.carry) {  // a code past the last one: the block's exponent is one more, its codes count from 8 further up
            int mx = x[0], my = y[0];
#pragma unroll
            for (int e = 1; e < EPT; ++e) mx = max(mx, x[e]), my = max(my, y[e]);
            const uint64_t px = __ballot(mx > 127), py = __ballot(my > 255);
            if (px | py) {  // (about a step in ten, of the two blocks of a wave)
                const bool ux = (uint32_t)(px >> (threadIdx.x & 32)) && em < 254, uy = (uint32_t)(py >> (threadIdx.x & 32)) && ev < 254;
                em += ux;  // (past 254 there is no value)
                ev += uy;
#pragma unroll
                for (int e = 0; e < EPT; ++e) {
                    x[e] -= ux ? 8 : 0;
                    y[e] -= uy ? 8 : 0;
                }
            }
        }
        uint32_t cm[EPT], cv[EPT];
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            cm[e] = (uint32_t)min(max(x[e], 0), 127) | (__float_as_uint(m[e]) >> 24 & 128u);
            cv[e] = (uint32_t)min(max(y[e], (int)min(uv[e], 1u)), 255);
        }
        store_codes<WHOLE>((uint8_t*)t.m + at, left, cm);
        store_codes<WHOLE>((uint8_t*)t.v + at, left, cv);
        if ((threadIdx.x & 31) == 0 && left) {
            t.exps[blk] = (uint8_t)em;
            t.exps[blocks + blk] = (uint8_t)ev;
        }
    }
}

template <bool EIGHT>
__global__ __launch_bounds__(256) void k_adamw(Batch b) {
    const AdamwScalars& a = b.a;
    StepScalars k;
    k.gs = a.grad_scale;
    if (a.clip) {
        const float c = *a.clip;
        if (!(fabsf(c) < __builtin_huge_valf())) return;  // not finite: the gradients' norm was not, nothing is changed
        k.gs *= c;
    }
    k.step_size = a.step_size;
    k.r2 = a.rsqrt_grown2;
    const bool live = a.device_lr || a.device_step;
    double lr = a.lr;
    uint32_t seed = a.seed;
    if (live) {
        if (a.device_lr) lr = (double)*a.device_lr;
        int64_t t = a.device_step ? *a.device_step : a.step;
        if (t < 1) t = 1;
        if (a.device_step) seed += (uint32_t)t * 0x85EBCA6Bu;  // a step that is replayed draws anew
        k.step_size = (float)(lr / -expm1((double)t * a.logb1));
        k.r2 = (float)(1.0 / sqrt(-expm1((double)t * a.logb2)));
    }
    const uint32_t chunks = b.first[b.count];
    int i = 0;
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        i = tensor_of(b.first, b.count, c, i);
        const AdamwTensor& t = b.t[i];
        const int64_t from = (int64_t)(c - b.first[i]) * CHUNK, at = from + threadIdx.x * EPT;
        k.decay = live ? (float)(1.0 - lr * (double)t.weight_decay) : t.decay;
        k.key = seed + 0x9E3779B9u * ((t.flags >> ADAMW_ORDINAL) + 1u);
        if (from + CHUNK <= t.n) adamw_elements<EIGHT, true>(t, a, k, at);
        else adamw_elements<EIGHT, false>(t, a, k, at);
    }
}

template <bool WHOLE>
__device__ __forceinline__ void code_values(const uint8_t* codes, uint32_t base, uint32_t top, int left, bf16_t* out) {
    uint32_t c[EPT], r[EPT];
    load_codes<WHOLE>(codes, left, c);
    // 3 mantissa bits: the upper half of the float is the bf16 value itself
#pragma unroll
    for (int e = 0; e < EPT; ++e) r[e] = __float_as_uint(decode(c[e] & top, base)) >> 16 | (c[e] & ~top) << 8;
    store_u16<WHOLE>(out, left, r);
}

__global__ __launch_bounds__(256) void k_adamw_values(int64_t n, const uint8_t* codes, const uint8_t* exps, uint32_t top,
                                                      bf16_t* out) {
    for (int64_t at = (blockIdx.x * 256ll + threadIdx.x) * EPT; at < n; at += gridDim.x * (int64_t)CHUNK) {
        const uint32_t base = code_base(exps[at / ADAMW_BLOCK], top);
        if (at + EPT <= n) code_values<true>(codes + at, base, top, EPT, out + at);
        else code_values<false>(codes + at, base, top, (int)(n - at), out + at);
    }
}

// Sum of 256 doubles over a workgroup, in a fixed order; the result is thread 0's.
__device__ __forceinline__ double block_sum(double x) {
    __shared__ double sh[4];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
    __syncthreads();
    return ((sh[0] + sh[1]) + sh[2]) + sh[3];
}

// Squares are added in 64 bits: a float gradient's square is exact there, cannot overflow, and the sum of 10^9 of
// them keeps its digits. The rate of those operations is far from the bound, which is the read.
// RUN chunks' loads are in flight per thread.
template <int RUN>
__global__ __launch_bounds__(256) void k_grad_norm(NormBatch b) {
    double s[2] = {0.0, 0.0};
    const uint32_t chunks = b.first[b.count];
    int i = 0;
    for (uint32_t c0 = blockIdx.x * RUN; c0 < chunks; c0 += gridDim.x * RUN) {
        float g[RUN][EPT];
#pragma unroll
        for (int u = 0; u < RUN; ++u) {
            if (c0 + u >= chunks) {
#pragma unroll
                for (int e = 0; e < EPT; ++e) g[u][e] = 0.f;
                continue;
            }
            i = tensor_of(b.first, b.count, c0 + u, i);
            const int64_t from = (int64_t)(c0 + u - b.first[i]) * CHUNK, at = from + threadIdx.x * EPT;
            const bool bf = b.flags[i] & ADAMW_GRAD_BF16;
            if (from + CHUNK <= b.n[i]) {
                if (bf) load_bf16<true>((const bf16_t*)b.grad[i] + at, EPT, g[u]);
                else load_f32<true>((const float*)b.grad[i] + at, EPT, g[u]);
            } else {
                const int left = at < b.n[i] ? (int)(b.n[i] - at < EPT ? b.n[i] - at : EPT) : 0;
                if (bf) load_bf16<false>((const bf16_t*)b.grad[i] + at, left, g[u]);
                else load_f32<false>((const float*)b.grad[i] + at, left, g[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < RUN; ++u)
#pragma unroll
            for (int e = 0; e < EPT; ++e) s[e & 1] = fma((double)g[u][e], (double)g[u][e], s[e & 1]);
    }
    const double t = block_sum(s[0] + s[1]);
    if (threadIdx.x == 0) b.part[blockIdx.x] = t;
}

__global__ __launch_bounds__(256) void k_grad_norm_end(const double* part, int64_t n, double scale, double max_norm, float* out) {
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 256) s += part[i];
    s = block_sum(s);
    if (threadIdx.x != 0) return;
    const double norm = sqrt(s) * scale;
    out[0] = (float)norm;
    if (!(norm < (double)__builtin_huge_valf())) out[1] = __builtin_nanf("");  // the step that reads it changes nothing
    else out[1] = norm > max_norm ? (float)(max_norm / norm) : 1.f;
}

constexpr uint32_t STEP_BLOCKS = 4096, NORM_BLOCKS = 2048;

// Fills `first` for up to PER_LAUNCH tensors from t[at]; returns their chunks.
uint32_t place(const AdamwTensor* t, int count, uint32_t* first) {
    uint32_t c = 0;
    for (int i = 0; i < count; ++i) {
        first[i] = c;
        c += (uint32_t)((t[i].n + CHUNK - 1) / CHUNK);
    }
    first[count] = c;
    return c;
}

// Workgroups of the norm, and the chunks that each reads at a time: one until the chip is full, then four (585 M bf16
// values: 340 us one at a time, 250 four; 9.6 M floats 9 and 11, a model of 68000 4 and 7.5).
int norm_run(uint32_t chunks) { return chunks >= 4 * NORM_BLOCKS ? 4 : 1; }
uint32_t norm_blocks(uint32_t chunks) { return chunks < NORM_BLOCKS ? chunks : NORM_BLOCKS; }

}  // namespace

hipError_t launch_adamw(const AdamwTensor* t, int count, const AdamwScalars& a, hipStream_t s) {
    Batch b;
    b.a = a;
    for (int kind = 0; kind < 2; ++kind) {  // tensors with float moments, then those with 8-bit ones
        b.count = 0;
        for (int i = 0; i <= count; ++i) {
            if (i < count && t[i].n > 0 && ((t[i].flags & ADAMW_8BIT) != 0) == (kind == 1)) b.t[b.count++] = t[i];
            if (b.count < PER_LAUNCH && (i < count || b.count == 0)) continue;
            const uint32_t chunks = place(b.t, b.count, b.first), grid = chunks < STEP_BLOCKS ? chunks : STEP_BLOCKS;
            if (kind) hipLaunchKernelGGL(k_adamw<true>, dim3(grid), dim3(256), 0, s, b);
            else hipLaunchKernelGGL(k_adamw<false>, dim3(grid), dim3(256), 0, s, b);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            b.count = 0;
        }
    }
    return hipSuccess;
}

int64_t grad_norm_partials(const AdamwTensor* t, int count) {
    int64_t n = 0;
    uint32_t first[PER_LAUNCH + 1];
    for (int at = 0; at < count; at += PER_LAUNCH) {
        n += norm_blocks(place(t + at, count - at < PER_LAUNCH ? count - at : PER_LAUNCH, first));
    }
    return n;
}

hipError_t launch_grad_norm(const AdamwTensor* t, int count, float grad_scale, float max_norm, double* part, float* out,
                            hipStream_t s) {
    int64_t n = 0;
    for (int at = 0; at < count; at += PER_LAUNCH) {
        NormBatch b;
        b.count = count - at < PER_LAUNCH ? count - at : PER_LAUNCH;
        const uint32_t chunks = place(t + at, b.count, b.first);
        for (int i = 0; i < b.count; ++i) {
            b.grad[i] = t[at + i].grad;
            b.n[i] = t[at + i].n;
            b.flags[i] = t[at + i].flags;
        }
        if (chunks == 0) continue;
        b.part = part + n;
        const uint32_t blocks = norm_blocks(chunks);
        n += blocks;
        if (norm_run(chunks) == 4) hipLaunchKernelGGL(k_grad_norm<4>, dim3(blocks), dim3(256), 0, s, b);
        else hipLaunchKernelGGL(k_grad_norm<1>, dim3(blocks), dim3(256), 0, s, b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(k_grad_norm_end, dim3(1), dim3(256), 0, s, part, n, fabs((double)grad_scale), (double)max_norm, out);
    return hipGetLastError();
}

hipError_t launch_adamw_values(int64_t n, const uint8_t* codes, const uint8_t* exps, bool is_signed, void* out,
                               hipStream_t s) {
    const int64_t b = (n + CHUNK - 1) / CHUNK;
    hipLaunchKernelGGL(k_adamw_values, dim3((unsigned)(b < 8192 ? b : 8192)), dim3(256), 0, s, n, codes, exps,
                       is_signed ? 127u : 255u, (bf16_t*)out);
    return hipGetLastError();
}

}  // namespace rdcn
