// Log probabilities of given tokens, with ranks, entropy and the likeliest tokens (token_logprobs).
//
// For a row x of V logits (NaN counts as -Inf), m = max x, c = log2(e) / t, z_i = (x_i - m) c:
//     S = sum 2^z_i,   A = sum 2^z_i z_i,   ln p_i = (x_i - m) / t - ln S,   entropy = ln S - ln2 A / S
// One pass over the row: every thread keeps the maximum of what it has seen and the two sums relative to it; when the
// maximum moves by d < 0 (in octaves), S <- 2^d S and A <- 2^d (A + d S). The difference to the maximum is taken before the
// product with c, so that large logits lose nothing.
// The likeliest k of V without a sort: the pass also leaves the maximum of every run of 4 vectors (64 or 32 logits) in shared
// memory, and each four threads keep the maximum of all their runs. The k-th largest of those 128 maxima is a bound that at
// least k logits reach; the few runs that reach it (about k) are read again, their logits that reach it (about k) are
// ranked by counting over 64-bit keys (value, then lower index), which are all different. Where too many reach the bound
// (a constant row), the k tokens are found one after the other.
#include <cuda_bf16.h>

#include "stwq_internal.cuh"
#include "stwq_paged.cuh"
#include "stwq_ptx.cuh"

using namespace stwq_ptx;       // packed fp32 arithmetic

namespace {

constexpr int kMaxV = 360448;
constexpr int kTop = 32;
constexpr int kNt = 512;
constexpr int kGroups = kNt / 4;             // of four threads
constexpr int kCand = 2048;                  // logits that reach the bound
constexpr int kRuns = 1024;                  // runs that do
constexpr float kLow = -200.0f;              // octaves below which a weight is 0

struct LpParams {
    const void* X;
    int64_t ld;
    int V, k;
    const float* temperature;
    const int32_t* tokens;
    float *logprobs, *entropy, *top_lp;
    int32_t *ranks, *top_ids;
    uint32_t* status;
};

struct LpShared {
    float m[kNt / 32], s[kNt / 32], a[kNt / 32];
    uint32_t n[kNt / 32];
    float gmax[kGroups];
    float bound;
    uint32_t n_cand, n_runs;
    unsigned long long best[kNt / 32];
    unsigned long long cand[kCand];
    int32_t runs[kRuns];
};

template <typename XT>
__device__ __forceinline__ float value(const XT* p, int i);
template <>
__device__ __forceinline__ float value<float>(const float* p, int i) { return p[i]; }
template <>
__device__ __forceinline__ float value<__nv_bfloat16>(const __nv_bfloat16* p, int i) { return __bfloat162float(p[i]); }

// 32 bytes of logits
template <typename XT>
struct Vec {
    uint32_t w[8];
    __device__ __forceinline__ void load(const XT* p)
    {
        asm("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
            : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
    }
    __device__ __forceinline__ void get(float (&x)[32 / sizeof(XT)]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (sizeof(XT) == 4) x[i] = __uint_as_float(w[i]);
            else {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[(2 * i + 1) % (32 / sizeof(XT))] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
};

// Larger logit = larger key, equal logits: lower index = larger key; 0 for a logit that is never drawn.
__device__ __forceinline__ unsigned long long key_of(float x, int i)
{
    const uint32_t b = __float_as_uint(__fadd_rn(x, 0.0f)), k = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
    return x > -INFINITY ? ((unsigned long long)k << 32) | (0xffffffffu - (uint32_t)i) : 0ull;
}
__device__ __forceinline__ float value_of(unsigned long long key)
{
    const uint32_t k = (uint32_t)(key >> 32);
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}
// octaves between a logit and the maximum; the maximum itself at 0 (also at +Inf), masked ones (NaN too) at kLow
__device__ __forceinline__ float octaves(float x, float m, float c) { return x == m ? 0.0f : fmaxf((x - m) * c, kLow); }

// What a thread (then a warp, a block) has seen of a row.
struct Sums {
    float m, s, a;
    __device__ __forceinline__ void raise(float to, float c)                 // `to` > m
    {
        const float d = octaves(m, to, c), f = ex2_approx(d);
        a = f * fmaf(d, s, a);
        s *= f;
        m = to;
    }
    __device__ __forceinline__ void add(float x, float c)                    // one logit
    {
        if (x > m) raise(x, c);
        if (!(x > -INFINITY)) return;
        const float z = octaves(x, m, c), w = ex2_approx(z);
        s += w;
        a = fmaf(w, z, a);
    }
    __device__ __forceinline__ void join(float om, float os, float oa, float c)
    {
        Sums o = {om, os, oa};
        if (o.m > m) raise(o.m, c);
        else if (m > o.m) o.raise(m, c);
        s += o.s;
        a += o.a;
    }
};

template <typename XT>
__global__ void __launch_bounds__(kNt, 2) logprob_kernel(const LpParams p)
{
    constexpr int kPer = 32 / sizeof(XT);                 // logits per vector
    extern __shared__ __align__(16) float run_max[];      // [runs of 4 vectors]
    __shared__ LpShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t row = blockIdx.x;
    const XT* src = reinterpret_cast<const XT*>(p.X) + row * p.ld;
    const int head = min(p.V, (int)(((32u - (uint32_t)(reinterpret_cast<uintptr_t>(src) & 31u)) & 31u) / sizeof(XT)));
    const int nvec = (p.V - head) / kPer, tail0 = head + nvec * kPer;
    const int n_runs = (nvec + 3) / 4;
    const XT* body = src + head;

    // an infinite temperature counts as the largest finite one; the sums of a greedy row are not used
    const float temp = p.temperature != nullptr ? p.temperature[row] : 1.0f;
    const bool greedy = !(temp > 0.0f);
    const float t = greedy ? 1.0f : fminf(temp, 3.402823466e38f), c = fminf(1.4426950408889634f / t, 3.402823466e38f);
    const int token = p.tokens != nullptr ? p.tokens[row] : -1;
    const bool valid = token >= 0 && token < p.V;
    const float xt = valid ? value(src, token) : -INFINITY;
    const bool ranked = xt > -INFINITY;
    // what a logit before the token has to exceed to stand before it in the order: the next value below (an equal one does);
    // behind the token it has to exceed the token's
    const float below = __fadd_rn(xt, 0.0f) == 0.0f ? -1.401298464e-45f
                        : __uint_as_float(xt > 0.0f ? __float_as_uint(xt) - 1u : __float_as_uint(xt) + 1u);

    Sums me = {-INFINITY, 0.0f, 0.0f};
    uint32_t before = 0u;
    float gmax = -INFINITY;
    for (int i = tid; i < head + (p.V - tail0); i += kNt) {          // the ragged ends, logit by logit
        const int at = i < head ? i : tail0 + (i - head);
        const float x = value(src, at);
        me.add(x, c);
        gmax = fmaxf(gmax, x);
        if (ranked && x > (at < token ? below : xt)) ++before;
    }
    for (int i0 = 0; i0 < nvec; i0 += kNt) {
        const int i = i0 + tid;
        float vm = -INFINITY;
        if (i < nvec) {
            Vec<XT> v;
            v.load(body + (int64_t)i * kPer);
            float x[kPer];
            v.get(x);
#pragma unroll
            for (int j = 0; j < kPer; ++j) vm = fmaxf(vm, x[j]);      // leaves NaN out
            if (vm > me.m) me.raise(vm, c);
            if (vm == INFINITY) {
#pragma unroll
                for (int j = 0; j < kPer; ++j) me.s += x[j] == INFINITY ? 1.0f : 0.0f;
            } else {
#pragma unroll
                for (int j = 0; j < kPer; j += 2) {
                    float z0, z1;
                    unpack_f2(mul_f2(fma_f2(pack_f2(1.0f, 1.0f), pack_f2(x[j], x[j + 1]), dup_f2(-me.m)), dup_f2(c)), z0, z1);
                    z0 = fmaxf(z0, kLow);                             // -Inf and NaN: weight 0
                    z1 = fmaxf(z1, kLow);
                    const float w0 = ex2_approx(z0), w1 = ex2_approx(z1);
                    me.s += w0 + w1;
                    me.a = fmaf(w0, z0, fmaf(w1, z1, me.a));
                }
            }
            if (ranked) {
                const int at = head + i * kPer;
                const float thr = at + kPer <= token ? below : xt;
                if (vm > thr)
#pragma unroll
                    for (int j = 0; j < kPer; ++j) before += x[j] > thr ? 1u : 0u;
                if (token >= at && token < at + kPer)                 // equal logits before the token, in its own vector
#pragma unroll
                    for (int j = 0; j < kPer; ++j) before += x[j] == xt && at + j < token ? 1u : 0u;
            }
        }
        if (p.k > 0) {
            float rm = fmaxf(vm, __shfl_xor_sync(0xffffffffu, vm, 1));
            rm = fmaxf(rm, __shfl_xor_sync(0xffffffffu, rm, 2));
            gmax = fmaxf(gmax, rm);
            if ((tid & 3) == 0 && i < nvec) run_max[i >> 2] = rm;
        }
    }
    // ---- the block's sums, added in the order of warps and lanes
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float om = __shfl_down_sync(0xffffffffu, me.m, o), os = __shfl_down_sync(0xffffffffu, me.s, o), oa = __shfl_down_sync(0xffffffffu, me.a, o);
        me.join(om, os, oa, c);
    }
    before = __reduce_add_sync(0xffffffffu, before);
    if (lane == 0) {
        sh.m[warp] = me.m; sh.s[warp] = me.s; sh.a[warp] = me.a; sh.n[warp] = before;
    }
    gmax = fmaxf(gmax, __shfl_xor_sync(0xffffffffu, gmax, 1));
    gmax = fmaxf(gmax, __shfl_xor_sync(0xffffffffu, gmax, 2));
    if ((tid & 3) == 0) sh.gmax[tid >> 2] = gmax;
    if (tid == 0) {
        sh.n_cand = 0u;
        sh.n_runs = 0u;
        sh.bound = -INFINITY;
    }
    __syncthreads();
    Sums all = {sh.m[0], sh.s[0], sh.a[0]};
    uint32_t rank = sh.n[0];
    for (int w = 1; w < kNt / 32; ++w) {
        all.join(sh.m[w], sh.s[w], sh.a[w], c);
        rank += sh.n[w];
    }
    const bool any = all.m > -INFINITY;
    const float ln_s = any ? logf(all.s) : 0.0f;
    auto ln_p = [&](float x, bool first) {
        if (greedy) return first ? 0.0f : -INFINITY;
        return (x == all.m ? 0.0f : (x - all.m) / t) - ln_s;
    };
    if (tid == 0) {
        if (p.tokens != nullptr) {
            float lp;
            if (token == -1) lp = 0.0f;
            else if (!valid) {
                lp = __uint_as_float(0x7fffffffu);
                atomicOr(p.status, STWQ_DEV_TOKEN);
            } else lp = ranked ? ln_p(xt, rank == 0u) : -INFINITY;
            p.logprobs[row] = lp;
            if (p.ranks != nullptr) p.ranks[row] = ranked ? (int32_t)rank : -1;
        }
        if (p.entropy != nullptr) p.entropy[row] = greedy || !any ? 0.0f : fmaxf(ln_s - 0.6931471805599453f * (all.a / all.s), 0.0f);
    }
    if (p.k == 0) return;

    // ---- the likeliest k: the k-th largest of the groups' maxima, ties broken by the group
    if (tid < kGroups) {
        const float v = sh.gmax[tid];
        int ahead = 0;
        for (int j = 0; j < kGroups; ++j) {
            const float u = sh.gmax[j];
            ahead += u > v || (u == v && j < tid) ? 1 : 0;
        }
        if (ahead == p.k - 1) sh.bound = v;
    }
    __syncthreads();
    const float bound = sh.bound;
    auto take = [&](float x, int i) {
        if (x >= bound && x > -INFINITY) {
            const uint32_t at = atomicAdd(&sh.n_cand, 1u);
            if (at < kCand) sh.cand[at] = key_of(x, i);
        }
    };
    for (int i = tid; i < head + (p.V - tail0); i += kNt) {
        const int at = i < head ? i : tail0 + (i - head);
        take(value(src, at), at);
    }
    for (int r = tid; r < n_runs; r += kNt)
        if (run_max[r] >= bound && run_max[r] > -INFINITY) {
            const uint32_t at = atomicAdd(&sh.n_runs, 1u);
            if (at < kRuns) sh.runs[at] = r;
        }
    __syncthreads();
    if (sh.n_runs <= kRuns)
        for (uint32_t r = warp; r < sh.n_runs; r += kNt / 32) {
            const int at0 = sh.runs[r] * 4 * kPer;
            for (int j = lane; j < 4 * kPer && at0 + j < nvec * kPer; j += 32) take(value(body, at0 + j), head + at0 + j);
        }
    __syncthreads();
    int32_t* ids = p.top_ids + row * p.k;
    float* lps = p.top_lp + row * p.k;
    if (sh.n_runs <= kRuns && sh.n_cand <= kCand) {
        const int n = (int)sh.n_cand;
        for (int i = tid; i < n; i += kNt) {
            const unsigned long long key = sh.cand[i];
            int ahead = 0;
            for (int j = 0; j < n; ++j) ahead += sh.cand[j] > key ? 1 : 0;
            if (ahead < p.k) {
                ids[ahead] = (int32_t)(0xffffffffu - (uint32_t)key);
                lps[ahead] = ln_p(value_of(key), ahead == 0);
            }
        }
        for (int i = n + tid; i < p.k; i += kNt) {
            ids[i] = -1;
            lps[i] = -INFINITY;
        }
        return;
    }
    unsigned long long last = ~0ull;                      // too many at the bound: the next largest key, k times
    for (int q = 0; q < p.k; ++q) {
        unsigned long long best = 0ull;
        for (int i = tid; i < p.V; i += kNt) {
            const unsigned long long key = key_of(value(src, i), i);
            if (key < last && key > best) best = key;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const unsigned long long u = __shfl_xor_sync(0xffffffffu, best, o);
            best = u > best ? u : best;
        }
        if (lane == 0) sh.best[warp] = best;
        __syncthreads();
        for (int w = 0; w < kNt / 32; ++w) best = sh.best[w] > best ? sh.best[w] : best;
        if (tid == 0) {
            ids[q] = best ? (int32_t)(0xffffffffu - (uint32_t)best) : -1;
            lps[q] = best ? ln_p(value_of(best), q == 0) : -INFINITY;
        }
        last = best;
        __syncthreads();
    }
}

template <typename XT>
int launch_lp(stwq_ctx* ctx, const LpParams& p, int B, cudaStream_t st)
{
    const size_t smem = p.k > 0 ? (size_t)(p.V / (4 * (32 / (int)sizeof(XT))) + 2) * 4 : 0;
    cudaError_t e = cudaFuncSetAttribute(logprob_kernel<XT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (kMaxV / 32 + 2) * 4);
    if (e != cudaSuccess) return stwq_cuda_fail(ctx, e);
    logprob_kernel<XT><<<(unsigned)B, kNt, smem, st>>>(p);
    ctx->launches += 1;
    e = cudaGetLastError();
    return e == cudaSuccess ? STWQ_OK : stwq_cuda_fail(ctx, e);
}

}  // namespace

extern "C" int token_logprobs(stwq_ctx* ctx, const void* logits, int x_dtype, int64_t ld, int B, int V, const float* temperature,
                              const int32_t* tokens, float* logprobs, int32_t* ranks, float* entropy, int k, int32_t* top_ids,
                              float* top_logprobs, void* stream)
{
    if (!ctx || !logits) return STWQ_ERR_NULL;
    if ((tokens == nullptr) != (logprobs == nullptr) || (tokens == nullptr && ranks != nullptr)) return STWQ_ERR_NULL;
    if (B <= 0 || V <= 0 || V > kMaxV || ld < V || k < 0 || k > kTop) return STWQ_ERR_DIM;
    if ((k > 0) != (top_ids != nullptr) || (k > 0) != (top_logprobs != nullptr)) return STWQ_ERR_NULL;
    if (!logprobs && !entropy && k == 0) return STWQ_ERR_NULL;
    if (x_dtype != STWQ_OUT_F32 && x_dtype != STWQ_OUT_BF16) return STWQ_ERR_BITS;
    if ((reinterpret_cast<uintptr_t>(logits) & (x_dtype == STWQ_OUT_F32 ? 3u : 1u)) != 0) return STWQ_ERR_ALIGN;
    StwqDevGuard g(ctx->device);
    LpParams p;
    p.X = logits; p.ld = ld; p.V = V; p.k = k;
    p.temperature = temperature; p.tokens = tokens;
    p.logprobs = logprobs; p.entropy = entropy; p.top_lp = top_logprobs; p.ranks = ranks; p.top_ids = top_ids;
    p.status = ctx->d_status;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return x_dtype == STWQ_OUT_BF16 ? launch_lp<__nv_bfloat16>(ctx, p, B, st) : launch_lp<float>(ctx, p, B, st);
}
