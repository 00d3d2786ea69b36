// Log probabilities of given tokens, with ranks, entropy and the likeliest tokens (token_logprobs).
//
// For a row x of V logits (NaN counts as -Inf), a reference m, c = log2(e) / t, z_i = (x_i - m) c:
//     S = sum 2^z_i,   A = sum 2^z_i z_i,   ln p_i = (x_i - m) / t - ln S,   entropy = ln S - ln2 A / S
// One pass over the row: every thread keeps a reference (at first the largest of its warp's first vectors) and the two sums relative
// to it; when the reference moves up by d octaves, S <- 2^-d S and A <- 2^-d (A - d S). The maximum itself is not looked for: sum 2^z z
// of a vector of logits shows when one stands well above the reference, and when one has no weight.
// The likeliest k of V without a sort: the pass also leaves the maximum of every run of 4 vectors (64 or 32 logits) in shared
// memory, and each four threads keep the maximum of all their runs. The k-th largest of those maxima (32 to 128 of them) is a bound
// that at least k logits reach; the few runs that reach it (about k) are read again, their logits that reach it (about k) are
// ranked by counting over 64-bit keys (value, then lower index), which are all different. More than 64 of them (short rows, rows
// with few logits left: a group may hold none) first meet a second bound, the k-th largest key among the maxima of 128 groups of them: 6
// rows of 1575, half masked, k = 32: 6.5 us, 76 by counting over all. Where too many reach the bound (a constant row), the k tokens are found one after the other. With few rows a cluster of up to eight blocks takes a row: slices
// that fit the registers give their candidates without a second read, and the first block joins sums and lists.
// Bound by HBM with many rows: 4096 rows of 128000 bf16 logits 193 us, 5.4 TB/s, 0.83 of the measured copy rate (seven instructions and one
// ex2 per logit, two more for its rank); 1000 rows of fp32 with twenty likeliest 108 us, 0.72 (3.4 rounds of blocks). Few rows by the
// chain of dependent steps: 8 rows of 128000 with twenty likeliest 11.4 us (5.7 without them), 256 of 16384 with five 8.3 us.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "stwq_internal.cuh"
#include "stwq_paged.cuh"
#include "stwq_ptx.cuh"

using namespace stwq_ptx;       // packed fp32 arithmetic
namespace cg = cooperative_groups;

namespace {

constexpr int kMaxV = 360448;
constexpr int kTop = 32;
constexpr int kMaxCluster = 8;
constexpr int kCand = 2048;                  // logits of a block that reach its bound
constexpr int kRuns = 1024;                  // runs that do
constexpr int kFew = 128;                    // groups of candidates for a second bound
constexpr float kLow = -200.0f;              // octaves below which a weight is 0

struct LpParams {
    const void* X;
    int64_t ld;
    int V, k, slice;                         // slice: logits of a block of the cluster
    const float* temperature;
    const int32_t* tokens;
    float *logprobs, *entropy, *top_lp;
    int32_t *ranks, *top_ids;
    uint32_t* status;
};

template <int NT>
struct LpShared {
    float m[NT / 32], s[NT / 32], a[NT / 32];
    uint32_t n[NT / 32];
    __align__(16) float gmax[NT > 128 ? NT / 4 : NT];                          // of the vectors of a group
    float bound;
    uint32_t n_cand, n_runs, n_few;
    unsigned long long best[NT / 32];
    unsigned long long cand[kCand];
    unsigned long long few_max[kFew], few_bound;
    union {                                  // one after the other
        int32_t runs[kRuns];
        unsigned long long few[kTop * kCand / kFew];
    };
    float row_m[kMaxCluster], row_s[kMaxCluster], row_a[kMaxCluster];          // of the blocks of a row, in the first one
    uint32_t row_n[kMaxCluster];
    unsigned long long row_top[kMaxCluster * kTop];
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
    static constexpr int kPer = 32 / sizeof(XT);
    uint32_t w[8];
    __device__ __forceinline__ void load(const XT* p)
    {
        asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
    }
    __device__ __forceinline__ void get(float (&x)[kPer]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (sizeof(XT) == 4) x[i] = __uint_as_float(w[i]);
            else {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[(2 * i + 1) % kPer] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
    // the largest, NaN left out (NaN where there is nothing else)
    __device__ __forceinline__ float largest(const float (&x)[kPer]) const
    {
        if (sizeof(XT) == 4) {
            float m = x[0];
#pragma unroll
            for (int i = 1; i < kPer; ++i) m = fmaxf(m, x[i]);
            return m;
        }
        __nv_bfloat162 m = *reinterpret_cast<const __nv_bfloat162*>(&w[0]);
#pragma unroll
        for (int i = 1; i < 8; ++i) m = __hmax2(m, *reinterpret_cast<const __nv_bfloat162*>(&w[i]));
        return fmaxf(__low2float(m), __high2float(m));
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
__device__ __forceinline__ int index_of(unsigned long long key) { return (int)(0xffffffffu - (uint32_t)key); }
// octaves between a logit and a reference; the reference itself at 0 (also at +Inf), masked ones (NaN too) at kLow
__device__ __forceinline__ float octaves(float x, float m, float c) { return x == m ? 0.0f : fmaxf((x - m) * c, kLow); }
__device__ __forceinline__ bool finite(float v) { return fabsf(v) < INFINITY; }
// m c, while its rounding is a small part of an octave; else Inf
__device__ __forceinline__ float times_c(float m, float c) { return fabsf(m * c) < 1e6f ? m * c : INFINITY; }

// What a thread has seen of a row: a reference m, not far below the largest logit, and S and A relative to it, each as two partial
// sums. With mc = m c rounded to fp32, a logit's octaves are x c - mc in one fma: off from (x - m) c by the rounding of mc, the same for
// every logit (the end takes it out of S, and A / S - log2 S does not see it). Where m c is large, octaves() serves instead.
template <int PER>
struct Sums {
    float m, mc, c;
    uint64_t s, a;
    bool odd;                                // a logit without a weight came by
    __device__ __forceinline__ float z_of(float x) const { return finite(mc) ? fmaxf(fmaf(x, c, -mc), kLow) : octaves(x, m, c); }
    // What sums relative to (m, mc) are multiplied by, in octaves, to stand relative to (to, toc). Where one product is kept, its sums are
    // relative to the rounded product, and the others to the reference itself: its rounding, up to 2^-5 of an octave, is made up for.
    __device__ __forceinline__ float shift(float to, float toc) const
    {
        if (__builtin_expect(finite(mc) && finite(toc), 1)) return fmaxf(mc - toc, kLow);
        if (m == to) return 0.0f;
        const float d = octaves(m, to, c);
        return finite(mc) ? d - fmaf(m, c, -mc) : finite(toc) ? d + fmaf(to, c, -toc) : d;
    }
    __device__ __forceinline__ void raise(float to)       // `to` > m
    {
        const float toc = times_c(to, c), d = shift(to, toc);
        const uint64_t f = dup_f2(ex2_approx(d));
        a = mul_f2(f, fma_f2(dup_f2(d), s, a));
        s = mul_f2(f, s);
        m = to;
        mc = toc;
    }
    __device__ __forceinline__ void add(float x)                             // one logit
    {
        if (x > m) raise(x);
        if (!(x > -INFINITY)) return;
        const float z = z_of(x), w = ex2_approx(z);
        s = add_f2(s, pack_f2(w, 0.0f));
        a = fma_f2(pack_f2(w, 0.0f), pack_f2(z, 0.0f), a);
    }
    // A vector. Neither its maximum nor logits without a weight are looked for: logits above the reference make sum w z grow, -Inf and NaN
    // make it NaN (0 * -Inf). Then, and for vectors of a thread that has met a logit without a weight, more is done.
    __device__ __forceinline__ void add(const float (&x)[PER])
    {
        if (!odd) {
            const uint64_t off = dup_f2(-mc), scale = dup_f2(c);
            uint64_t vs = 0ull, va = 0ull;
#pragma unroll
            for (int j = 0; j < PER; j += 2) {
                const uint64_t z = fma_f2(pack_f2(x[j], x[j + 1]), scale, off);
                float z0, z1;
                unpack_f2(z, z0, z1);
                const uint64_t w = pack_f2(ex2_approx(z0), ex2_approx(z1));
                vs = add_f2(vs, w);
                va = fma_f2(w, z, va);
            }
            float a0, a1;
            unpack_f2(va, a0, a1);
            if (a0 + a1 < 64.0f) {                        // no logit 4 octaves above the reference: ln p near 0 keeps its digits
                s = add_f2(s, vs);
                a = add_f2(a, va);
                return;
            }
        }
        float vm = x[0];
#pragma unroll
        for (int j = 1; j < PER; ++j) vm = fmaxf(vm, x[j]);                   // NaN left out
        if (vm > m) raise(vm);
        float vs = 0.0f, va = 0.0f;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            odd |= !(x[j] > -INFINITY);
            const float z = z_of(x[j]), w = ex2_approx(z);
            vs += w;
            va = fmaf(w, z, va);
        }
        s = add_f2(s, pack_f2(vs, 0.0f));
        a = add_f2(a, pack_f2(va, 0.0f));
    }
    static __device__ __forceinline__ uint64_t add_f2(uint64_t u, uint64_t v)
    {
        uint64_t r;
        asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(u), "l"(v));
        return r;
    }
};
// How many logits of a vector exceed thr.
template <typename XT>
__device__ __forceinline__ uint32_t above(const Vec<XT>& v, const float (&x)[Vec<XT>::kPer], float thr)
{
    if (sizeof(XT) == 4) {
        uint32_t n = 0u;
#pragma unroll
        for (int j = 0; j < Vec<XT>::kPer; ++j) n += x[j] > thr ? 1u : 0u;
        return n;
    }
    const __nv_bfloat162 t = __float2bfloat162_rn(thr);   // thr is a bf16 value; the counts are small integers
    __nv_bfloat162 n = __hgt2(*reinterpret_cast<const __nv_bfloat162*>(&v.w[0]), t);
#pragma unroll
    for (int i = 1; i < 8; ++i) n = __hadd2(n, __hgt2(*reinterpret_cast<const __nv_bfloat162*>(&v.w[i]), t));
    return (uint32_t)(__low2float(n) + __high2float(n));
}

__device__ __forceinline__ float warp_max(float v)                           // NaN left out
{
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// How many of the n keys are larger than key `i`, counted by eight threads together (all 32 of a warp call it); keys that are equal (those
// that are 0) count by position.
__device__ __forceinline__ int place_of(const unsigned long long* keys, int n, int i, int lane)
{
    int ahead_of = 0;
    if (i < n) {
        const unsigned long long key = keys[i];
#pragma unroll 4
        for (int j = lane & 7; j < n; j += 8) {
            const unsigned long long u = keys[j];
            ahead_of += u > key || (u == key && j < i) ? 1 : 0;
        }
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) ahead_of += __shfl_xor_sync(0xffffffffu, ahead_of, o);
    return ahead_of;
}

// A block of NT threads takes a row, or (CL) a slice of one; the first block of the cluster joins the slices. TOP: k > 0.
template <typename XT, int NT, bool CL, bool TOP>
__global__ void __launch_bounds__(NT, CL ? 1 : 1024 / NT) logprob_kernel(const LpParams p)
{
    constexpr int kPer = Vec<XT>::kPer, kWarps = NT / 32, kAhead = CL ? 4 : 2;       // vectors in flight per thread
    extern __shared__ __align__(16) float run_max[];      // [runs of 4 vectors]
    __shared__ LpShared<NT> sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    cg::cluster_group::arrival_token begun;
    if (CL) begun = cg::this_cluster().barrier_arrive();  // waited for before shared memory of another block is written
    const int blocks = CL ? (int)cg::this_cluster().num_blocks() : 1, rank = CL ? (int)cg::this_cluster().block_rank() : 0;
    const int64_t row = CL ? blockIdx.x / blocks : blockIdx.x;
    const int i0 = rank * p.slice, V = max(0, min(p.V - i0, p.slice));           // this block's logits: i0 .. i0 + V - 1 of the row
    const XT* src = reinterpret_cast<const XT*>(p.X) + row * p.ld + i0;
    const int head = min(V, (int)(((32u - (uint32_t)(reinterpret_cast<uintptr_t>(src) & 31u)) & 31u) / sizeof(XT)));
    const int nvec = (V - head) / kPer, tail0 = head + nvec * kPer, ends = head + (V - tail0);
    const int n_runs = (nvec + 3) / 4;
    const XT* body = src + head;
    const bool held = nvec <= kAhead * NT;                // all vectors stay in registers

    Vec<XT> ahead[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
        if (tid + u * NT < nvec) ahead[u].load(body + (int64_t)(tid + u * NT) * kPer);
    // an infinite temperature counts as the largest finite one; the sums of a greedy row are not used
    const float temp = p.temperature != nullptr ? p.temperature[row] : 1.0f;
    const bool greedy = !(temp > 0.0f);
    const float t = greedy ? 1.0f : fminf(temp, 3.402823466e38f), c = fminf(1.4426950408889634f / t, 3.402823466e38f);
    const int given = p.tokens != nullptr ? p.tokens[row] : -1;
    const bool valid = given >= 0 && given < p.V;
    const float xt = valid ? value(reinterpret_cast<const XT*>(p.X) + row * p.ld, given) : -INFINITY;
    const bool ranked = xt > -INFINITY;
    const int token = given - i0;                         // in this block's count
    // what a logit before the token has to exceed to stand before it in the order: the next value below (an equal one does);
    // behind the token it has to exceed the token's
    constexpr uint32_t kUlp = sizeof(XT) == 4 ? 1u : 0x10000u;
    const float below = __fadd_rn(xt, 0.0f) == 0.0f ? -__uint_as_float(kUlp)
                        : __uint_as_float(xt > 0.0f ? __float_as_uint(xt) - kUlp : __float_as_uint(xt) + kUlp);

    // threads that share a group of the bound: four, but one where 32 groups are hardly more than k (300 rows of 4768, k = 32: 18 us, 11.6;
    // k = 5: 6.3, 7.7)
    const int share = NT > 128 || p.k <= 16 ? 4 : 1;
    Sums<kPer> me = {-INFINITY, INFINITY, c, 0ull, 0ull, false};
    uint32_t before = 0u;
    float gmax = -INFINITY, vmax[kAhead];
    if (tid < ends) {                                     // the ragged ends, logit by logit (fewer than 32)
        const int at = tid < head ? tid : tail0 + (tid - head);
        const float x = value(src, at);
        me.add(x);
        gmax = fmaxf(gmax, x);
        if (ranked && x > (at < token ? below : xt)) ++before;
    }
    {   // the largest of the warp's first vectors for a start: logits far above it are rare then, and with them divergence
        float vm = -INFINITY;
        if (tid < nvec) {
            float x[kPer];
            ahead[0].get(x);
            vm = fmaxf(vm, ahead[0].largest(x));
        }
        vm = warp_max(vm);
        if (vm > me.m) me.raise(vm);
    }
    // the token's vector (or -1 where it lies before the vectors or behind): those before it count equal logits too
    const int token_vec = token < head ? -1 : (token - head) / kPer;
    const XT* next = body + (int64_t)(tid + kAhead * NT) * kPer;
    auto vector = [&](int u, int i) {
        float vm = -INFINITY;
        if (i < nvec) {
            float x[kPer];
            ahead[u].get(x);
            if (TOP) vm = fmaxf(vm, ahead[u].largest(x));
            if (ranked) {
                before += above<XT>(ahead[u], x, i < token_vec ? below : xt);
                if (i == token_vec)                       // equal logits before the token, in its own vector
#pragma unroll
                    for (int j = 0; j < kPer; ++j) before += x[j] == xt && head + i * kPer + j < token ? 1u : 0u;
            }
            if (i + kAhead * NT < nvec) ahead[u].load(next);
            me.add(x);
        }
        next += NT * kPer;
        if (TOP) {
            vmax[u] = vm;
            gmax = fmaxf(gmax, vm);
            if (!held) {
                float rm = fmaxf(vm, __shfl_xor_sync(0xffffffffu, vm, 1));
                rm = fmaxf(rm, __shfl_xor_sync(0xffffffffu, rm, 2));
                if ((tid & 3) == 0 && i < nvec) run_max[i >> 2] = rm;
            }
        }
    };
#pragma unroll 1
    for (int b0 = 0; b0 < nvec; b0 += kAhead * NT)
#pragma unroll
        for (int u = 0; u < kAhead; ++u) vector(u, b0 + u * NT + tid);
    // ---- the block's maximum, then its sums relative to it, added in the order of lanes and warps
    const float wm = warp_max(me.m);
    if (lane == 0) sh.m[warp] = wm;
    if (share == 4) {
        gmax = fmaxf(gmax, __shfl_xor_sync(0xffffffffu, gmax, 1));
        gmax = fmaxf(gmax, __shfl_xor_sync(0xffffffffu, gmax, 2));
    }
    if ((tid & (share - 1)) == 0) sh.gmax[tid / share] = gmax;
    if (tid == 0) {
        sh.n_cand = 0u;
        sh.n_runs = 0u;
        sh.n_few = 0u;
    }
    __syncthreads();
    float bm = sh.m[0];                                    // the blocks' common reference
#pragma unroll
    for (int w = 1; w < kWarps; ++w) bm = fmaxf(bm, sh.m[w]);
    {
        float s0, s1, a0, a1;
        unpack_f2(me.s, s0, s1);
        unpack_f2(me.a, a0, a1);
        const float d = me.shift(bm, times_c(bm, c)), f = ex2_approx(d), s = s0 + s1;
        const float ws = warp_sum(f * s), wa = warp_sum(f * fmaf(d, s, a0 + a1));
        before = __reduce_add_sync(0xffffffffu, before);
        if (lane == 0) {
            sh.s[warp] = ws;
            sh.a[warp] = wa;
            sh.n[warp] = before;
        }
    }
    // ---- the k-th largest of the groups' maxima, ties broken by the group: a group's threads count for it
    if (TOP) {
        const int q = tid / share, each = NT / (share * share), from = (tid & (share - 1)) * each;
        const float v = sh.gmax[q];
        int ahead_of = 0;
#pragma unroll 4
        for (int j = from; j < from + each; j += 4) {
            const float4 u = *reinterpret_cast<const float4*>(&sh.gmax[j]);
            ahead_of += (u.x > v || (u.x == v && j < q)) + (u.y > v || (u.y == v && j + 1 < q)) + (u.z > v || (u.z == v && j + 2 < q)) +
                        (u.w > v || (u.w == v && j + 3 < q));
        }
        if (share == 4) {
            ahead_of += __shfl_xor_sync(0xffffffffu, ahead_of, 1);
            ahead_of += __shfl_xor_sync(0xffffffffu, ahead_of, 2);
        }
        if ((tid & (share - 1)) == 0 && ahead_of == p.k - 1) sh.bound = v;
    }
    __syncthreads();
    float bs = 0.0f, ba = 0.0f;
    uint32_t bn = 0u;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        bs += sh.s[w];
        ba += sh.a[w];
        bn += sh.n[w];
    }
    if (CL) cg::this_cluster().barrier_wait(static_cast<cg::cluster_group::arrival_token&&>(begun));
    if (CL && tid == 0) {
        LpShared<NT>* first = cg::this_cluster().map_shared_rank(&sh, 0);
        first->row_m[rank] = bm;
        first->row_s[rank] = bs;
        first->row_a[rank] = ba;
        first->row_n[rank] = bn;
    }

    // ---- the block's likeliest k, as keys in `top`, largest first
    unsigned long long* top = CL ? cg::this_cluster().map_shared_rank(&sh, 0)->row_top + rank * p.k : sh.row_top;
    if (TOP) {
        const float bound = sh.bound;
        auto take = [&](float x, int i) {
            if (x >= bound && x > -INFINITY) {
                const uint32_t at = atomicAdd(&sh.n_cand, 1u);
                if (at < kCand) sh.cand[at] = key_of(x, i0 + i);
            }
        };
        if (tid < ends) {
            const int at = tid < head ? tid : tail0 + (tid - head);
            take(value(src, at), at);
        }
        if (held) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int i = u * NT + tid;
                if (i < nvec && vmax[u] >= bound) {
                    float x[kPer];
                    ahead[u].get(x);
#pragma unroll
                    for (int j = 0; j < kPer; ++j) take(x[j], head + i * kPer + j);
                }
            }
        } else {
            for (int r = tid; r < n_runs; r += NT)
                if (run_max[r] >= bound && run_max[r] > -INFINITY) {
                    const uint32_t at = atomicAdd(&sh.n_runs, 1u);
                    if (at < kRuns) sh.runs[at] = r;
                }
            __syncthreads();
            if (sh.n_runs <= kRuns)
                for (uint32_t r = warp; r < sh.n_runs; r += kWarps) {
                    const int at0 = sh.runs[r] * 4 * kPer;
#pragma unroll
                    for (int j = 0; j < 4 * kPer; j += 32)
                        if (at0 + j + lane < nvec * kPer) take(value(body, at0 + j + lane), head + at0 + j + lane);
                }
        }
        __syncthreads();
        if (sh.n_runs <= kRuns && sh.n_cand <= kCand) {
            int n = (int)sh.n_cand;
            const unsigned long long* cand = sh.cand;
            if (n > kFew / 2) {
                // Short rows with groups hardly more than k, or many without a logit: again a bound, from the maxima of kFew groups of candidates.
                // It is a key, so k groups reach it, with n / kFew candidates each at most.
                unsigned long long best = 0ull;
                if (tid < kFew) {
                    for (int i = tid; i < n; i += kFew) best = sh.cand[i] > best ? sh.cand[i] : best;
                    sh.few_max[tid] = best;
                }
                __syncthreads();
                if (tid < kFew) {
                    int ahead_of = 0;
#pragma unroll 8
                    for (int j = 0; j < kFew; ++j) ahead_of += sh.few_max[j] > best ? 1 : 0;
                    if (ahead_of == p.k - 1) sh.few_bound = best;
                }
                __syncthreads();
                for (int i = tid; i < n; i += NT)
                    if (sh.cand[i] >= sh.few_bound) sh.few[atomicAdd(&sh.n_few, 1u)] = sh.cand[i];
                __syncthreads();
                n = (int)sh.n_few;
                cand = sh.few;
            }
            for (int first = 0; first < n; first += NT / 8) {
                const int i = first + (tid >> 3), at = place_of(cand, n, i, lane);
                if (i < n && at < p.k && (lane & 7) == 0) top[at] = cand[i];
            }
            for (int i = n + tid; i < p.k; i += NT) top[i] = 0ull;
        } else {                                          // too many at the bound: the next largest key, k times
            unsigned long long last = ~0ull;
            for (int q = 0; q < p.k; ++q) {
                unsigned long long best = 0ull;
                for (int i = tid; i < V; i += NT) {
                    const unsigned long long key = key_of(value(src, i), i0 + i);
                    if (key < last && key > best) best = key;
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    const unsigned long long u = __shfl_xor_sync(0xffffffffu, best, o);
                    best = u > best ? u : best;
                }
                if (lane == 0) sh.best[warp] = best;
                __syncthreads();
                for (int w = 0; w < kWarps; ++w) best = sh.best[w] > best ? sh.best[w] : best;
                if (tid == 0) top[q] = best;
                last = best;
                __syncthreads();
            }
        }
    }
    if (CL) {
        cg::this_cluster().sync();
        if (rank != 0) return;
        bm = sh.row_m[0];
        for (int r = 1; r < blocks; ++r) bm = fmaxf(bm, sh.row_m[r]);
        bs = ba = 0.0f;
        bn = 0u;
        for (int r = 0; r < blocks; ++r) {
            const Sums<kPer> part = {sh.row_m[r], times_c(sh.row_m[r], c), c, 0ull, 0ull, false};
            const float d = part.shift(bm, times_c(bm, c)), f = ex2_approx(d);
            bs += f * sh.row_s[r];
            ba += f * fmaf(d, sh.row_s[r], sh.row_a[r]);
            bn += sh.row_n[r];
        }
    } else if (TOP) __syncthreads();

    // ---- the row
    const bool any = bm > -INFINITY;
    const float ln2 = 0.6931471805599453f, bmc = times_c(bm, c), ln_sums = any ? logf(bs) : 0.0f;
    // S relative to bm itself: less the rounding of bm c
    const float ln_s = finite(bmc) ? fmaf(-ln2, fmaf(bm, c, -bmc), ln_sums) : ln_sums;
    // differences may pass the largest number: halves of them, which are exact there. S is rounded and may fall short of the token's own weight.
    const float part = fabsf(bm) > 1e30f ? 0.5f : 1.0f;
    auto ln_p = [&](float x, bool first) {
        if (greedy) return first ? 0.0f : -INFINITY;
        return fminf((x == bm ? 0.0f : fmaf(part, x, -part * bm) / (part * t)) - ln_s, 0.0f);
    };
    if (tid == 0) {
        if (p.tokens != nullptr) {
            float lp;
            if (given == -1) lp = 0.0f;
            else if (!valid) {
                lp = __uint_as_float(0x7fffffffu);
                atomicOr(p.status, STWQ_DEV_TOKEN);
            } else lp = ranked ? ln_p(xt, bn == 0u) : -INFINITY;
            p.logprobs[row] = lp;
            if (p.ranks != nullptr) p.ranks[row] = ranked ? (int32_t)bn : -1;
        }
        if (p.entropy != nullptr) p.entropy[row] = greedy || !any ? 0.0f : fmaxf(fmaf(-ln2, ba / bs, ln_sums), 0.0f);
    }
    if (!TOP) return;
    int32_t* ids = p.top_ids + row * p.k;
    float* lps = p.top_lp + row * p.k;
    auto put = [&](unsigned long long key, int at) {
        ids[at] = key ? index_of(key) : -1;
        lps[at] = key ? ln_p(value_of(key), at == 0) : -INFINITY;
    };
    if (!CL) {
        if (tid < p.k) put(sh.row_top[tid], tid);
        return;
    }
    // the blocks' lists together (p.k apart); places without a token hold 0 and come last
    const int n = blocks * p.k;
    for (int first = 0; first < n; first += NT / 8) {
        const int i = first + (tid >> 3), at = place_of(sh.row_top, n, i, lane);
        if (i < n && at < p.k && (lane & 7) == 0) put(sh.row_top[i], at);
    }
}

template <typename XT, int NT, bool CL, bool TOP>
int launch_lp_as(stwq_ctx* ctx, LpParams& p, int B, int blocks, cudaStream_t st)
{
    constexpr int kRun = 4 * Vec<XT>::kPer;
    p.slice = CL ? ((p.V + blocks - 1) / blocks + kRun - 1) / kRun * kRun : p.V;
    const size_t smem = TOP ? (size_t)(p.slice / kRun + 2) * 4 : 0;
    auto kern = logprob_kernel<XT, NT, CL, TOP>;
    cudaError_t e = cudaSuccess;
    if (smem > 16 * 1024) e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (kMaxV / 32 + 2) * 4);
    if (e != cudaSuccess) return stwq_cuda_fail(ctx, e);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(B * blocks));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    if (CL) {
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = (unsigned)blocks;
        at[0].val.clusterDim.y = 1;
        at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
    }
    e = cudaLaunchKernelEx(&cfg, kern, p);
    ctx->launches += 1;
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? STWQ_OK : stwq_cuda_fail(ctx, e);
}

template <typename XT, int NT, bool CL>
int launch_lp(stwq_ctx* ctx, LpParams& p, int B, int blocks, cudaStream_t st)
{
    return p.k > 0 ? launch_lp_as<XT, NT, CL, true>(ctx, p, B, blocks, st) : launch_lp_as<XT, NT, CL, false>(ctx, p, B, blocks, st);
}

template <typename XT>
int launch_lp_any(stwq_ctx* ctx, LpParams& p, int B, cudaStream_t st)
{
    // few rows: several blocks a row while SMs would idle and a block keeps enough to do (20 likeliest of 32000: 10.2 us in one block, 8.6 in
    // four; of 16384: 7.4 and 11.8)
    int blocks = 1;
    while (blocks < kMaxCluster && B * blocks * 2 <= ctx->sm_count && p.V / (2 * blocks) >= 12288) blocks *= 2;
    if (blocks > 1) return launch_lp<XT, 512, true>(ctx, p, B, blocks, st);
    const int vecs = p.V / Vec<XT>::kPer;
    if (vecs <= 512) return launch_lp<XT, 128, false>(ctx, p, B, 1, st);
    if (vecs <= 2048) return launch_lp<XT, 256, false>(ctx, p, B, 1, st);
    return launch_lp<XT, 512, false>(ctx, p, B, 1, st);
}

}  // namespace

extern "C" int token_logprobs(stwq_ctx* ctx, const void* logits, int x_dtype, int64_t ld, int B, int V, const float* temperature,
                              const int32_t* tokens, float* logprobs, int32_t* ranks, float* entropy, int k, int32_t* top_ids,
                              float* top_logprobs, void* stream)
{
    if (!ctx || !logits) return STWQ_ERR_NULL;
    if ((tokens == nullptr) != (logprobs == nullptr) || (tokens == nullptr && ranks != nullptr)) return STWQ_ERR_NULL;
    if (B <= 0 || B > (1 << 27) || V <= 0 || V > kMaxV || ld < V || k < 0 || k > kTop) return STWQ_ERR_DIM;
    if ((k > 0) != (top_ids != nullptr) || (k > 0) != (top_logprobs != nullptr)) return STWQ_ERR_NULL;
    if (!logprobs && !entropy && k == 0) return STWQ_ERR_NULL;
    if (x_dtype != STWQ_OUT_F32 && x_dtype != STWQ_OUT_BF16) return STWQ_ERR_BITS;
    if ((reinterpret_cast<uintptr_t>(logits) & (x_dtype == STWQ_OUT_F32 ? 3u : 1u)) != 0) return STWQ_ERR_ALIGN;
    // rows are read by many threads while others are already answered
    const int64_t x_bytes = ((B - 1) * ld + V) * (x_dtype == STWQ_OUT_F32 ? 4 : 2), n = (int64_t)B * 4;
    if (stwq_overlap(logits, x_bytes, logprobs, n) || stwq_overlap(logits, x_bytes, ranks, n) || stwq_overlap(logits, x_bytes, entropy, n) ||
        stwq_overlap(logits, x_bytes, top_ids, n * k) || stwq_overlap(logits, x_bytes, top_logprobs, n * k))
        return STWQ_ERR_ALIGN;
    StwqDevGuard g(ctx->device);
    LpParams p;
    p.X = logits; p.ld = ld; p.V = V; p.k = k;
    p.temperature = temperature; p.tokens = tokens;
    p.logprobs = logprobs; p.entropy = entropy; p.top_lp = top_logprobs; p.ranks = ranks; p.top_ids = top_ids;
    p.status = ctx->d_status;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return x_dtype == STWQ_OUT_BF16 ? launch_lp_any<__nv_bfloat16>(ctx, p, B, st) : launch_lp_any<float>(ctx, p, B, st);
}
