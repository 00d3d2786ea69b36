// Token sampling from logits with temperature, top-k, top-p and min-p, driven by given uniform numbers.
//
// For a row x of V logits (NaN counts as -Inf, a token at -Inf is never drawn), m = max x, temperature t:
//     w_i = exp((x_i - m) / t)                      order: larger x first, equal x by lower index
//     top-k keeps the first k in that order; W = sum of the w kept
//     top-p keeps the shortest prefix of those whose mass reaches p W (at least one token)
//     min-p keeps the w_i >= min_p (w of the largest is 1)
//     token = first kept index i, in index order, with  sum_{j <= i, kept} w_j > u * sum_{kept} w_j
// No sort: a kept set is "every key above K, and the first r tokens (by index) whose key equals K", so both limits
// are order statistics, found by radix selection over the monotone 32-bit image of the logits (11 + 11 + 10
// bits, one histogram per digit): counts for top-k, masses for top-p.
//
// Weights are integers, round(w 2^43), summed in 64 bits: sums do not depend on the order of the atomics that form
// them, so the same call gives the same token every time, and p W and u W are compared exactly. 2^43 leaves room for
// 2^20 tokens and puts the rounding of a weight (2^-44 of the largest) far below the fp64 rounding of a long sum;
// with fp32 weights one row in some ten thousand would fall on the other side of a border. exp is table-driven
// (2^(j/64) from a table, a degree-4 polynomial for the rest; the method of Tang, "Table-driven implementation of
// the exponential function", 1989), in fp64: 11 fp64 operations per weight, error below 5e-14.
//
// A row is read from HBM once, into the shared memory of one CTA or of a cluster of up to 8 (the histograms are then
// added up over distributed shared memory); every later pass runs on shared memory.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "stwq_internal.cuh"
#include "stwq_paged.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int kBins = 2048;
constexpr int kMaxCluster = 8;
constexpr int kMaxSlice = 50 * 1024;         // logits per CTA: 200 KB of shared memory
constexpr int kFrac = 43;                    // fraction bits of a weight

struct SmpParams {
    const void* X;
    int64_t ld;
    int V, chunk;                            // chunk: tokens per CTA of a cluster
    const float *temperature, *top_p, *min_p, *u;
    const int32_t* top_k;
    int32_t* tokens;
    float* probs;
    int32_t* kept;
};

struct SmpShared {
    double table[64];
    unsigned long long warp_a[32], warp_b[32];
    unsigned long long total;                // of this CTA: exchanged inside a cluster
    unsigned long long sel_above;
    uint32_t maxkey;
    uint32_t sel_bin;
    uint32_t cnt_total, ties;
    uint32_t hist_lo[kBins], hist_hi[kBins];
};

// fp32 -> unsigned key, larger logit = larger key, -0 = +0; 0 for NaN and -Inf (never drawn)
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(__fadd_rn(x, 0.0f));
    const uint32_t k = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
    return x > -INFINITY ? k : 0u;
}
__device__ __forceinline__ float value_of(uint32_t k)
{
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}

struct Weigher {
    double m, c;                             // row maximum, 64 log2(e) / temperature
    uint32_t maxkey;
    const double* table;
    // round(exp((x - m) / t) 2^43); w_out gets the unrounded weight
    __device__ __forceinline__ unsigned long long fixed(uint32_t key, double& w_out) const
    {
        if (key == maxkey) {
            w_out = 1.0;
            return 1ull << kFrac;
        }
        const double z = ((double)value_of(key) - m) * c;
        if (!(z > -64.0 * 46.0)) {           // below 2^-46: rounds to zero (also x - m = -Inf)
            w_out = z > -64.0 * 1000.0 ? exp2(z * 0.015625) : 0.0;
            return 0ull;
        }
        const double magic = 6755399441055744.0;                       // 1.5 * 2^52: the integer part lands in the low word
        const double s = z + magic;
        const int n = __double2loint(s);
        const double f = z - (s - magic);                              // |f| <= 1/2, in 64ths of an octave
        // 2^(f/64) - 1 = sum (f ln2/64)^k / k!
        double q = 5.732851688640402e-10;                             // (ln2/64)^4 / 24
        q = fma(q, f, 2.1173137155464774e-07);                         // (ln2/64)^3 / 6
        q = fma(q, f, 5.864904955056169e-05);                           // (ln2/64)^2 / 2
        q = fma(q, f, 0.010830424696249145);                           // ln2 / 64
        const double t = table[n & 63];
        const double ts = __hiloint2double(__double2hiint(t) + ((n >> 6) << 20), __double2loint(t));
        const double w = fma(ts, f * q, ts);
        w_out = w;
        const double fx = fma(w, (double)(1ull << kFrac), 4503599627370496.0);   // + 2^52
        return (unsigned long long)__double_as_longlong(fx) & 0xfffffffffffffull;
    }
};

// x * 2^64 for x in [0, 1), exact for every fp32 that has no bits below 2^-64
__device__ __forceinline__ unsigned long long frac64(float x)
{
    if (!(x > 0.0f)) return 0ull;
    if (x >= 1.0f) return ~0ull;
    return __double2ull_rz((double)x * 18446744073709551616.0);
}

template <int NT>
__device__ __forceinline__ unsigned long long block_scan_u64(unsigned long long v, unsigned long long* sums, unsigned long long& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long t = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += t;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = s;
    __syncthreads();
    if (warp == 0) {
        unsigned long long w = lane < NT / 32 ? sums[lane] : 0ull;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long t = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += t;
        }
        if (lane < NT / 32) sums[lane] = w;
    }
    __syncthreads();
    total = sums[NT / 32 - 1];
    return (warp > 0 ? sums[warp - 1] : 0ull) + s - v;
}

template <int NT, bool CL, typename XT>
__global__ void __launch_bounds__(NT) sample_kernel(const SmpParams p)
{
    extern __shared__ __align__(16) uint32_t keys[];
    __shared__ SmpShared sh;
    const int C = CL ? (int)cg::this_cluster().num_blocks() : 1;
    const int rank = CL ? (int)cg::this_cluster().block_rank() : 0;
    const int row = CL ? (int)(blockIdx.x / C) : (int)blockIdx.x;
    const int tid = threadIdx.x;
    auto sync_all = [&]() {
        if (CL) cg::this_cluster().sync();
        else __syncthreads();
    };
    auto peer = [&](auto* ptr, int r) { return CL ? cg::this_cluster().map_shared_rank(ptr, r) : ptr; };

    const int i0 = rank * p.chunk;
    const int n = max(0, min(p.V - i0, p.chunk));
    const int run = ((n + NT - 1) / NT) | 1;              // consecutive tokens per thread: odd, so that no two lanes share a bank

    if (tid < 64) sh.table[tid] = exp2((double)tid * 0.015625);
    // ---- the row, once
    uint32_t mx = 0u;
    {
        constexpr int kPer = 16 / sizeof(XT);
        const XT* src = reinterpret_cast<const XT*>(p.X) + (int64_t)row * p.ld + i0;
        const int mis = (int)((reinterpret_cast<uintptr_t>(src) & 15u) / sizeof(XT));
        const int head = mis == 0 ? 0 : min(n, kPer - mis);
        const int nvec = (n - head) / kPer;
        const uint4* vsrc = reinterpret_cast<const uint4*>(src + head);
        for (int i = tid; i < nvec; i += NT) {
            const uint4 v = __ldcs(vsrc + i);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            const int at = head + i * kPer;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (sizeof(XT) == 4) {
                    const uint32_t a = key_of(__uint_as_float(w[k]));
                    keys[at + k] = a;
                    mx = max(mx, a);
                } else {
                    const uint32_t a = key_of(__uint_as_float(w[k] << 16)), b = key_of(__uint_as_float(w[k] & 0xffff0000u));
                    keys[at + 2 * k] = a;
                    keys[at + 2 * k + 1] = b;
                    mx = max(mx, max(a, b));
                }
            }
        }
        const int rest = n - head - nvec * kPer;
        if (tid < head + rest) {
            const int i = tid < head ? tid : head + nvec * kPer + (tid - head);
            const uint32_t a = key_of((float)src[i]);
            keys[i] = a;
            mx = max(mx, a);
        }
    }
    mx = __reduce_max_sync(0xffffffffu, mx);
    if (tid == 0) sh.maxkey = 0u;
    __syncthreads();
    if ((tid & 31) == 0) atomicMax(&sh.maxkey, mx);
    sync_all();
    uint32_t maxkey = 0u;
    for (int r = 0; r < C; ++r) maxkey = max(maxkey, *peer(&sh.maxkey, r));
    if (maxkey == 0u) {                                   // nothing can be drawn
        if (rank == 0 && tid == 0) {
            p.tokens[row] = -1;
            if (p.probs) p.probs[row] = 0.0f;
            if (p.kept) p.kept[row] = 0;
        }
        sync_all();
        return;
    }

    const float temp = p.temperature ? p.temperature[row] : 1.0f;
    const bool greedy = !(temp > 0.0f);
    const int top_k = greedy ? 1 : (p.top_k ? p.top_k[row] : 0);
    const float top_p = p.top_p ? p.top_p[row] : 1.0f;
    const float min_pf = p.min_p ? p.min_p[row] : 0.0f;
    const double min_p = min_pf > 0.0f ? fmin((double)min_pf, 1.0) : 0.0;
    Weigher wg;
    wg.m = (double)value_of(maxkey);
    wg.c = greedy ? 64.0 : 92.33248261689366 / (double)temp;      // 64 log2(e)
    wg.maxkey = maxkey;
    wg.table = sh.table;

    // The bin (from the top) in which the running sum of the histograms, on top of `above`, reaches `target`;
    // `total` receives the sum over all bins. False if the target is not reached.
    auto find_bin = [&](unsigned long long above, unsigned long long target, bool mass, unsigned long long& total, uint32_t& bin,
                        unsigned long long& above_out) -> bool {
        constexpr int kPerT = kBins / NT;
        unsigned long long b[kPerT], sum = 0;
#pragma unroll
        for (int k = 0; k < kPerT; ++k) {
            const int i = kBins - 1 - (tid * kPerT + k);  // from the top
            unsigned long long v = 0;
            for (int r = 0; r < C; ++r) {
                v += *peer(&sh.hist_lo[i], r);
                if (mass) v += (unsigned long long)*peer(&sh.hist_hi[i], r) << 32;
            }
            b[k] = v;
            sum += v;
        }
        unsigned long long at = above + block_scan_u64<NT>(sum, sh.warp_a, total);
        if (tid == 0) sh.sel_bin = 0xffffffffu;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPerT; ++k) {
            if (at < target && at + b[k] >= target) {
                sh.sel_bin = kBins - 1 - (tid * kPerT + k);
                sh.sel_above = at;
            }
            at += b[k];
        }
        __syncthreads();
        bin = sh.sel_bin;
        above_out = sh.sel_above;
        return bin != 0xffffffffu;
    };
    auto clear_hist = [&]() {
        for (int i = tid; i < kBins; i += NT) {
            sh.hist_lo[i] = 0u;
            sh.hist_hi[i] = 0u;
        }
        __syncthreads();
    };
    const int shift_of[3] = {21, 10, 0}, bins_of[3] = {2048, 2048, 1024};

    // kept set: key > K, and the first r tokens with key == K
    uint32_t K = 0u;
    unsigned long long r_keep = 0ull;
    if (top_k == 1) {                                     // greedy, or top-1: no selection needed
        K = maxkey;
        r_keep = 1ull;
    } else if (top_k > 1 && top_k < p.V) {
        unsigned long long above = 0ull;
        uint32_t prefix = 0u;
        bool found = true;
#pragma unroll
        for (int ps = 0; ps < 3 && found; ++ps) {
            clear_hist();
            const int sh_hi = ps == 0 ? 32 : shift_of[ps - 1];
            for (int i = tid; i < n; i += NT) {
                const uint32_t k = keys[i];
                if (k != 0u && (ps == 0 || ((k ^ prefix) >> (sh_hi & 31)) == 0u))
                    atomicAdd(&sh.hist_lo[(k >> shift_of[ps]) & (bins_of[ps] - 1)], 1u);
            }
            sync_all();
            unsigned long long total, ab;
            uint32_t bin;
            found = find_bin(above, (unsigned long long)top_k, false, total, bin, ab);
            if (found) {
                above = ab;
                prefix |= bin << shift_of[ps];
            }
            sync_all();                                   // the histograms have been read by every CTA
        }
        if (found) {                                      // else fewer than k tokens can be drawn: no limit
            K = prefix;
            r_keep = (unsigned long long)top_k - above;
        }
    }
    if (top_p < 1.0f && top_k != 1) {
        double wd;
        const unsigned long long wk = r_keep > 0 ? wg.fixed(K, wd) : 0ull;
        const unsigned long long pfx = frac64(top_p);
        unsigned long long above = 0ull, target = 0ull;
        uint32_t prefix = 0u;
        bool inside = true;
#pragma unroll
        for (int ps = 0; ps < 3 && inside; ++ps) {
            clear_hist();
            const int sh_hi = ps == 0 ? 32 : shift_of[ps - 1];
            for (int i = tid; i < n; i += NT) {
                const uint32_t k = keys[i];
                if (k > K && (ps == 0 || ((k ^ prefix) >> (sh_hi & 31)) == 0u)) {
                    const unsigned long long w = wg.fixed(k, wd);
                    const uint32_t bin = (k >> shift_of[ps]) & (bins_of[ps] - 1);
                    const uint32_t lo = (uint32_t)w;
                    const uint32_t old = atomicAdd(&sh.hist_lo[bin], lo);
                    const uint32_t hi = (uint32_t)(w >> 32) + (old + lo < old ? 1u : 0u);
                    if (hi != 0u) atomicAdd(&sh.hist_hi[bin], hi);
                }
            }
            sync_all();
            unsigned long long total, ab;
            uint32_t bin;
            if (ps == 0) {
                // the mass first: the target is p times it
                unsigned long long sum = 0;
                for (int i = tid; i < kBins; i += NT)
                    for (int r = 0; r < C; ++r)
                        sum += (unsigned long long)*peer(&sh.hist_lo[i], r) + ((unsigned long long)*peer(&sh.hist_hi[i], r) << 32);
                unsigned long long mass;
                block_scan_u64<NT>(sum, sh.warp_b, mass);
                const unsigned long long W = mass + r_keep * wk;
                target = __umul64hi(pfx, W) + (pfx * W != 0ull ? 1ull : 0ull);         // ceil(p W)
                if (target == 0ull) target = 1ull;
                if (mass < target) {                      // every key above K, and some of those equal to K
                    inside = false;
                    const unsigned long long want = wk > 0 ? (target - mass + wk - 1) / wk : r_keep;
                    r_keep = min(r_keep, want);
                    sync_all();
                    break;
                }
            }
            find_bin(above, target, true, total, bin, ab);
            above = ab;
            prefix |= bin << shift_of[ps];
            sync_all();
        }
        if (inside) {
            K = prefix;
            const unsigned long long wp = wg.fixed(K, wd);
            r_keep = wp > 0 ? (target - above + wp - 1) / wp : 1ull;
        }
    }

    // ---- ranks of the tokens whose key equals K, in index order
    const int j0 = min(n, tid * run), j1 = min(n, j0 + run);
    unsigned long long tie_at = 0ull;
    if (r_keep > 0) {
        unsigned long long ties = 0, tot;
        for (int j = j0; j < j1; ++j) ties += keys[j] == K;
        tie_at = block_scan_u64<NT>(ties, sh.warp_a, tot);
        if (CL) {
            if (tid == 0) sh.total = tot;
            sync_all();
            for (int r = 0; r < rank; ++r) tie_at += *peer(&sh.total, r);
            sync_all();
        }
    }
    // ---- mass and number of the kept tokens
    unsigned long long sum = 0, tie = tie_at;
    uint32_t cnt = 0;
    for (int j = j0; j < j1; ++j) {
        const uint32_t k = keys[j];
        const bool eq = k == K && r_keep > 0;
        if ((k > K) || (eq && tie < r_keep)) {
            double w;
            const unsigned long long f = wg.fixed(k, w);
            if (w >= min_p) {
                sum += f;
                ++cnt;
            }
        }
        tie += eq;
    }
    unsigned long long mine, kept_cnt;
    const unsigned long long before_cta = block_scan_u64<NT>(sum, sh.warp_a, mine);
    block_scan_u64<NT>((unsigned long long)cnt, sh.warp_b, kept_cnt);
    unsigned long long all = mine, base = 0ull;
    if (CL) {
        if (tid == 0) {
            sh.total = mine;
            sh.cnt_total = (uint32_t)kept_cnt;
        }
        sync_all();
        all = 0ull;
        kept_cnt = 0ull;
        for (int r = 0; r < C; ++r) {
            const unsigned long long t = *peer(&sh.total, r);
            if (r < rank) base += t;
            all += t;
            kept_cnt += *peer(&sh.cnt_total, r);
        }
    }
    const unsigned long long thr = __umul64hi(frac64(p.u[row]), all);  // floor(u W) < W
    const unsigned long long from = base + before_cta;
    const bool owner = from <= thr && thr < from + sum;
    const unsigned own = __ballot_sync(0xffffffffu, owner);
    if (own != 0u) {
        // the warp of the thread whose run holds the token walks that run 32 tokens at a time
        const int src = __ffs(own) - 1, lane = tid & 31;
        const int a0 = __shfl_sync(0xffffffffu, j0, src), a1 = __shfl_sync(0xffffffffu, j1, src);
        unsigned long long at = __shfl_sync(0xffffffffu, from, src), tr = __shfl_sync(0xffffffffu, tie_at, src);
        for (int j = a0; j < a1; j += 32) {
            const uint32_t k = j + lane < a1 ? keys[j + lane] : 0u;
            const bool eq = j + lane < a1 && k == K && r_keep > 0;
            const unsigned eqs = __ballot_sync(0xffffffffu, eq);
            unsigned long long f = 0ull;
            if (j + lane < a1 && (k > K || (eq && tr + __popc(eqs & ((1u << lane) - 1u)) < r_keep))) {
                double w;
                f = wg.fixed(k, w);
                if (!(w >= min_p)) f = 0ull;
            }
            unsigned long long s = f;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned long long t = __shfl_up_sync(0xffffffffu, s, o);
                if (lane >= o) s += t;
            }
            if (f > 0ull && at + s > thr && at + s - f <= thr) {
                p.tokens[row] = i0 + j + lane;
                if (p.probs) p.probs[row] = (float)((double)f / (double)all);
                if (p.kept) p.kept[row] = (int32_t)kept_cnt;
            }
            at += __shfl_sync(0xffffffffu, s, 31);
            tr += __popc(eqs);
        }
    }
    if (CL) sync_all();                                   // no CTA leaves while another reads its shared memory
}

template <int NT, bool CL, typename XT>
int launch_sample(stwq_ctx* ctx, const SmpParams& p, int B, int C, size_t smem, cudaStream_t st)
{
    auto kern = sample_kernel<NT, CL, XT>;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSlice * 4);
    if (e != cudaSuccess) return stwq_cuda_fail(ctx, e);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(B * C));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    if (CL) {
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = (unsigned)C;
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

}  // namespace

extern "C" int sample_tokens(stwq_ctx* ctx, const void* logits, int x_dtype, int64_t ld, int B, int V, const float* temperature,
                             const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* tokens,
                             float* probs, int32_t* kept, void* stream)
{
    if (!ctx || !logits || !u || !tokens) return STWQ_ERR_NULL;
    if (B <= 0 || B > (1 << 27) || V <= 0 || V > kMaxSlice * kMaxCluster || ld < V) return STWQ_ERR_DIM;
    if (x_dtype != STWQ_OUT_F32 && x_dtype != STWQ_OUT_BF16) return STWQ_ERR_BITS;
    if ((reinterpret_cast<uintptr_t>(logits) & (x_dtype == STWQ_OUT_F32 ? 3u : 1u)) != 0) return STWQ_ERR_ALIGN;
    StwqDevGuard g(ctx->device);
    int C = 1;
    while ((V + C - 1) / C > kMaxSlice || (C < kMaxCluster && B * C * 2 <= ctx->sm_count && V / C >= 4096)) C *= 2;
    SmpParams p;
    p.X = logits; p.ld = ld; p.V = V;
    p.chunk = ((V + C - 1) / C + 31) & ~31;
    p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p; p.u = u;
    p.tokens = tokens; p.probs = probs; p.kept = kept;
    const size_t smem = (size_t)p.chunk * 4;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool bf = x_dtype == STWQ_OUT_BF16;
    if (C > 1) return bf ? launch_sample<1024, true, __nv_bfloat16>(ctx, p, B, C, smem, st) : launch_sample<1024, true, float>(ctx, p, B, C, smem, st);
    return bf ? launch_sample<1024, false, __nv_bfloat16>(ctx, p, B, C, smem, st) : launch_sample<1024, false, float>(ctx, p, B, C, smem, st);
}
