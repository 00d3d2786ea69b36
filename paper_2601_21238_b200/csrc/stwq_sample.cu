// Token sampling from logits with temperature, top-k, top-p and min-p, driven by given uniform numbers.
//
// For a row x of V logits (NaN counts as -Inf, a token at -Inf is never drawn), m = max x, temperature t:
//     w_i = exp((x_i - m) / t)                      order: larger x first, equal x by lower index
//     top-k keeps the first k in that order; W = sum of the w kept
//     top-p keeps the shortest prefix of those whose mass reaches p W (at least one token)
//     min-p keeps the w_i >= min_p (w of the largest is 1)
//     token = first kept index i, in index order, with  sum_{j <= i, kept} w_j > u * sum_{kept} w_j
// No sort: a kept set is "every key above K, and the first r tokens (by index) whose key equals K", so both limits
// are order statistics over the monotone 32-bit image of the logits. Each is found in two steps: 64 coarse bins (by
// distance from the maximum; counts for top-k, masses for top-p) give the bin that holds the border, and a radix
// selection (up to 11 bits a pass) over that bin's few members gives K. A coarse bin has a counter per lane, so that the
// atomics of a warp never meet, however the logits cluster. What top-k keeps, if it is at most kList tokens, is
// compacted in index order, and everything after it works on that list.
//
// Weights are integers, round(w 2^42), summed in 64 bits: sums do not depend on the order of the atomics that form
// them, so the same call gives the same token every time, and p W and u W are compared exactly. 2^42 leaves room for
// the sums of 2^19 tokens and puts the rounding of a weight (2^-43 of the largest) far below what could move a border;
// with fp32 weights one row in some ten thousand would fall on the other side of one. exp is table-driven (2^(j/256) from
// a table, a cubic for the rest; the method of Tang, "Table-driven implementation of the exponential function", 1989),
// in fp64: 10 fp64 operations per weight, error below 2e-13.
//
// A row is read from HBM once, into the shared memory of one CTA or of a cluster of up to 8 (the bins are then
// added up over distributed shared memory); every later pass runs on shared memory. What bounds it: instruction issue
// of the passes (a row of 16384 logits with top-k 2000 and top-p takes about 70 thousand cycles of a 512-thread CTA, two
// of which share an SM: 256 rows in 46 us), and the latency of a pass for few rows. HBM needs 1.3 us for the same rows.
// Top-p without top-k computes an fp64 weight for every token: 64 rows of 128000 in 102 to 133 us (how many clusters of eight
// are resident at once differs from GPU to GPU). Without limits the same rows take 56 us, greedy ones 34.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "stwq_internal.cuh"
#include "stwq_paged.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int kBins = 2048;                 // of a radix digit
constexpr int kCoarse = 64;                 // coarse bins, a counter per lane each
constexpr int kList = 2048;                 // tokens of a compacted list
constexpr int kMaxCluster = 8;
constexpr int kMaxSlice = 44 * 1024;         // logits per CTA: 176 KB of shared memory
constexpr int kPairSlice = 17 * 1024;        // two CTAs fit an SM
constexpr int kFrac = 42;                    // fraction bits of a weight
constexpr int kLow = 21;                     // a coarse counter holds the low bits, another the rest: 44 K / 32 adds fit both

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
    double table[256];
    unsigned long long warp_a[32];
    uint32_t warp_n[32];
    unsigned long long total;                // of this CTA: exchanged inside a cluster
    unsigned long long tot[kCoarse];
    unsigned long long sel_above, sel_total;
    uint32_t maxkey, kmin, kmax;
    uint32_t sel_bin;
    uint32_t cnt_total, n_in;
    uint32_t hist_lo[kBins], hist_hi[kBins]; // radix digits; or kCoarse x 32 lanes
    uint32_t list_key[kList], list_idx[kList];                             // what top-k keeps, in index order
    uint32_t in_key[kList];                  // members of the border bin (3 kList of them where the list above is not in use)
};
static_assert(kMaxSlice <= 65536, "16-bit offsets");
static_assert(kCoarse * 32 <= kBins, "coarse counters share the radix histograms");

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
    double c, m;                             // 256 log2(e) / temperature, the row maximum
    float low;                               // below this logit a weight rounds to zero
    uint32_t maxkey;
    const double* table;
    // round(exp((x - m) / t) 2^42); w_out gets the unrounded weight (0 below 2^-46)
    __device__ __forceinline__ unsigned long long fixed(uint32_t key, double& w_out) const
    {
        const float x = value_of(key);
        if (key == maxkey || !(x > low)) {               // the maximum itself (also at +Inf), or rounds to zero
            w_out = key == maxkey ? 1.0 : 0.0;
            return key == maxkey ? 1ull << kFrac : 0ull;
        }
        const double xd = (double)x, magic = 6755399441055744.0;       // 1.5 * 2^52: the integer part lands in the low word
        const double z = (xd - m) * c, s = z + magic;                  // the difference first: large logits lose nothing
        const int n = __double2loint(s);
        const double f = z - (s - magic);                              // |f| <= 1/2, in 256ths of an octave
        // 2^(f/256) - 1 = sum (f ln2/256)^k / k!, the next term is below 1.4e-13
        double q = fma(f, 3.308302680541371e-09, 3.665565596910106e-06);
        q = fma(q, f, 0.0027076061740622863);
        const double t = table[n & 255];
        const double ts = __hiloint2double(__double2hiint(t) + ((n >> 8) << 20), __double2loint(t));
        const double w = fma(ts, f * q, ts);
        w_out = w;
        const double fx = fma(w, (double)(1ull << kFrac), 4503599627370496.0);   // + 2^52
        return (unsigned long long)__double_as_longlong(fx) & 0xfffffffffffffull;
    }
    // the weight itself, however small (for a min-p below 2^-46)
    __device__ __noinline__ double exact(uint32_t key) const
    {
        return key == maxkey ? 1.0 : exp2(((double)value_of(key) - m) * c * 0.00390625);
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
__global__ void __launch_bounds__(NT, 1024 / NT) sample_kernel(const SmpParams p)
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

    if (tid < 256) sh.table[tid] = exp2((double)tid * 0.00390625);
    // ---- the row, once
    uint32_t mx = 0u;
    {
        constexpr int kPer = 16 / sizeof(XT);
        const XT* src = reinterpret_cast<const XT*>(p.X) + (int64_t)row * p.ld + i0;
        const int mis = (int)((reinterpret_cast<uintptr_t>(src) & 15u) / sizeof(XT));
        const int head = mis == 0 ? 0 : min(n, kPer - mis);
        const int nvec = (n - head) / kPer;
        const uint4* vsrc = reinterpret_cast<const uint4*>(src + head);
        for (int i0v = tid; i0v < nvec; i0v += 4 * NT) {                   // four 16-byte loads in flight per thread
            uint4 v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (i0v + q * NT < nvec) v[q] = __ldcs(vsrc + i0v + q * NT);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (i0v + q * NT >= nvec) break;
                const uint32_t w[4] = {v[q].x, v[q].y, v[q].z, v[q].w};
                const int at = head + (i0v + q * NT) * kPer;
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
    // 256 log2(e) / t; an infinite temperature counts as the largest finite one, so that nothing is divided Inf by Inf
    wg.c = greedy ? 256.0 : 369.3299304675746 / (double)fminf(temp, 3.4028234663852886e38f);
    wg.low = (float)fmax(wg.m - 46.0 * 256.0 / wg.c, -3.4028234663852886e38);      // 46 octaves below (an infinite maximum leaves the others at 0)
    wg.maxkey = maxkey;
    wg.table = sh.table;
    const bool tiny_min_p = min_p > 0.0 && min_p < 1.5e-14;

    const int lane = tid & 31, warp = tid >> 5;
    auto clear_hist = [&]() {
        for (int i = tid; i < kBins; i += NT) {
            sh.hist_lo[i] = 0u;
            sh.hist_hi[i] = 0u;
        }
        if (tid == 0) {
            sh.n_in = 0u;
            sh.kmin = 0xffffffffu;
            sh.kmax = 0u;
        }
        __syncthreads();
    };
    // A thread owns a run of consecutive tokens of the source: odd length, so that no two lanes share a bank. What it picks
    // from its run it holds as bits, up to kMasks words of them.
    constexpr int kMasks = 3;
    static_assert((kMaxSlice / NT | 1) <= 32 * kMasks, "bits for a run");
    auto pick = [&](const uint32_t* from, int j0, int j1, uint32_t (&m)[kMasks], auto&& pred) {
#pragma unroll
        for (int q = 0; q < kMasks; ++q) {
            m[q] = 0u;
            const int c = min(32, j1 - j0 - 32 * q);
#pragma unroll 4
            for (int t = 0; t < c; ++t) m[q] |= (pred(from[j0 + 32 * q + t]) ? 1u : 0u) << t;
        }
    };
    auto picked = [&](const uint32_t (&m)[kMasks]) -> uint32_t { return __popc(m[0]) + __popc(m[1]) + __popc(m[2]); };
    auto each = [&](int j0, const uint32_t (&m)[kMasks], auto&& body) {
#pragma unroll
        for (int q = 0; q < kMasks; ++q)
            for (uint32_t x = m[q]; x != 0u; x &= x - 1u) body(j0 + 32 * q + __ffs(x) - 1);
    };
    // sum of v over the threads before this one; total: over the CTA
    auto scan_u32 = [&](uint32_t v, uint32_t& total) -> uint32_t {
        uint32_t x = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t t = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += t;
        }
        __syncthreads();
        if (lane == 31) sh.warp_n[warp] = x;
        __syncthreads();
        const uint32_t w = lane < NT / 32 ? sh.warp_n[lane] : 0u;
        total = __reduce_add_sync(0xffffffffu, w);
        return __reduce_add_sync(0xffffffffu, lane < warp ? w : 0u) + x - v;
    };
    auto run_of = [&](int ns, int& j0, int& j1) {
        const int run = ((ns + NT - 1) / NT) | 1;
        j0 = min(ns, tid * run);
        j1 = min(ns, j0 + run);
    };
    // The first coarse bin in which the running sum reaches `target(total)`; sets sel_bin, sel_above, sel_total.
    auto find_coarse = [&](bool mass, auto&& target) {
        __syncthreads();
        for (int b = warp; b < kCoarse; b += NT / 32) {
            unsigned long long v = sh.hist_lo[b * 32 + lane];
            if (mass) v += (unsigned long long)sh.hist_hi[b * 32 + lane] << kLow;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (lane == 0) sh.tot[b] = v;
        }
        sync_all();                                       // the sums of every CTA are complete
        unsigned long long all_bins = 0;
        if (tid < kCoarse)
            for (int r = 0; r < C; ++r) all_bins += *peer(&sh.tot[tid], r);
        if (CL) {
            sync_all();                                   // and have been read
            if (tid < kCoarse) sh.tot[tid] = all_bins;
            __syncthreads();
        }
        if (warp == 0) {
            static_assert(kCoarse == 64, "two bins per lane");
            const unsigned long long a = sh.tot[2 * lane], b = sh.tot[2 * lane + 1];
            unsigned long long s = a + b;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned long long t = __shfl_up_sync(0xffffffffu, s, o);
                if (lane >= o) s += t;
            }
            const unsigned long long total = __shfl_sync(0xffffffffu, s, 31), tg = target(total);
            const unsigned long long before = s - a - b;
            if (lane == 0) {
                sh.sel_bin = 0xffffffffu;
                sh.sel_total = total;
            }
            __syncwarp();
            if (before < tg && before + a + b >= tg) {
                const bool second = before + a < tg;
                sh.sel_bin = 2 * lane + (second ? 1 : 0);
                sh.sel_above = before + (second ? a : 0ull);
            }
        }
        __syncthreads();
    };
    // K of the border inside a coarse bin: on top of `above`, the running sum (counts or masses) over the bin's keys, from
    // the largest, first reaches `target` at K. member(key): the key is in the bin. Leaves the sum above K in `above`.
    // *whole is set if every token at K is part of it.
    auto select_in_bin = [&](const uint32_t* src, int ns, auto&& member, bool mass, unsigned long long& above, unsigned long long target,
                             bool& whole) -> uint32_t {
        clear_hist();
        // the members, gathered from every CTA of the row into each: from here on no CTA waits for another
        const int cap = src == sh.list_key ? kList : 3 * kList;
        uint32_t* members = src == sh.list_key ? sh.in_key : sh.list_key;
        int j0, j1;
        run_of(ns, j0, j1);
        uint32_t m[kMasks], kmin = 0xffffffffu, kmax = 0u, n_mine;
        pick(src, j0, j1, m, member);
        each(j0, m, [&](int j) {
            kmin = min(kmin, src[j]);
            kmax = max(kmax, src[j]);
        });
        const uint32_t at0 = scan_u32(picked(m), n_mine);
        kmin = __reduce_min_sync(0xffffffffu, kmin);
        kmax = __reduce_max_sync(0xffffffffu, kmax);
        if (lane == 0 && kmax != 0u) {
            atomicMin(&sh.kmin, kmin);
            atomicMax(&sh.kmax, kmax);
        }
        if (tid == 0) sh.n_in = n_mine;
        sync_all();
        uint32_t lo = 0xffffffffu, hi = 0u, n_all = 0u, n_before = 0u;
        for (int r = 0; r < C; ++r) {
            lo = min(lo, *peer(&sh.kmin, r));
            hi = max(hi, *peer(&sh.kmax, r));
            const uint32_t v = *peer(&sh.n_in, r);
            n_all += v;
            n_before += r < rank ? v : 0u;
        }
        const bool listed = n_all <= (uint32_t)cap;       // else the members are looked up in the source again, CTA by CTA
        if (listed) {
            uint32_t at = n_before + at0;
            each(j0, m, [&](int j) { members[at++] = src[j]; });
            sync_all();
            if (CL) {
                // CTA r wrote the members from its n_before on; copy the others'
                uint32_t from = 0u;
                for (int r = 0; r < C; ++r) {
                    const uint32_t v = *peer(&sh.n_in, r);
                    if (r != rank)
                        for (uint32_t i = from + tid; i < from + v; i += NT) members[i] = *peer(&members[i], r);
                    from += v;
                }
                sync_all();
            }
        }
        const uint32_t* from = listed ? members : src;
        const int nf = listed ? (int)n_all : ns;
        auto sync_sel = [&]() {
            if (listed) __syncthreads();
            else sync_all();
        };
        int rem = hi > lo ? 32 - __clz(hi - lo) : 0;      // bits of a key above the bin's lowest that are still open
        uint32_t prefix = 0u;
        unsigned long long at_k = 0ull;
        bool first = true;
        do {
            const int width = min(rem, 11), shift = rem - width;
            const uint32_t open = rem >= 32 ? 0u : prefix >> rem;
            if (!first) {
                for (int i = tid; i < kBins; i += NT) {
                    sh.hist_lo[i] = 0u;
                    sh.hist_hi[i] = 0u;
                }
                __syncthreads();
            }
            first = false;
            for (int i = tid; i < nf; i += NT) {
                const uint32_t k = from[i];
                if (!listed && !member(k)) continue;
                const uint32_t x = k - lo;
                if (rem < 32 && (x >> rem) != open) continue;
                const uint32_t d = (x >> shift) & ((1u << width) - 1u);
                if (mass) {
                    double wd;
                    const unsigned long long w = wg.fixed(k, wd);
                    const uint32_t old = atomicAdd(&sh.hist_lo[d], (uint32_t)w);
                    const uint32_t up = (uint32_t)(w >> 32) + (old + (uint32_t)w < old ? 1u : 0u);
                    if (up != 0u) atomicAdd(&sh.hist_hi[d], up);
                } else atomicAdd(&sh.hist_lo[d], 1u);
            }
            sync_sel();
            constexpr int kPerT = kBins / NT;
            unsigned long long b[kPerT], sum = 0, total;
#pragma unroll
            for (int k = 0; k < kPerT; ++k) {
                const int i = kBins - 1 - (tid * kPerT + k);               // from the top
                unsigned long long v = 0;
                if (listed) v = (unsigned long long)sh.hist_lo[i] + ((unsigned long long)sh.hist_hi[i] << 32);
                else
                    for (int r = 0; r < C; ++r) v += (unsigned long long)*peer(&sh.hist_lo[i], r) + ((unsigned long long)*peer(&sh.hist_hi[i], r) << 32);
                b[k] = v;
                sum += v;
            }
            unsigned long long run = above + block_scan_u64<NT>(sum, sh.warp_a, total);
#pragma unroll
            for (int k = 0; k < kPerT; ++k) {
                if (run < target && run + b[k] >= target) {
                    sh.sel_bin = kBins - 1 - (tid * kPerT + k);
                    sh.sel_above = run;
                    sh.sel_total = b[k];
                }
                run += b[k];
            }
            sync_sel();                                   // chosen, and the histograms read by every CTA
            above = sh.sel_above;
            at_k = sh.sel_total;
            prefix |= sh.sel_bin << shift;
            rem = shift;
            __syncthreads();
        } while (rem > 0);
        whole = above + at_k == target;
        return lo + prefix;
    };
    // Coarse bins, both monotone in the key. For counts: the distance below the maximum, four bins per octave from 2^-6 on.
    // For masses: half octaves of the weight (fp32: only the grouping depends on it).
    const float fmax_ = value_of(maxkey);
    auto distance_bin = [&](uint32_t key) -> int {
        if (key == maxkey) return 0;
        const int e = (int)(__float_as_uint(__fsub_rn(fmax_, value_of(key))) >> 21) - (121 << 2);
        return min(max(e, 0), kCoarse - 1);
    };
    const float half_octaves = greedy ? 1.0f : 2.885390082f / fminf(temp, 3.4028234663852886e38f);
    auto weight_bin = [&](uint32_t key) -> int {
        if (key == maxkey) return 0;
        return (int)fminf(__fmul_rn(__fsub_rn(fmax_, value_of(key)), half_octaves), (float)(kCoarse - 1));
    };

    // kept set: key > K, and the first r tokens with key == K. src: the slice, or a list of it (then all of it is kept so far).
    const uint32_t* src = keys;
    const uint32_t* src_idx = nullptr;
    int ns = n;
    uint32_t K = 0u;
    unsigned long long r_keep = 0ull;
    if (top_k == 1) {                                     // greedy, or top-1: no selection needed
        K = maxkey;
        r_keep = 1ull;
    } else if (top_k > 1 && top_k < p.V) {
        clear_hist();
#pragma unroll 4
        for (int i = tid; i < n; i += NT) {
            const uint32_t k = keys[i];
            if (k != 0u) atomicAdd(&sh.hist_lo[distance_bin(k) * 32 + lane], 1u);
        }
        find_coarse(false, [&](unsigned long long) { return (unsigned long long)top_k; });
        if (sh.sel_bin != 0xffffffffu) {                  // else fewer than k tokens can be drawn: no limit
            const int border = (int)sh.sel_bin;
            unsigned long long above = sh.sel_above;
            __syncthreads();
            bool whole;
            K = select_in_bin(keys, n, [&](uint32_t k) { return k != 0u && distance_bin(k) == border; }, false, above, (unsigned long long)top_k, whole);
            r_keep = (unsigned long long)top_k - above;
            if (whole) {                                  // every token at K is kept: no ranks needed
                K -= 1u;
                r_keep = 0ull;
            }
        }
    }
    // bits of the tokens of the thread's run that are kept: above K, and the ties whose rank, in index order, is below r
    int j0, j1;
    auto kept_bits = [&](uint32_t (&m)[kMasks]) {
        run_of(ns, j0, j1);
        pick(src, j0, j1, m, [&](uint32_t k) { return k > K; });
        if (r_keep > 0) {                                 // uniform
            uint32_t e[kMasks], total;
            pick(src, j0, j1, e, [&](uint32_t k) { return k == K; });
            unsigned long long rank_at = scan_u32(picked(e), total);
            if (CL) {
                if (tid == 0) sh.cnt_total = total;
                sync_all();
                for (int r = 0; r < rank; ++r) rank_at += *peer(&sh.cnt_total, r);
                sync_all();
            }
#pragma unroll
            for (int q = 0; q < kMasks; ++q)
                for (uint32_t x = e[q]; x != 0u && rank_at < r_keep; x &= x - 1u, ++rank_at) m[q] |= x & (0u - x);
        }
    };
    if (K != 0u && top_k > 1 && top_k <= kList) {
        // at most kList tokens are left: list them in index order
        uint32_t m[kMasks], listed;
        kept_bits(m);
        uint32_t at = scan_u32(picked(m), listed);
        each(j0, m, [&](int j) {
            sh.list_key[at] = keys[j];
            sh.list_idx[at++] = (uint32_t)(i0 + j);
        });
        __syncthreads();
        src = sh.list_key;
        src_idx = sh.list_idx;
        ns = (int)listed;
        K = 0u;
        r_keep = 0ull;
    }
    if (top_p < 1.0f && top_k != 1) {
        double wd;
        const unsigned long long wk = r_keep > 0 ? wg.fixed(K, wd) : 0ull;
        const unsigned long long pfx = frac64(top_p);
        unsigned long long W = 0ull, target = 0ull;
        clear_hist();
        for (int i = tid; i < ns; i += NT) {
            const uint32_t k = src[i];
            if (k > K) {
                const unsigned long long w = wg.fixed(k, wd);
                const int bn = weight_bin(k);
                const uint32_t low = (uint32_t)w & ((1u << kLow) - 1u), up = (uint32_t)(w >> kLow);
                if (low != 0u) atomicAdd(&sh.hist_lo[bn * 32 + lane], low);
                if (up != 0u) atomicAdd(&sh.hist_hi[bn * 32 + lane], up);
            }
        }
        auto goal = [&](unsigned long long mass) {
            W = mass + r_keep * wk;
            const unsigned long long t = __umul64hi(pfx, W) + (pfx * W != 0ull ? 1ull : 0ull);     // ceil(p W)
            return t == 0ull ? 1ull : t;
        };
        find_coarse(true, goal);
        const unsigned long long mass = sh.sel_total;
        target = goal(mass);
        if (sh.sel_bin == 0xffffffffu) {                  // every key above K, and some of those equal to K
            const unsigned long long want = wk > 0 ? (target - mass + wk - 1) / wk : r_keep;
            r_keep = min(r_keep, want);
        } else {
            const int border = (int)sh.sel_bin;
            unsigned long long above = sh.sel_above;
            const uint32_t K0 = K;
            bool whole;
            __syncthreads();
            K = select_in_bin(src, ns, [&](uint32_t k) { return k > K0 && weight_bin(k) == border; }, true, above, target, whole);
            const unsigned long long wp = wg.fixed(K, wd);
            r_keep = wp > 0 ? (target - above + wp - 1) / wp : 1ull;
        }
        __syncthreads();
    }

    // ---- mass and number of the kept tokens. Over a slice the kept ones are listed first (16-bit offsets), so that the fp64
    // weights run on full warps; then a warp takes a contiguous segment and a lane sums each quarter of it.
    uint16_t* offs = reinterpret_cast<uint16_t*>(sh.list_key);             // 6 kList of them, behind one another
    bool by_offset = false;
    if (src == keys) {
        uint32_t m[kMasks], listed;
        kept_bits(m);
        uint32_t at = scan_u32(picked(m), listed);
        by_offset = listed <= 6 * kList;                  // uniform over the CTA; the slice is shorter than 2^16
        if (by_offset) {
            each(j0, m, [&](int j) { offs[at++] = (uint16_t)j; });
            ns = (int)listed;
        } else {
            // too many for the list: mark the others in place (their keys are not needed any more)
            for (int q = 0; q < kMasks; ++q)
                for (int t = 0; t < 32 && j0 + 32 * q + t < j1; ++t)
                    if (((m[q] >> t) & 1u) == 0u) keys[j0 + 32 * q + t] = 0u;
        }
        __syncthreads();
    } else if (K != 0u || r_keep > 0) {
        uint32_t m[kMasks];
        kept_bits(m);
        __syncthreads();
        for (int q = 0; q < kMasks; ++q)
            for (int t = 0; t < 32 && j0 + 32 * q + t < j1; ++t)
                if (((m[q] >> t) & 1u) == 0u) sh.list_key[j0 + 32 * q + t] = 0u;
        __syncthreads();
    }
    constexpr int kW = NT / 32;
    const int seg = ((ns + kW - 1) / kW + 31) & ~31, quarter = ((seg / 4) + 31) & ~31;
    const int s0 = min(ns, warp * seg), s1 = min(ns, s0 + seg);
    unsigned long long part[4] = {0ull, 0ull, 0ull, 0ull};
    uint32_t cnt = 0;
    auto weight_at = [&](int j, bool& kept) -> unsigned long long {        // of token j + lane (key 0: not kept)
        const uint32_t k = j + lane < s1 ? (by_offset ? keys[offs[j + lane]] : src[j + lane]) : 0u;
        kept = false;
        if (k == 0u) return 0ull;
        double w;
        const unsigned long long f = wg.fixed(k, w);
        if (tiny_min_p && w == 0.0) w = wg.exact(k);
        kept = w >= min_p;
        return kept ? f : 0ull;
    };
#pragma unroll
    for (int q = 0; q < 4; ++q)
        for (int j = s0 + q * quarter; j < min(s1, s0 + (q + 1) * quarter); j += 32) {
            bool kept;
            part[q] += weight_at(j, kept);
            cnt += kept;
        }
    unsigned long long sum = part[0] + part[1] + part[2] + part[3];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    cnt = __reduce_add_sync(0xffffffffu, cnt);
    __syncthreads();
    if (lane == 0) {
        sh.warp_a[warp] = sum;
        sh.warp_n[warp] = cnt;
    }
    __syncthreads();
    unsigned long long all = 0ull, base = 0ull;           // of the row; before this warp
    uint32_t kept_cnt = __reduce_add_sync(0xffffffffu, lane < kW ? sh.warp_n[lane] : 0u);
#pragma unroll 4
    for (int w = 0; w < kW; ++w) {
        const unsigned long long v = sh.warp_a[w];
        all += v;
        base += w < warp ? v : 0ull;
    }
    if (CL) {
        if (tid == 0) {
            sh.total = all;
            sh.cnt_total = kept_cnt;
        }
        sync_all();
        all = 0ull;
        kept_cnt = 0u;
        for (int r = 0; r < C; ++r) {
            const unsigned long long t = *peer(&sh.total, r);
            if (r < rank) base += t;
            all += t;
            kept_cnt += *peer(&sh.cnt_total, r);
        }
    }
    const unsigned long long thr = __umul64hi(frac64(p.u[row]), all);  // floor(u W) < W
    if (base <= thr && thr < base + sum) {                // the warp whose segment holds the token finds the quarter, then walks it
        unsigned long long at = base;
        int j = s0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            unsigned long long v = part[q];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (at <= thr && thr >= at + v && q < 3) {
                at += v;
                j = s0 + (q + 1) * quarter;
            } else break;
        }
        for (; j < s1 && at <= thr; j += 32) {
            bool kept;
            const unsigned long long f = weight_at(j, kept);
            unsigned long long s = f;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned long long t = __shfl_up_sync(0xffffffffu, s, o);
                if (lane >= o) s += t;
            }
            if (f > 0ull && at + s > thr && at + s - f <= thr) {
                p.tokens[row] = src_idx != nullptr ? (int32_t)src_idx[j + lane] : i0 + (by_offset ? (int)offs[j + lane] : j + lane);
                if (p.probs) p.probs[row] = (float)((double)f / (double)all);
                if (p.kept) p.kept[row] = (int32_t)kept_cnt;
            }
            at += __shfl_sync(0xffffffffu, s, 31);
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
    // slices that leave room for two CTAs per SM, if a cluster of 8 gets there; more CTAs per row while SMs would idle
    while (C < kMaxCluster && ((V + C - 1) / C > kPairSlice || (B * C * 2 <= ctx->sm_count && V / C >= 4096))) C *= 2;
    if ((V + C - 1) / C > kMaxSlice) return STWQ_ERR_DIM;
    SmpParams p;
    p.X = logits; p.ld = ld; p.V = V;
    p.chunk = ((V + C - 1) / C + 31) & ~31;
    p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p; p.u = u;
    p.tokens = tokens; p.probs = probs; p.kept = kept;
    const size_t smem = (size_t)p.chunk * 4;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool bf = x_dtype == STWQ_OUT_BF16;
    if (C > 1) return bf ? launch_sample<512, true, __nv_bfloat16>(ctx, p, B, C, smem, st) : launch_sample<512, true, float>(ctx, p, B, C, smem, st);
    return bf ? launch_sample<512, false, __nv_bfloat16>(ctx, p, B, C, smem, st) : launch_sample<512, false, float>(ctx, p, B, C, smem, st);
}
