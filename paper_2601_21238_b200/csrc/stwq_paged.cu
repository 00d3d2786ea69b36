// The paged KV cache around attention: page bookkeeping of a step (page_plan), and the pass that turns the
// output of the qkv linear into normed, rotated queries and into cache entries (qk_norm_rope, kv_append_paged).
//
// page_plan. With page size S, request b holding c[b] tokens and getting n[b] more:
//     cu = exclusive prefix sum of n,  kv[b] = c[b] + n[b],
//     before[b] = ceil(c[b] / S), after[b] = ceil(kv[b] / S), first[b] = exclusive prefix sum of (after - before),
//     table[b, before[b] + i] = free[first[b] + i]                         for i < after[b] - before[b]
//     slot[cu[b] + i] = table[b, (c[b] + i) / S] * S + (c[b] + i) % S,  pos[cu[b] + i] = c[b] + i
// A few kilobytes in, 8 bytes per token out: bound by the launch. Every block repeats the two prefix sums over
// the requests (they fit its shared memory), so that one launch does all of it without a device-wide step.
//
// qk_norm_rope / kv_append_paged. For a head vector x of d channels, in fp32:
//     RMS: y = x / sqrt(mean(x^2) + eps) * w,   L2: y = x / max(|x|, eps) * w,   none: y = x
//     rotation of the pair (a, b) = (y[i], y[i + rot/2]) or (y[2i], y[2i + 1]) by the table's angle:
//     (a c - b s, b c + a s), channels from rot on as they are.
// One pass: each vector is read once, its sum of squares is a shuffle reduction inside the 8, 16 or 32 lanes that
// hold it (8 channels = one or two 16-byte accesses per lane), the partner of a half-split pair comes by shuffle
// from the lane rot/16 further. Bound by HBM. A lane group takes up to kHeads heads of one kind of one token: their
// loads are in flight together, and weights and angles are read once for all of them. Measured: 8192 rows of 90 heads of
// 64, bf16 in and out, 45 us, 4.2 TB/s; 65536 rows of 32 heads of 80, fp32, 275 us, 4.9 TB/s (0.64 and 0.74 of the
// measured copy rate; a vector of 80 leaves 6 of its 16 lanes idle). 256-thread blocks at 79 registers took 55 and 319 us; held to
// 64 registers, the forms for up to 128 channels spill 12 to 56 bytes a thread. The same 8192 rows into code pages take 53 us.
#include <cuda_bf16.h>

#include "stwq_internal.cuh"
#include "stwq_paged.cuh"
#include "stwq_ptx.cuh"

using namespace stwq_ptx;       // packed fp32 arithmetic

namespace {

constexpr int kPlanThreads = 512;
constexpr int kPlanMaxB = 4096;

struct PlanParams {
    const int32_t *cached, *fresh, *free_pages;
    int B, F, S, W, T;
    int32_t *table, *cu, *kv, *slots, *pos, *used;
    uint32_t* status;
};

// exclusive scan of v over the block (kPlanThreads threads); returns the prefix and the total
__device__ __forceinline__ long long block_scan(long long v, long long* warp_sums, long long& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += u;
    }
    __syncthreads();                                     // the sums of an earlier call have been read
    if (lane == 31) warp_sums[warp] = s;
    __syncthreads();
    long long before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 32; ++w) {
        const long long x = warp_sums[w];
        if (w < warp) before += x;
        all += x;
    }
    total = all;
    return before + s - v;
}

// last index b in [0, B) with a[b] <= x (a ascending, a[0] = 0 <= x): the request that owns element x of the
// concatenation; requests of length zero share their start with the next one and are passed over
__device__ __forceinline__ int owner(const int32_t* a, int B, int x)
{
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const PlanParams p)
{
    extern __shared__ int32_t plan_smem[];
    int32_t* s_cu = plan_smem;                           // [B + 1] first token of each request
    int32_t* s_pg = s_cu + p.B + 1;                      // [B + 1] first new page of each request
    int32_t* s_c = s_pg + p.B + 1;                       // [B] cached tokens
    __shared__ long long warp_sums[kPlanThreads / 32];
    const int per = (p.B + kPlanThreads - 1) / kPlanThreads;
    const int b0 = min((int)threadIdx.x * per, p.B), b1 = min(b0 + per, p.B);
    const long long cap = (long long)p.W * p.S;          // tokens a row of the table can hold
    bool bad = false;

    long long n = 0;
    for (int b = b0; b < b1; ++b) {
        long long c = p.cached[b];
        if (c < 0 || c > cap) { bad = true; c = c < 0 ? 0 : cap; }
        s_c[b] = (int32_t)c;
        n += max(p.fresh[b], 0);
        bad |= p.fresh[b] < 0;
    }
    long long total;
    long long at = block_scan(n, warp_sums, total);
    bad |= total > p.T;
    for (int b = b0; b < b1; ++b) {                      // tokens that the slot list cannot hold are cut off
        s_cu[b] = (int32_t)min(at, (long long)p.T);
        at += max(p.fresh[b], 0);
    }
    const int tokens = (int)min(total, (long long)p.T);
    if (threadIdx.x == 0) s_cu[p.B] = tokens;
    __syncthreads();

    long long need = 0;
    for (int b = b0; b < b1; ++b) {
        const long long c = s_c[b], want = c + (s_cu[b + 1] - s_cu[b]), kv = min(want, cap);
        bad |= want > cap;
        need += (kv + p.S - 1) / p.S - (c + p.S - 1) / p.S;
    }
    long long pages;
    long long pg = block_scan(need, warp_sums, pages);
    bad |= pages > p.F;
    const bool writer = blockIdx.x == 0;
    for (int b = b0; b < b1; ++b) {
        const long long c = s_c[b], kv = min(c + (s_cu[b + 1] - s_cu[b]), cap);
        const long long before = (c + p.S - 1) / p.S, take = (kv + p.S - 1) / p.S - before;
        const long long got = max(0ll, min(take, p.F - pg));
        s_pg[b] = (int32_t)min(pg, 0x7fffffffll);
        if (writer) {
            p.cu[b] = s_cu[b];
            p.kv[b] = (int32_t)(got < take ? min(kv, max(c, (before + got) * p.S)) : kv);   // what its pages can hold
        }
        pg += take;
    }
    const int n_pages = (int)min(pages, 0x7fffffffll);
    if (threadIdx.x == 0) s_pg[p.B] = n_pages;
    if (writer && threadIdx.x == 0) {
        p.cu[p.B] = tokens;
        p.used[0] = (int32_t)min(pages, (long long)p.F);
    }
    __syncthreads();

    // A row holds below 2^31 tokens, and so does a step: lengths, positions and the roundings to pages fit unsigned 32 bits.
    const uint32_t S = (uint32_t)p.S;
    const int stride = gridDim.x * kPlanThreads, me = blockIdx.x * kPlanThreads + threadIdx.x;
    for (long long x = me; x < n_pages; x += stride) {
        const int b = owner(s_pg, p.B, (int)x);
        const int col = (int)(((uint32_t)s_c[b] + S - 1u) / S) + (int)(x - s_pg[b]);
        if (col < p.W) p.table[(int64_t)b * p.W + col] = x < p.F ? p.free_pages[x] : -1;
    }
    for (long long t = me; t < p.T; t += stride) {
        int slot = -1, pos = -1;
        if (t < tokens) {
            const int b = owner(s_cu, p.B, (int)t);
            const uint32_t c = (uint32_t)s_c[b], at = c + (uint32_t)(t - s_cu[b]);
            const uint32_t pi = at / S, before = (c + S - 1u) / S, off = at - pi * S;
            pos = (int)min(at, 0x7fffffffu);                        // a token that far lies behind its row
            int id = -1;
            if (pi < (uint32_t)p.W) {
                if (pi < before) {
                    id = p.table[(int64_t)b * p.W + pi];            // the page that the cached tokens end in
                    bad |= id < 0;
                } else {
                    const int64_t f = (int64_t)s_pg[b] + (int)(pi - before);
                    if (f < p.F) id = p.free_pages[f];
                    bad |= f < p.F && id < 0;
                }
            }
            if (id >= 0 && (int64_t)id * p.S + off <= 0x7fffffff) slot = id * p.S + (int)off;
            else bad = true;
        }
        p.slots[t] = slot;
        p.pos[t] = pos;
    }
    if (bad) atomicOr(p.status, STWQ_DEV_PAGES);
}

// ------------------------------------------------------------------------------------------ norm + rotation + append
constexpr int kHeads = 4;          // heads of one token that a lane group takes
constexpr int kNrThreads = 128;

struct NrParams {
    const void* X;
    int64_t ld;                    // elements between rows of X
    const int32_t *pos, *slots;
    int64_t T;
    int Hq, Hkv, d, norm, rot, pairs, P, need_pos;
    float eps;
    const float *wq, *wk;
    int wq_hs, wk_hs;              // elements between the weights of two heads (0 = shared)
    const float* cs;
    void *Qo, *Ko;
    int64_t q_ts, q_hs, k_ts, k_hs;
    void *Kp, *Vp;
    int S;
    int64_t n_slots;
    const float *s_k, *s_v;
    int qmin, qmax;
    uint32_t* status;
};

__device__ __forceinline__ float min_nan(float a, float b)          // NaN if either is
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8])
{
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8])
{
    const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8])
{
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8_codes(int8_t* p, const float (&v)[8], const float (&r)[8], int qmin, int qmax)
{
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        w[i >> 2] |= (uint32_t)(stwq_code(__fmul_rn(v[i], r[i]), qmin, qmax) & 0xFF) << (8 * (i & 3));
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}

// LPV lanes hold a head vector. XT: element type of X; QT: of the queries (and of the keys when DEST is 0).
// DEST 0: keys to a dense tensor, values untouched; 1: bf16 pages; 2: pages of codes.
// blockIdx.y selects a chunk of kHeads heads of one kind (queries, then keys, then values), so that the kind, its weights
// and its destination are the same for the whole block; a lane group takes one token.
template <int LPV, typename XT, typename QT, int DEST>
__global__ void __launch_bounds__(kNrThreads, 8) norm_rope_kernel(const NrParams p)
{
    const int l = threadIdx.x % LPV;
    const int64_t t = (int64_t)blockIdx.x * (kNrThreads / LPV) + threadIdx.x / LPV;
    const int e0 = 8 * l;
    const int nq = (p.Hq + kHeads - 1) / kHeads, nk = (p.Hkv + kHeads - 1) / kHeads;
    int y = blockIdx.y;
    const int kind = y < nq ? 0 : (y < nq + nk ? 1 : 2);
    y -= kind == 0 ? 0 : (kind == 1 ? nq : nq + nk);
    const int h0 = y * kHeads;                            // first head, counted within its kind
    const int heads = min(kHeads, (kind == 0 ? p.Hq : p.Hkv) - h0);
    const int hx = h0 + (kind == 0 ? 0 : (kind == 1 ? p.Hq : p.Hq + p.Hkv));              // and in the row of X
    const bool in = t < p.T && e0 < p.d;
    const int pos = t < p.T ? p.pos[t] : -1;
    const bool row = in && pos != -1;                     // position -1 marks a padding row: nothing is written for it
    const bool zero = p.need_pos && !(pos >= 0 && pos < p.P);     // no angle, no key scale: the query row becomes zeros
    if (row && zero && l == 0 && blockIdx.y == 0) atomicOr(p.status, STWQ_DEV_POS_RANGE);

    float x[kHeads][8];
    const XT* src = reinterpret_cast<const XT*>(p.X) + t * p.ld + (int64_t)hx * p.d + e0;
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
        if (row && k < heads) load8(src + k * p.d, x[k]);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[k][i] = 0.0f;
        }
    }
    // ---- where the vectors go
    int64_t dst = -1, dst_step = 0;                       // of the first head, elements to the next; -1: nowhere
    if (DEST != 0 && kind != 0) {
        if (row) {
            int slot = p.slots[t];
            if (slot < -1 || slot >= p.n_slots) {
                if (l == 0 && kind == 1 && h0 == 0) atomicOr(p.status, STWQ_DEV_PAGES);
                slot = -1;
            }
            if (slot >= 0 && !zero) {
                const int page = slot / p.S;
                dst = (((int64_t)page * p.Hkv + h0) * p.S + (slot - page * p.S)) * p.d + e0;
                dst_step = (int64_t)p.S * p.d;
            }
        }
    } else if (row) {
        dst = t * (kind == 0 ? p.q_ts : p.k_ts) + h0 * (kind == 0 ? p.q_hs : p.k_hs) + e0;
        dst_step = kind == 0 ? p.q_hs : p.k_hs;
    }

    if (kind != 2) {
        const unsigned lanes = LPV == 32 ? 0xffffffffu : ((1u << (LPV & 31)) - 1u) << (threadIdx.x & 31 & ~(LPV - 1));
        if (p.norm != STWQ_NORM_NONE) {
            const float* wp = kind == 0 ? p.wq : p.wk;
            const int whs = kind == 0 ? p.wq_hs : p.wk_hs;
            float w[8];
            if (wp != nullptr && e0 < p.d) load8(wp + (int64_t)h0 * whs + e0, w);
            else {
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = 1.0f;
            }
            float ss[kHeads];
#pragma unroll
            for (int k = 0; k < kHeads; ++k) {
                uint64_t s2 = mul_f2(pack_f2(x[k][0], x[k][1]), pack_f2(x[k][0], x[k][1]));
#pragma unroll
                for (int i = 2; i < 8; i += 2) s2 = fma_f2(pack_f2(x[k][i], x[k][i + 1]), pack_f2(x[k][i], x[k][i + 1]), s2);
                float a, b;
                unpack_f2(s2, a, b);
                ss[k] = a + b;
            }
#pragma unroll
            for (int o = LPV / 2; o > 0; o >>= 1)
#pragma unroll
                for (int k = 0; k < kHeads; ++k) ss[k] += __shfl_xor_sync(lanes, ss[k], o);
            const float inv_d = 1.0f / (float)p.d, inv_eps = 1.0f / p.eps;
#pragma unroll
            for (int k = 0; k < kHeads; ++k) {
                // 1 / max(|x|, eps) = min(rsqrt(x.x), 1 / eps); rsqrtf is good to 2 ulp, and takes 0 and Inf as the formula does.
                // The minimum keeps NaN, as the formula does: a vector with one is NaN in all its channels.
                const float r = p.norm == STWQ_NORM_RMS ? rsqrtf(fmaf(ss[k], inv_d, p.eps)) : min_nan(rsqrtf(ss[k]), inv_eps);
                if (k > 0 && whs != 0 && wp != nullptr && k < heads && e0 < p.d) load8(wp + (int64_t)(h0 + k) * whs + e0, w);
#pragma unroll
                for (int i = 0; i < 8; i += 2)
                    unpack_f2(mul_f2(mul_f2(pack_f2(x[k][i], x[k][i + 1]), dup_f2(r)), pack_f2(w[i], w[i + 1])), x[k][i], x[k][i + 1]);
            }
        }
        if (p.rot > 0) {
            // the angles of this lane's channels: one per channel (half-split) or one per pair
            const int half = p.rot >> 1;
            const bool turns = e0 < p.rot;
            float c[8], s[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) { c[i] = 1.0f; s[i] = 0.0f; }
            if (row && turns && !zero) {
                const float* cs = p.cs + (int64_t)pos * p.rot;
                if (p.pairs) {
                    const float4 a = __ldg(reinterpret_cast<const float4*>(cs + e0 / 2)), b = __ldg(reinterpret_cast<const float4*>(cs + half + e0 / 2));
                    c[0] = a.x; c[1] = a.y; c[2] = a.z; c[3] = a.w;
                    s[0] = b.x; s[1] = b.y; s[2] = b.z; s[3] = b.w;
                } else {
                    const int i0 = e0 < half ? e0 : e0 - half;
                    load8(cs + i0, c);
                    load8(cs + half + i0, s);
                }
            }
            if (p.pairs) {
                if (turns) {
#pragma unroll
                    for (int k = 0; k < kHeads; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float a = x[k][2 * i], b = x[k][2 * i + 1];
                            unpack_f2(fma_f2(pack_f2(b, a), pack_f2(-s[i], s[i]), mul_f2(pack_f2(a, b), dup_f2(c[i]))), x[k][2 * i], x[k][2 * i + 1]);
                        }
                }
            } else {
                const bool lower = e0 < half;
                const int from = turns ? (lower ? l + half / 8 : l - half / 8) : l;
                if (turns && lower) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[i] = -s[i];
                }
#pragma unroll
                for (int k = 0; k < kHeads; ++k)
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const uint64_t o = pack_f2(__shfl_sync(lanes, x[k][i], from, LPV), __shfl_sync(lanes, x[k][i + 1], from, LPV));
                        if (turns)                        // (an Inf in a channel that is not turned stays one: 0 * Inf is not 0)
                            unpack_f2(fma_f2(o, pack_f2(s[i], s[i + 1]), mul_f2(pack_f2(x[k][i], x[k][i + 1]), pack_f2(c[i], c[i + 1]))), x[k][i], x[k][i + 1]);
                    }
            }
        }
        if (zero) {
#pragma unroll
            for (int k = 0; k < kHeads; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[k][i] = 0.0f;
        }
    }
    if (dst < 0) return;
    if (DEST == 2 && kind != 0) {
        const float rk = kind == 1 ? __frcp_rn(p.s_k[pos]) : 1.0f;
        int8_t* out = reinterpret_cast<int8_t*>(kind == 1 ? p.Kp : p.Vp) + dst;
#pragma unroll
        for (int k = 0; k < kHeads; ++k) {
            if (k >= heads) break;
            float r[8];
            if (kind == 1) {
#pragma unroll
                for (int i = 0; i < 8; ++i) r[i] = rk;
            } else {
                load8(p.s_v + (int64_t)(h0 + k) * p.d + e0, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) r[i] = __frcp_rn(r[i]);
            }
            store8_codes(out + k * dst_step, x[k], r, p.qmin, p.qmax);
        }
    } else if (DEST != 0 && kind != 0) {
        __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(kind == 1 ? p.Kp : p.Vp) + dst;
#pragma unroll
        for (int k = 0; k < kHeads; ++k)
            if (k < heads) store8(out + k * dst_step, x[k]);
    } else {
        QT* out = reinterpret_cast<QT*>(kind == 0 ? p.Qo : p.Ko) + dst;
#pragma unroll
        for (int k = 0; k < kHeads; ++k)
            if (k < heads) store8(out + k * dst_step, x[k]);
    }
}

template <int LPV, typename XT>
int launch_nr(stwq_ctx* ctx, const NrParams& p, int q_f32, int dest, cudaStream_t st)
{
    const int64_t blocks = (p.T + kNrThreads / LPV - 1) / (kNrThreads / LPV);
    const int nq = (p.Hq + kHeads - 1) / kHeads, nk = (p.Hkv + kHeads - 1) / kHeads;
    if (blocks > 0x7fffffff || nq + 2 * nk > 65535) return STWQ_ERR_DIM;
    const dim3 gx((unsigned)blocks, (unsigned)(nq + (dest == 0 ? nk : 2 * nk)));
    if (dest == 0) {
        if (q_f32) norm_rope_kernel<LPV, XT, float, 0><<<gx, kNrThreads, 0, st>>>(p);
        else norm_rope_kernel<LPV, XT, __nv_bfloat16, 0><<<gx, kNrThreads, 0, st>>>(p);
    } else if (dest == 1) norm_rope_kernel<LPV, XT, __nv_bfloat16, 1><<<gx, kNrThreads, 0, st>>>(p);
    else norm_rope_kernel<LPV, XT, __nv_bfloat16, 2><<<gx, kNrThreads, 0, st>>>(p);
    ctx->launches += 1;
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? STWQ_OK : stwq_cuda_fail(ctx, e);
}

int launch_nr_any(stwq_ctx* ctx, const NrParams& p, int x_bf16, int q_f32, int dest, cudaStream_t st)
{
    if (p.d <= 64) return x_bf16 ? launch_nr<8, __nv_bfloat16>(ctx, p, q_f32, dest, st) : launch_nr<8, float>(ctx, p, q_f32, dest, st);
    if (p.d <= 128) return x_bf16 ? launch_nr<16, __nv_bfloat16>(ctx, p, q_f32, dest, st) : launch_nr<16, float>(ctx, p, q_f32, dest, st);
    return x_bf16 ? launch_nr<32, __nv_bfloat16>(ctx, p, q_f32, dest, st) : launch_nr<32, float>(ctx, p, q_f32, dest, st);
}

// Checks shared by the two entry points; fills the common part of the parameters.
int nr_common(NrParams& p, const void* X, int64_t ld, int x_dtype, const int32_t* pos_ids, int64_t T, int Hq, int Hkv, int d,
              const float* w_q, int w_q_heads, const float* w_k, int w_k_heads, int norm, float eps, const float* cs, int rot,
              int rope, int P, const void* Qo, int64_t q_ts, int64_t q_hs, int q_dtype)
{
    if (!X || !pos_ids || !Qo) return STWQ_ERR_NULL;
    if (cs == nullptr && rot != 0) return STWQ_ERR_NULL;
    if (T <= 0 || T > 0x7fffffff || Hq <= 0 || Hkv <= 0 || Hq > (1 << 16) || Hkv > (1 << 16) || d <= 0 || d > 256 || P <= 0) return STWQ_ERR_DIM;
    if (rot < 0 || rot > d) return STWQ_ERR_DIM;
    if (x_dtype != STWQ_OUT_F32 && x_dtype != STWQ_OUT_BF16) return STWQ_ERR_BITS;
    if (q_dtype != STWQ_OUT_F32 && q_dtype != STWQ_OUT_BF16) return STWQ_ERR_BITS;
    if (norm < STWQ_NORM_NONE || norm > STWQ_NORM_L2 || (rope != STWQ_ROPE_HALF && rope != STWQ_ROPE_PAIRS)) return STWQ_ERR_BITS;
    if (!(eps >= 0.0f)) return STWQ_ERR_DIM;
    if (w_q_heads != 0 && w_q_heads != 1 && w_q_heads != Hq) return STWQ_ERR_DIM;
    if (w_k_heads != 0 && w_k_heads != 1 && w_k_heads != Hkv) return STWQ_ERR_DIM;
    if ((w_q == nullptr) != (w_q_heads == 0) || (w_k == nullptr) != (w_k_heads == 0)) return STWQ_ERR_NULL;
    const int64_t width = (int64_t)(Hq + 2 * (int64_t)Hkv) * d;
    const int64_t elem16x = x_dtype == STWQ_OUT_F32 ? 4 : 8;      // elements per 16 bytes
    const int64_t elem16q = q_dtype == STWQ_OUT_F32 ? 4 : 8;
    if (ld < width) return STWQ_ERR_DIM;
    if ((d & 15) != 0 || (rot & 15) != 0 || ld % elem16x != 0 || !stwq_aligned16(X) || !stwq_aligned16(Qo) || !stwq_aligned16(cs) ||
        !stwq_aligned16(w_q) || !stwq_aligned16(w_k))
        return STWQ_ERR_ALIGN;
    if (!stwq_disjoint(T, Hq, d, q_ts, q_hs)) return STWQ_ERR_DIM;
    if (q_ts % elem16q != 0 || q_hs % elem16q != 0) return STWQ_ERR_ALIGN;
    p.X = X; p.ld = ld; p.pos = pos_ids; p.T = T;
    p.Hq = Hq; p.Hkv = Hkv; p.d = d; p.norm = norm; p.rot = rot; p.pairs = rope == STWQ_ROPE_PAIRS; p.P = P;
    p.eps = eps; p.wq = w_q; p.wk = w_k;
    p.wq_hs = w_q_heads > 1 ? d : 0;
    p.wk_hs = w_k_heads > 1 ? d : 0;
    p.cs = cs;
    p.Qo = const_cast<void*>(Qo); p.q_ts = q_ts; p.q_hs = q_hs;
    p.need_pos = rot > 0;
    return STWQ_OK;
}

}  // namespace

extern "C" {

int page_plan(stwq_ctx* ctx, const int32_t* cached_lens, const int32_t* new_lens, int B, const int32_t* free_pages, int n_free,
              int page_size, int32_t* block_table, int W, int32_t* cu_new, int32_t* kv_lens, int32_t* slot_map, int32_t* pos_ids,
              int64_t T, int32_t* pages_used, void* stream)
{
    if (!ctx || !cached_lens || !new_lens || !block_table || !cu_new || !kv_lens || !slot_map || !pos_ids || !pages_used) return STWQ_ERR_NULL;
    if (!free_pages && n_free > 0) return STWQ_ERR_NULL;
    if (B <= 0 || B > kPlanMaxB || n_free < 0 || W <= 0 || page_size <= 0 || T <= 0 || T > 0x7fffffff) return STWQ_ERR_DIM;
    if ((int64_t)W * page_size > 0x7fffffff) return STWQ_ERR_DIM;
    // every block reads the inputs for itself, while the first already writes the lists: not in place
    const struct { const int32_t* at; int64_t n; } in[] = {{cached_lens, B}, {new_lens, B}, {free_pages, n_free}},
        out[] = {{block_table, (int64_t)B * W}, {cu_new, B + 1}, {kv_lens, B}, {slot_map, T}, {pos_ids, T}, {pages_used, 1}};
    for (const auto& a : in)
        for (const auto& b : out)
            if (a.n > 0 && a.at < b.at + b.n && b.at < a.at + a.n) return STWQ_ERR_ALIGN;
    StwqDevGuard g(ctx->device);
    PlanParams p;
    p.cached = cached_lens; p.fresh = new_lens; p.free_pages = free_pages;
    p.B = B; p.F = n_free; p.S = page_size; p.W = W; p.T = (int)T;
    p.table = block_table; p.cu = cu_new; p.kv = kv_lens; p.slots = slot_map; p.pos = pos_ids; p.used = pages_used;
    p.status = ctx->d_status;
    const size_t smem = (size_t)(3 * B + 2) * 4;
    if (smem > 48 * 1024 - 256) {                        // beside the kernel's static shared memory (the warps' sums)
        const cudaError_t e = cudaFuncSetAttribute(page_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (3 * kPlanMaxB + 2) * 4);
        if (e != cudaSuccess) return stwq_cuda_fail(ctx, e);
    }
    const int64_t want = (T + kPlanThreads - 1) / kPlanThreads;
    const int blocks = (int)(want < ctx->sm_count ? want : ctx->sm_count);
    page_plan_kernel<<<blocks, kPlanThreads, smem, static_cast<cudaStream_t>(stream)>>>(p);
    ctx->launches += 1;
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? STWQ_OK : stwq_cuda_fail(ctx, e);
}

int qk_norm_rope(stwq_ctx* ctx, const void* QKV, int64_t ld, int x_dtype, const int32_t* pos_ids, int64_t T, int Hq, int Hkv,
                 int d, const float* w_q, int w_q_heads, const float* w_k, int w_k_heads, int norm, float eps, const float* cs,
                 int rot, int rope, int P, void* Qo, int64_t q_ts, int64_t q_hs, void* Ko, int64_t k_ts, int64_t k_hs,
                 int out_dtype, void* stream)
{
    if (!ctx || !Ko) return STWQ_ERR_NULL;
    NrParams p = {};
    const int rc = nr_common(p, QKV, ld, x_dtype, pos_ids, T, Hq, Hkv, d, w_q, w_q_heads, w_k, w_k_heads, norm, eps, cs, rot, rope, P, Qo,
                             q_ts, q_hs, out_dtype);
    if (rc != STWQ_OK) return rc;
    const int64_t elem16 = out_dtype == STWQ_OUT_F32 ? 4 : 8;
    if (!stwq_disjoint(T, Hkv, d, k_ts, k_hs)) return STWQ_ERR_DIM;
    if (!stwq_aligned16(Ko) || k_ts % elem16 != 0 || k_hs % elem16 != 0) return STWQ_ERR_ALIGN;
    p.Ko = Ko; p.k_ts = k_ts; p.k_hs = k_hs;
    p.status = ctx->d_status;
    StwqDevGuard g(ctx->device);
    return launch_nr_any(ctx, p, x_dtype == STWQ_OUT_BF16, out_dtype == STWQ_OUT_F32, 0, static_cast<cudaStream_t>(stream));
}

int kv_append_paged(stwq_ctx* ctx, const void* QKV, int64_t ld, int x_dtype, const int32_t* pos_ids, const int32_t* slot_map,
                    int64_t T, int Hq, int Hkv, int d, const float* w_q, int w_q_heads, const float* w_k, int w_k_heads, int norm,
                    float eps, const float* cs, int rot, int rope, int P, const float* s_k, const float* s_v, int bits, void* Qo,
                    int64_t q_ts, int64_t q_hs, void* Kp, void* Vp, int n_pages, int page_size, int kv_dtype, void* stream)
{
    if (!ctx || !slot_map || !Kp || !Vp) return STWQ_ERR_NULL;
    NrParams p = {};
    const int rc = nr_common(p, QKV, ld, x_dtype, pos_ids, T, Hq, Hkv, d, w_q, w_q_heads, w_k, w_k_heads, norm, eps, cs, rot, rope, P, Qo,
                             q_ts, q_hs, STWQ_OUT_BF16);
    if (rc != STWQ_OK) return rc;
    if (n_pages <= 0 || page_size <= 0) return STWQ_ERR_DIM;
    if (kv_dtype != STWQ_KV_BF16 && kv_dtype != STWQ_KV_INT8) return STWQ_ERR_BITS;
    if (kv_dtype == STWQ_KV_INT8) {
        if (!s_k || !s_v) return STWQ_ERR_NULL;
        if (bits != 8 && bits != 6) return STWQ_ERR_BITS;
        p.qmax = (1 << (bits - 1)) - 1;
        p.qmin = -(1 << (bits - 1));
        p.need_pos = 1;
    }
    if (!stwq_aligned16(Kp) || !stwq_aligned16(Vp) || !stwq_aligned16(s_v)) return STWQ_ERR_ALIGN;
    p.slots = slot_map;
    p.Kp = Kp; p.Vp = Vp; p.S = page_size; p.n_slots = (int64_t)n_pages * page_size;
    p.s_k = s_k; p.s_v = s_v;
    p.status = ctx->d_status;
    StwqDevGuard g(ctx->device);
    return launch_nr_any(ctx, p, x_dtype == STWQ_OUT_BF16, 0, kv_dtype == STWQ_KV_INT8 ? 2 : 1, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
