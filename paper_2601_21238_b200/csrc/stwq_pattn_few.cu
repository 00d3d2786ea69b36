// Paged attention for few rows (a decode step, a few speculative tokens): at most 16 query rows per key head and request,
// rows being the new tokens times the query heads that share the key head.
//     S[j, r] = scale * k_j . q_r,   O[r] = sum_j softmax_j(S[., r]) v_j,   j below the row's visible length
// Reads the request's keys and values once and is bound by that: HBM bytes, 0.5 to 16 flops per byte.
//
//  * Split: all (request, key head) units are laid end to end as 64-key blocks and cut into equal contiguous ranges, one
//    per CTA, whatever the lengths. A CTA has at most two units that it shares with neighbours; their partial
//    (max, sum, O) go to workspace and the last CTA to arrive adds them up in the order of the keys (so the result does
//    not depend on who was last).
//  * A warp takes 16 keys at a time, whole: S^T = K Q^T by mma m16n8k16 with the KEYS as the 16 rows and up to 8 query
//    rows as columns, then O^T = V^T P^T with 16 CHANNELS as rows. The channel order inside the first product and the key
//    and channel order inside the second are free, and are chosen so that every operand register pair comes out of
//    16 consecutive bytes of a key or value row. P^T is the transpose of the S^T fragment: one movmatrix per 8 keys.
//  * Loads: 16 keys of a page are contiguous, so a warp's block is two bulk copies into a ring that only this warp reads:
//    one lane issues them, a barrier per stage counts their bytes, and nothing in the loop waits for another warp. The ring is
//    up to 64 KB per CTA. Ranges are cut for three CTAs per SM (four over codes), which fit with up to 5 rows per key head at
//    128 channels (3 over codes) and few requests: the exchange buffer takes 2 KB per row and the prefix sums 8 bytes per
//    request; beyond that two or three of them are resident and the rest runs behind (64 requests of up to 4096 keys, 4 key heads
//    of 128, bf16: 69 us with 4 query heads per key head, 87 us with 8). fp32 output is cut for two. The form for 9 to 16 rows at
//    128 channels with bf16 output spills 128 (codes) to 180 bytes a thread. The rows stay as they lie: bank conflicts of 2 and 4 ways cost less
//    than HBM takes for the bytes. Copies of 16 bytes per thread into a conflict-free layout moved 4.2 TB/s where
//    these move 5.7 (16 requests of up to 32768 keys, 8 key heads of 128, bf16: 233 us, 0.87 of the measured copy rate).
//    Over codes the conversion's instructions come in beside HBM: 256 requests of 256 keys, 16 heads, 70 us, 3.9 TB/s.
//  * The running maximum is a reference, not the maximum: it moves only when a score exceeds it by more than 2^10 (a vote
//    per block instead of six shuffles). fp32 sums; P in bf16, or in fp16 over the code cache.
//  * fp32 output: P goes in as a sum of 16-bit terms (bf16: three, fp16: two; 22 to 24 significant bits), and each block's
//    product is added to O by fp32 instructions: the tensor core truncates its running sums, which over thousands of keys
//    would show in an fp32 result (1e-5 over 5000 keys). For bf16 output P is one term, an error like that of the store.
//  * Codes (int8) become fp16, exactly: byte ^ 0x80 under the exponent of 1024, minus 1152. Queries are scaled by a power of
//    two per row so that their largest lies in [2^13, 2^14): bf16 -> fp16 is then exact down to 2^-37 of that
//    largest. Key scales multiply S (fp32), value scales multiply O at the end.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "stwq_paged.cuh"
#include "stwq_pattn.cuh"
#include "stwq_ptx.cuh"

using namespace stwq_ptx;

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kBlk = 16 * kWarps;            // keys per CTA block: 16 per warp
constexpr int kMaxParts = 64;                // CTAs that share one unit
constexpr float kSlack = 10.0f;              // log2: how far a score may exceed the running reference

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel)
{
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(sel));
    return r;
}
__device__ __forceinline__ float ex2(float x) { return ex2_approx(x); }
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
// two codes (already ^ 0x80) at bytes lo, hi of w -> half2, exact
__device__ __forceinline__ uint32_t codes_half2(uint32_t w, uint32_t sel)
{
    const uint32_t x = prmt(w, 0x64646464u, sel), k = 0x64806480u;
    __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&k));
    return *reinterpret_cast<uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
template <bool F16>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    if (F16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&b);
}

template <bool I8, int DP>
struct Ring {
    static constexpr int es = I8 ? 1 : 2;
    static constexpr int npk = DP * es / 64;              // 16-byte key pieces per thread and key (4 threads share a key)
    static constexpr int vbytes = DP * es / 8;            // value bytes per thread and key (8 threads share a key)
    static constexpr int half = 16 * DP * es;             // bytes of 16 key rows, or value rows, at most
    static constexpr int stage = 2 * half;                // per warp and 16 keys
    static constexpr int stages = DP * es >= 256 ? 2 : (DP * es >= 128 ? (I8 ? 3 : 4) : 6);
    static constexpr int ctas(int nr) { return I8 && nr == 1 ? 4 : 3; }   // per SM: codes take more instructions a byte
    static constexpr int ring = kWarps * stages * stage;
    static constexpr int bars = ring;                     // one barrier per warp and stage
    static constexpr int smem = bars + 256;
};

template <bool F16>
__device__ __forceinline__ float2 unpack2(uint32_t w)
{
    if (F16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

template <bool I8, int DP, int NR, bool F32>
__global__ void __launch_bounds__(kThreads, F32 ? 2 : Ring<I8, DP>::ctas(NR)) pattn_few_kernel(const PaParams p, const int min_blocks, const int ex_rows)
{
    using R = Ring<I8, DP>;
    constexpr int NT = DP / 16;                           // channel tiles of O^T
    constexpr int NK = DP / 16;                           // steps of S^T
    extern __shared__ __align__(16) uint8_t smem[];
    // after the ring: the exchange buffer, then the first block of each request
    long long* pre = reinterpret_cast<long long*>(smem + R::smem + kWarps * ex_rows * DP * 4);        // [B + 1]
    __shared__ long long wsum[kWarps];
    __shared__ int wbig[kWarps];
    __shared__ float sm_m[kWarps][8 * NR], sm_l[kWarps][8 * NR];
    __shared__ uint32_t sm_last, sm_abort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int r = lane >> 2, t = lane & 3;
    bool bad = false;
    const uint32_t bars = (uint32_t)__cvta_generic_to_shared(smem) + R::bars + warp * R::stages * 8;
    if (lane == 0) {
        for (int s = 0; s < R::stages; ++s) mbar_init(bars + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    if (tid == 0) sm_abort = 0u;
    __syncwarp();

    // ---- the blocks of every request, end to end
    auto blocks_of = [&](const PaReq& q) -> long long {   // a request with rows but no keys still writes zeros
        if (q.n <= 0 || (int64_t)q.n * p.g > 8 * NR) return 0;
        return (long long)p.Hkv * max(1, (q.kv + kBlk - 1) / kBlk);
    };
    {
        const int per = (p.B + kThreads - 1) / kThreads;
        const int b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
        long long sum = 0;
        int big = 0;                                      // blocks of the largest unit
        for (int b = b0; b < b1; ++b) {
            const PaReq q = pa_request(p, b, bad);
            const long long n = blocks_of(q);
            sum += n;
            if (n > 0) big = max(big, max(1, (q.kv + kBlk - 1) / kBlk));
        }
        big = __reduce_max_sync(0xffffffffu, big);
        if (lane == 0) wbig[warp] = big;
        long long s = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += u;
        }
        if (lane == 31) wsum[warp] = s;
        __syncthreads();
        long long at = s - sum;
        for (int w = 0; w < warp; ++w) at += wsum[w];
        for (int b = b0; b < b1; ++b) {
            pre[b] = at;
            at += blocks_of(pa_request(p, b, bad));
        }
        if (tid == kThreads - 1) pre[p.B] = at;
        __syncthreads();
    }
    if (bad && blockIdx.x == 0) atomicOr(p.status, STWQ_DEV_PAGES);
    const long long N = pre[p.B];
    // Behind the tiled kernel this one is launched as its programmatic dependent and shares nothing with it; it only must
    // not complete before it, so that what follows in the stream finds both done.
    auto after_tiled = []() { asm volatile("griddepcontrol.wait;" ::: "memory"); };
    if (N == 0) {
        after_tiled();
        return;
    }
    // Ranges of at least min_blocks: a range costs a set-up and, when it splits a unit, a trip through workspace. And so long
    // that no unit is split over more than kMaxParts of them.
    long long G = max(1ll, min((long long)gridDim.x, (N + min_blocks - 1) / min_blocks));
    {
        int big = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) big = max(big, wbig[w]);
        G = min(G, max(1ll, (long long)((double)N / (double)big * (kMaxParts - 2))));
    }
    if (blockIdx.x >= G) {
        after_tiled();
        return;
    }
    auto share = [&](long long c) -> long long {          // N c / G
        return N <= (1 << 21) ? (long long)((uint32_t)N * (uint32_t)c / (uint32_t)G) : N * c / G;
    };
    auto request_at = [&](long long at) -> int {          // last b with pre[b] <= at
        int x0 = 0, x1 = p.B;
        while (x1 - x0 > 1) {
            const int m = (x0 + x1) >> 1;
            if (pre[m] <= at) x0 = m;
            else x1 = m;
        }
        return x0;
    };
    // A border inside a unit that is small against the ranges moves to the unit's start: no workspace trip for it. One
    // within two blocks of a unit's end or start moves there, unless that is more than half a range: a range that holds the
    // end of one unit and the start of another pays two exchanges and two trips, one after the other (8 requests of up to
    // 1024 keys: 12 of 348 ranges took 6 to 10 us where the others took 2.5).
    const long long len = N <= (1 << 21) ? (long long)(((uint32_t)N + (uint32_t)G - 1u) / (uint32_t)G) : (N + G - 1) / G;
    const int up = (int)min(2ll, len / 2), down = (int)min(2ll, (len - 1) / 2);
    auto border = [&](long long at, int& b) -> long long {
        if (at >= N) return N;
        b = request_at(at);
        const int nb = (int)((pre[b + 1] - pre[b]) / p.Hkv);
        const long long in = at - pre[b];
        const long long u0 = (in < 0x7fffffff ? (long long)((int)in / nb) : in / nb) * nb;
        if ((long long)nb * 6 * G <= N || in - u0 <= down) return pre[b] + u0;
        return u0 + nb - in <= up ? pre[b] + u0 + nb : at;
    };
    int b = 0, b_end = 0;
    const long long hi = border(share(blockIdx.x + 1), b_end), lo = border(share(blockIdx.x), b);
    if (lo >= hi) {
        after_tiled();
        return;
    }

    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * R::stages * R::stage;
    const int d = p.d, S = p.S, per_page = S / 16;
    const int64_t row_bytes = (int64_t)d * R::es;

    uint32_t used = 0;                                    // blocks this warp has taken: stage and parity run on over the units
    // A segment: the blocks blk0 .. blk1 of the unit (request, key head), and this warp's 16-key blocks first + 4 i of them.
    struct Seg {
        PaReq q;
        int b, hk, nb, blk0, blk1, first, n16;
        long long unit0;
    };
    auto locate = [&](long long at, int b) -> Seg {
        Seg s;
        while (pre[b + 1] <= at) ++b;
        bool dummy = false;
        s.b = b;
        s.q = pa_request(p, b, dummy);
        s.nb = max(1, (s.q.kv + kBlk - 1) / kBlk);
        const long long in = at - pre[b];
        s.hk = in < 0x7fffffff ? (int)in / s.nb : (int)(in / s.nb);
        s.unit0 = pre[b] + (long long)s.hk * s.nb;
        s.blk0 = (int)(at - s.unit0);
        s.blk1 = (int)min((long long)s.nb, hi - s.unit0);
        s.first = s.blk0 * kWarps + warp;
        const int end16 = min(s.blk1 * kWarps, (s.q.kv + 15) / 16);
        s.n16 = s.first < end16 ? (end16 - s.first + kWarps - 1) / kWarps : 0;
        return s;
    };
    // where the segment's block it0 + lane lies in the pools, in blocks of 16 keys (at least 256 bytes: fits 32 bits)
    auto load_ids = [&](const Seg& s, int it0) -> uint32_t {
        const int it = it0 + lane;
        if (it >= s.n16) return 0u;
        const int b16 = s.first + kWarps * it, page = b16 / per_page;
        int id = __ldg(p.table + (int64_t)s.b * p.W + page);
        if (id < 0 || id >= p.n_pages) {
            atomicOr(p.status, STWQ_DEV_PAGES);
            id = 0;
        }
        return ((uint32_t)id * (uint32_t)p.Hkv + (uint32_t)s.hk) * (uint32_t)per_page + (uint32_t)(b16 - page * per_page);
    };
    const uint32_t blk_bytes = (uint32_t)(16 * row_bytes);
    uint32_t ids = 0, ids_next = 0;                       // of the segment being loaded: its blocks 0 .. 31, 32 .. 63, and so on
    auto issue = [&](const Seg& sg, int it) {             // the whole warp; the stage has been read
        if (it >= sg.n16) return;
        if ((it & 31) == 0 && it > 0) {
            ids = ids_next;
            ids_next = load_ids(sg, it + 32);
        }
        const uint32_t at16 = __shfl_sync(0xffffffffu, ids, it & 31);
        if (lane == 0) {
            const int s = (used + it) % R::stages;
            const uint64_t base = (uint64_t)at16 * blk_bytes;
            const uint32_t dst = ring + s * R::stage;
            mbar_expect_tx(bars + 8 * s, 2 * blk_bytes);
            bulk_load(dst, reinterpret_cast<const uint8_t*>(p.Kp) + base, blk_bytes, bars + 8 * s);
            bulk_load(dst + R::half, reinterpret_cast<const uint8_t*>(p.Vp) + base, blk_bytes, bars + 8 * s);
        }
    };

    // ---- queries: B operand, row r (and r + 8), this thread's channels
    uint32_t qf[NR][NK][2];
    float qscale[NR][2];                                  // for rows 2t, 2t + 1: softmax scale, log2(e), inverse power of two
    auto load_q = [&](const Seg& sg) {
        const PaReq& q = sg.q;
        const int rows = q.n * p.g, hk = sg.hk;
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            const int row = nr * 8 + r;
            const bool live = row < rows;
            const int ti = live ? row / p.g : 0;
            const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(p.Q) + (int64_t)(q.t0 + ti) * p.q_ts +
                                       (int64_t)(hk * p.g + (live ? row - ti * p.g : 0)) * p.q_hs;
            float inv = 1.0f;
            if (!I8) {
#pragma unroll
                for (int j = 0; j < R::npk; ++j) {
                    const int ch = (t + 4 * j) * 8;
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (live && ch < d) v = __ldg(reinterpret_cast<const uint4*>(src + ch));
                    qf[nr][2 * j][0] = v.x;
                    qf[nr][2 * j][1] = v.y;
                    qf[nr][2 * j + 1][0] = v.z;
                    qf[nr][2 * j + 1][1] = v.w;
                }
            } else {
                uint32_t raw[R::npk][8];
                float mx = 0.0f;
#pragma unroll
                for (int j = 0; j < R::npk; ++j) {
                    const int ch = (t + 4 * j) * 16;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint4 v = make_uint4(0u, 0u, 0u, 0u);
                        if (live && ch < d) v = __ldg(reinterpret_cast<const uint4*>(src + ch) + h);
                        raw[j][4 * h] = v.x; raw[j][4 * h + 1] = v.y; raw[j][4 * h + 2] = v.z; raw[j][4 * h + 3] = v.w;
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        mx = fmaxf(mx, fmaxf(fabsf(__uint_as_float(raw[j][k] << 16)), fabsf(__uint_as_float(raw[j][k] & 0xffff0000u))));
                }
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                // 2^(13 - e), e the exponent of the row's largest; both powers stay normal numbers
                int e = (int)(__float_as_uint(mx) >> 23) - 127;
                e = mx > 0.0f && mx < INFINITY ? max(e, -100) : 13;
                const float up = __uint_as_float((uint32_t)(13 - e + 127) << 23);
                inv = __uint_as_float((uint32_t)(e - 13 + 127) << 23);
#pragma unroll
                for (int j = 0; j < R::npk; ++j)
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        qf[nr][4 * j + k / 2][k & 1] = pack2<true>(__uint_as_float(raw[j][k] << 16) * up, __uint_as_float(raw[j][k] & 0xffff0000u) * up);
            }
#pragma unroll
            for (int e2 = 0; e2 < 2; ++e2) qscale[nr][e2] = p.scale * kPaLog2e * __shfl_sync(0xffffffffu, inv, (2 * t + e2) * 4);
        }
    };

    Seg cur = locate(lo, b);
    ids = load_ids(cur, 0);
    ids_next = load_ids(cur, 32);
#pragma unroll
    for (int s = 0; s < R::stages; ++s) issue(cur, s);
    load_q(cur);
    for (;;) {
        const PaReq q = cur.q;
        const int hk = cur.hk, nb = cur.nb, blk0 = cur.blk0, blk1 = cur.blk1, first = cur.first, n16 = cur.n16;
        const long long unit0 = cur.unit0;
        const int rows = q.n * p.g;
        // the segment after this one: its page ids are on their way while this one is worked on
        const bool more = unit0 + blk1 < hi;
        Seg nxt = cur;
        uint32_t nxt_ids = 0, nxt_ids2 = 0;
        if (more) {
            nxt = locate(unit0 + blk1, cur.b);
            nxt_ids = load_ids(nxt, 0);
            nxt_ids2 = load_ids(nxt, 32);
        }
        int limit[NR][2];                                 // visible keys of rows 2t, 2t + 1
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int e2 = 0; e2 < 2; ++e2) {
                const int rr = nr * 8 + 2 * t + e2;
                limit[nr][e2] = rr >= rows ? 0 : (p.causal ? q.kv - q.n + rr / p.g + 1 : q.kv);
            }
        const int min_limit = p.causal ? q.kv - q.n + 1 : q.kv;           // the shortest row that exists

        float o[NR][NT][4];
        float m[NR][2], l[NR][2];
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[nr][i][k] = 0.0f;
            m[nr][0] = m[nr][1] = -INFINITY;
            l[nr][0] = l[nr][1] = 0.0f;
        }

        bool ok = true;
        const int rb = (int)row_bytes;
        int it = 0;
        for (; it < n16; ++it) {
            const int sg = (used + it) % R::stages;
            float ska = 1.0f, skb = 1.0f;
            if (I8) {
                const int j = (first + kWarps * it) * 16 + r;
                ska = __ldg(p.s_k + min(j, p.P - 1));
                skb = __ldg(p.s_k + min(j + 8, p.P - 1));
            }
            ok = __all_sync(0xffffffffu, mbar_wait(bars + 8 * sg, (uint32_t)((used + it) / R::stages) & 1u, &sm_abort, p.wait_limit_ns));
            if (!ok) break;
            const uint32_t st = ring + sg * R::stage;
            const uint32_t krow = st + r * rb + t * 16, vrow = st + R::half + 2 * t * rb;
            if ((first + kWarps * it) * 16 + 16 > q.kv) {
                // the last keys' block: value rows beyond them may hold anything, and 0 * Inf is not 0
                for (int x = lane; x < 16 * rb / 16; x += 32)
                    if ((first + kWarps * it) * 16 + x * 16 / rb >= q.kv) st_shared_v4(st + R::half + x * 16, 0u, 0u, 0u, 0u);
                fence_async_smem();                       // ordinary stores, before the bulk copy that refills the stage
                __syncwarp();
            }
            const int j0 = (first + kWarps * it) * 16;
            // ---- S^T: keys r, r + 8 x rows 2t, 2t + 1
            float s[NR][4];
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) s[nr][0] = s[nr][1] = s[nr][2] = s[nr][3] = 0.0f;
#pragma unroll
            for (int j = 0; j < R::npk; ++j) {
                uint4 ka = lds16(krow + j * 64), kb = lds16(krow + 8 * rb + j * 64);
                if ((t + 4 * j) * 16 >= rb) ka = kb = make_uint4(0u, 0u, 0u, 0u);        // beyond the row
                if (!I8) {
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr) {
                        mma<false>(s[nr], ka.x, kb.x, ka.y, kb.y, qf[nr][2 * j][0], qf[nr][2 * j][1]);
                        mma<false>(s[nr], ka.z, kb.z, ka.w, kb.w, qf[nr][2 * j + 1][0], qf[nr][2 * j + 1][1]);
                    }
                } else {
                    const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t xa = wa[k] ^ 0x80808080u, xb = wb[k] ^ 0x80808080u;
                        const uint32_t a0 = codes_half2(xa, 0x4140u), a2 = codes_half2(xa, 0x4342u);
                        const uint32_t a1 = codes_half2(xb, 0x4140u), a3 = codes_half2(xb, 0x4342u);
#pragma unroll
                        for (int nr = 0; nr < NR; ++nr) mma<true>(s[nr], a0, a1, a2, a3, qf[nr][4 * j + k][0], qf[nr][4 * j + k][1]);
                    }
                }
            }
            const bool masked = j0 + 16 > min_limit;      // uniform
            bool over = false;
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    s[nr][e] *= qscale[nr][e] * ska;
                    s[nr][2 + e] *= qscale[nr][e] * skb;
                    if (masked) {
                        if (j0 + r >= limit[nr][e]) s[nr][e] = -INFINITY;
                        if (j0 + 8 + r >= limit[nr][e]) s[nr][2 + e] = -INFINITY;
                    }
                    over |= fmaxf(s[nr][e], s[nr][2 + e]) > m[nr][e] + kSlack;
                }
            }
            if (__any_sync(0xffffffffu, over)) {          // the reference moves to the maximum so far
#pragma unroll
                for (int nr = 0; nr < NR; ++nr)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = fmaxf(s[nr][e], s[nr][2 + e]);
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                        const float mn = fmaxf(m[nr][e], mx);
                        const float f = mn == -INFINITY ? 1.0f : ex2(m[nr][e] - mn);
                        m[nr][e] = mn;
                        l[nr][e] *= f;
#pragma unroll
                        for (int i = 0; i < NT; ++i) {
                            o[nr][i][e] *= f;
                            o[nr][i][2 + e] *= f;
                        }
                    }
            }
            constexpr int kTerms = !F32 ? 1 : (I8 ? 2 : 3);
            uint32_t pf[kTerms][NR][2];                   // P^T fragments: the value, then what rounding it left over
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
                float pv[4];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    // over the code cache P is fp16: four octaves up, so that small probabilities keep their bits
                    const float mm = m[nr][e] == -INFINITY ? 0.0f : m[nr][e] - (I8 ? 4.0f : 0.0f);
                    pv[e] = ex2(s[nr][e] - mm);
                    pv[2 + e] = ex2(s[nr][2 + e] - mm);
                    l[nr][e] += pv[e] + pv[2 + e];
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float a = pv[2 * e], c = pv[2 * e + 1];
#pragma unroll
                    for (int k = 0; k < kTerms; ++k) {
                        const uint32_t h = pack2<I8>(a, c);
                        pf[k][nr][e] = transpose8x8(h);
                        const float2 v = unpack2<I8>(h);
                        a -= v.x;
                        c -= v.y;
                    }
                }
            }
            auto pv_mma = [&](int nr, int i, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
                if (F32) {
                    float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int k = kTerms - 1; k >= 0; --k) mma<I8>(c, a0, a1, a2, a3, pf[k][nr][0], pf[k][nr][1]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[nr][i][k] += c[k];
                } else mma<I8>(o[nr][i], a0, a1, a2, a3, pf[0][nr][0], pf[0][nr][1]);
            };
            // ---- O^T += V^T P^T
            if (!I8) {
#pragma unroll
                for (int hh = 0; hh < (R::vbytes >= 16 ? R::vbytes / 16 : 1); ++hh) {
                    uint4 v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = lds16(vrow + ((k & 1) + 8 * (k >> 1)) * rb + hh * 128 + r * 16);
                    const uint32_t w[4][4] = {{v[0].x, v[0].y, v[0].z, v[0].w}, {v[1].x, v[1].y, v[1].z, v[1].w},
                                              {v[2].x, v[2].y, v[2].z, v[2].w}, {v[3].x, v[3].y, v[3].z, v[3].w}};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t a0 = prmt(w[0][i], w[1][i], 0x5410u), a1 = prmt(w[0][i], w[1][i], 0x7632u);
                        const uint32_t a2 = prmt(w[2][i], w[3][i], 0x5410u), a3 = prmt(w[2][i], w[3][i], 0x7632u);
#pragma unroll
                        for (int nr = 0; nr < NR; ++nr) pv_mma(nr, hh * 4 + i, a0, a1, a2, a3);
                    }
                }
            } else {
                constexpr int nw = R::vbytes / 4;
                uint32_t w[4][nw];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (nw == 4) {
                        const uint4 v = lds16(vrow + ((k & 1) + 8 * (k >> 1)) * rb + r * 16);
                        w[k][0] = v.x; w[k][1] = v.y; w[k][nw > 2 ? 2 : 0] = v.z; w[k][nw > 2 ? 3 : 1] = v.w;
                    } else {
                        const uint2 v = lds8(vrow + ((k & 1) + 8 * (k >> 1)) * rb + r * 8);
                        w[k][0] = v.x; w[k][1] = v.y;
                    }
#pragma unroll
                    for (int i = 0; i < nw; ++i) w[k][i] ^= 0x80808080u;
                }
#pragma unroll
                for (int i = 0; i < nw; ++i) {
                    // bytes of channels 0, 1 (2, 3) of two keys side by side
                    const uint32_t x01 = prmt(w[0][i], w[1][i], 0x5140u), y01 = prmt(w[0][i], w[1][i], 0x7362u);
                    const uint32_t x23 = prmt(w[2][i], w[3][i], 0x5140u), y23 = prmt(w[2][i], w[3][i], 0x7362u);
                    const uint32_t a0 = codes_half2(x01, 0x4140u), a1 = codes_half2(x01, 0x4342u);
                    const uint32_t a2 = codes_half2(x23, 0x4140u), a3 = codes_half2(x23, 0x4342u);
                    const uint32_t c0 = codes_half2(y01, 0x4140u), c1 = codes_half2(y01, 0x4342u);
                    const uint32_t c2 = codes_half2(y23, 0x4140u), c3 = codes_half2(y23, 0x4342u);
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr) {
                        pv_mma(nr, 2 * i, a0, a1, a2, a3);
                        pv_mma(nr, 2 * i + 1, c0, c1, c2, c3);
                    }
                }
            }
            __syncwarp();                                 // the stage's bytes are in registers: refill it
            issue(cur, it + R::stages);
        }
        if (!ok && lane == 0) {                           // gave up: let the copies in flight land before their buffer goes
            const unsigned long long w0 = globaltimer_ns();
            for (int k = it; k < min(n16, it + R::stages); ++k)
                while (!mbar_try_wait(bars + 8 * ((used + k) % R::stages), (uint32_t)((used + k) / R::stages) & 1u))
                    if (globaltimer_ns() - w0 > p.wait_limit_ns) break;
        }
        used += n16;
        if (more) {                                       // the next segment's blocks and queries come in during the exchange
            ids = nxt_ids;
            ids_next = nxt_ids2;
#pragma unroll
            for (int s = 0; s < R::stages; ++s) issue(nxt, s);
            load_q(nxt);
        }

        // ---- the four warps' parts
        float* ex = reinterpret_cast<float*>(smem + R::smem);             // [kWarps][ex_rows][DP]
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float s = l[nr][e];
                s += __shfl_xor_sync(0xffffffffu, s, 4);
                s += __shfl_xor_sync(0xffffffffu, s, 8);
                s += __shfl_xor_sync(0xffffffffu, s, 16);
                const int row = nr * 8 + 2 * t + e;
                if (r == 0) {
                    sm_m[warp][row] = m[nr][e];
                    sm_l[warp][row] = s;
                }
                if (row < rows) {
                    float* dst = ex + (warp * ex_rows + row) * DP;
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        const int ch = I8 ? r * (DP / 8) + 2 * i : (i >> 2) * 64 + r * 8 + (i & 3) * 2;
                        *reinterpret_cast<float2*>(dst + ch) = make_float2(o[nr][i][e], o[nr][i][2 + e]);
                    }
                }
            }
        __syncthreads();
        const bool whole = blk0 == 0 && blk1 == nb;
        const int slots = 8 * NR * (DP + 2);              // floats of a partial result: O, then (max, sum) per row
        float* part = p.part + ((int64_t)blockIdx.x * 2 + (blk0 == 0 ? 1 : 0)) * slots;
        auto write_out = [&](int row, int ch, float a, float b2, float lsum) {       // two channels of a row
            const int ti = row / p.g;
            const bool sees = (p.causal ? q.kv - q.n + ti + 1 : q.kv) > 0;           // no visible key: zeros
            const float inv = __fdividef(1.0f, lsum);                                // all scores at -Inf: 0 / 0
            a = sees ? a * inv : 0.0f;
            b2 = sees ? b2 * inv : 0.0f;
            if (I8) {
                const float2 sv = *reinterpret_cast<const float2*>(p.s_v + (int64_t)hk * d + ch);
                a *= sv.x;
                b2 *= sv.y;
            }
            const int64_t at_o = (int64_t)(q.t0 + ti) * p.o_ts + (int64_t)(hk * p.g + row - ti * p.g) * p.o_hs + ch;
            if (!F32) *reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(p.O) + at_o) = pack2<false>(a, b2);
            else *reinterpret_cast<float2*>(reinterpret_cast<float*>(p.O) + at_o) = make_float2(a, b2);
        };
        for (int x = tid; x < rows * (DP / 2); x += kThreads) {
            const int row = x / (DP / 2), ch = (x - row * (DP / 2)) * 2;
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm_m[w][row]);
            float a = 0.0f, b2 = 0.0f, L = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = M == -INFINITY ? 0.0f : ex2(sm_m[w][row] - M);
                const float2 v = *reinterpret_cast<const float2*>(ex + (w * ex_rows + row) * DP + ch);
                a = fmaf(f, v.x, a);
                b2 = fmaf(f, v.y, b2);
                L = fmaf(f, sm_l[w][row], L);
            }
            if (whole) {
                if (ch < d) write_out(row, ch, a, b2, L);
            } else {
                __stcg(reinterpret_cast<float2*>(part + row * DP + ch), make_float2(a, b2));
                if (ch == 0) __stcg(reinterpret_cast<float2*>(part + 8 * NR * DP + 2 * row), make_float2(M, L));
            }
        }
        if (!whole) {
            // the last CTA whose share begins at block L or before it; with the borders that moved, the unit's CTAs are those
            // from the last that begins no more than `down` blocks into it to the last that begins more than `up` before its end
            auto holder = [&](long long L) -> long long {
                return N <= (1 << 21) ? (long long)(((uint32_t)(L + 1) * (uint32_t)G - 1u) / (uint32_t)N) : ((L + 1) * G - 1) / N;
            };
            const int c0 = (int)holder(unit0 + down), np = (int)holder(unit0 + nb - 1 - up) - c0 + 1;
            __threadfence();
            __syncthreads();
            uint32_t* cnt = p.counters + ((int64_t)cur.b * p.Hkv + hk);
            if (tid == 0) {
                const uint32_t n = atomicAdd(cnt, 1u);
                sm_last = n == (uint32_t)(np - 1) ? 1u : 0u;
                if (sm_last) *cnt = 0u;                   // zero again for the next call
                __threadfence();
            }
            __syncthreads();
            if (sm_last) {
                auto part_of = [&](int c) { return p.part + ((int64_t)(c0 + c) * 2 + (c == 0 ? 1 : 0)) * slots; };
                float2* pm = reinterpret_cast<float2*>(ex);               // [np][rows]: (max, sum), then (factor, sum); np <= kMaxParts
                static_assert(kMaxParts * 8 <= kWarps * DP * 4, "fits the exchange buffer for any number of rows");
                for (int x = tid; x < np * rows; x += kThreads) {
                    const int c = x / rows;
                    pm[x] = __ldcg(reinterpret_cast<const float2*>(part_of(c) + 8 * NR * DP + 2 * (x - c * rows)));
                }
                __syncthreads();
                if (tid < rows) {
                    float M = -INFINITY, L = 0.0f;
                    for (int c = 0; c < np; ++c) M = fmaxf(M, pm[c * rows + tid].x);
                    for (int c = 0; c < np; ++c) {
                        const float2 v = pm[c * rows + tid];
                        const float f = M == -INFINITY ? 0.0f : ex2(v.x - M);
                        L = fmaf(f, v.y, L);
                        pm[c * rows + tid].x = f;
                    }
                    sm_l[0][tid] = L;
                }
                __syncthreads();
                for (int x = tid; x < rows * (DP / 2); x += kThreads) {
                    const int row = x / (DP / 2), ch = (x - row * (DP / 2)) * 2;
                    if (ch >= d) continue;
                    float a = 0.0f, b2 = 0.0f;
#pragma unroll 8
                    for (int c = 0; c < np; ++c) {
                        const float2 v = __ldcg(reinterpret_cast<const float2*>(part_of(c) + row * DP + ch));
                        const float f = pm[c * rows + row].x;
                        a = fmaf(f, v.x, a);
                        b2 = fmaf(f, v.y, b2);
                    }
                    write_out(row, ch, a, b2, sm_l[0][row]);
                }
            }
        }
        if (!more) break;
        __syncthreads();                                  // the exchange buffer has been read
        cur = nxt;
    }
    // a wait that ran out leaves wrong values behind, but the units' counters as they have to be
    if (tid == 0 && sm_abort != 0u) atomicOr(p.status, STWQ_DEV_TIMEOUT);
    after_tiled();
}

template <bool I8, int DP, int NR, bool F32>
int launch_as(stwq_ctx* ctx, const PaParams& p, bool dependent, cudaStream_t st)
{
    auto kern = pattn_few_kernel<I8, DP, NR, F32>;
    const int ex_rows = (int)std::min<int64_t>((int64_t)p.max_new * p.g, 8 * NR);
    const int smem = Ring<I8, DP>::smem + kWarps * ex_rows * DP * 4 + (p.B + 1) * 8;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem > 48 * 1024 ? 140 * 1024 : 48 * 1024);
    if (e != cudaSuccess) return stwq_cuda_fail(ctx, e);
    int64_t grid = (int64_t)ctx->sm_count * (F32 ? 2 : Ring<I8, DP>::ctas(NR));
    if (grid > (int64_t)p.B * p.Hkv * kMaxParts) grid = (int64_t)p.B * p.Hkv * kMaxParts;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = dependent ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, kern, p, 2, ex_rows);
    ctx->launches += 1;
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? STWQ_OK : stwq_cuda_fail(ctx, e);
}

template <bool I8, int DP, int NR>
int launch(stwq_ctx* ctx, const PaParams& p, bool dependent, cudaStream_t st)
{
    return p.out_bf16 ? launch_as<I8, DP, NR, false>(ctx, p, dependent, st) : launch_as<I8, DP, NR, true>(ctx, p, dependent, st);
}

}  // namespace

size_t stwq_pattn_few_part_bytes(const stwq_ctx* ctx, int B, int Hkv, int d)
{
    (void)B; (void)Hkv;
    const int DP = d <= 64 ? 64 : 128;
    return (size_t)ctx->sm_count * 4 * 2 * 16 * (DP + 2) * 4;
}

int stwq_launch_pattn_few(stwq_ctx* ctx, const PaParams& p, bool dependent, cudaStream_t st)
{
    const bool i8 = p.s_k != nullptr;
    const bool two = (int64_t)p.max_new * p.g > 8;
    if (p.d <= 64) {
        if (i8) return two ? launch<true, 64, 2>(ctx, p, dependent, st) : launch<true, 64, 1>(ctx, p, dependent, st);
        return two ? launch<false, 64, 2>(ctx, p, dependent, st) : launch<false, 64, 1>(ctx, p, dependent, st);
    }
    if (i8) return two ? launch<true, 128, 2>(ctx, p, dependent, st) : launch<true, 128, 1>(ctx, p, dependent, st);
    return two ? launch<false, 128, 2>(ctx, p, dependent, st) : launch<false, 128, 1>(ctx, p, dependent, st);
}
