// Paged attention for many rows (a prefill chunk, a scale of an image pyramid): 256 query rows of one key head against
// 128 keys at a time on the tensor cores. Rows are (new token, query head of the key head), token-major, so shared
// key heads fill a tile with fewer tokens.
//     S = Q K^T (fp32 in tensor memory),  P = 2^(S c - m),  O += P V,  O / l at the end
//
//  * Two tiles of 128 rows (A, B) share every K and V tile. Each has a group of 128 threads, one per row; while one group
//    computes its probabilities the tensor core works for the other. The bound is the tensor core for d = 128 (2048 cycles
//    per 256 x 128 tile) and the ex2 unit (16 per clock: 2048 cycles) for both d = 64 and d = 128.
//  * S, P, O live in tensor memory: S_A, S_B 128 columns each, O_A, O_B d columns each. P (16-bit) is written over the S
//    columns already read and is the A operand of the second product straight from there: no trip through shared memory.
//  * K and V tiles are gathered page by page by four loader warps with cp.async into the 128-byte-swizzled layouts: K rows as
//    K-major, V rows as they are (MN-major B operand: no transpose). Codes pass through registers and become fp16.
//  * The running maximum is a reference that moves only when a row exceeds it by about 2^10 (see the few-row kernel),
//    which the sum of its exponentials shows (and a maximum over the quarter that the cubic takes): the rescale of O in tensor
//    memory is rare, and each score is read once.
//  * With fewer units than SMs the keys of a unit are cut into equal ranges; partial (m, l, O) go to workspace and the
//    last CTA adds them in key order.
//  * fp32 output: P is kept as a sum of 16-bit terms (bf16: three, fp16: two; 22 to 24 significant bits), all multiplied by V.
//    The tensor core truncates its running sums (1e-5 over 5000 keys), so the row threads add each tile's product to an
//    fp32 sum beside it. Both want tensor memory: a CTA then has one tile of rows, not two.
//  * Measured: 2 requests of 2048 tokens behind 2048, 16 heads over 4 of 128, bf16, causal: 108 us, 950 TFLOP/s, 0.57 of
//    the measured burst rate (2048 cycles of products per 256 x 128 tile, the rest waits between products and rows).
//    4 requests of 1024 to 2048 tokens behind up to 6144, 32 heads over 8: 550 us in a burst, 630 to 645 in long runs; 1777 us with
//    fp32 output. 32 requests of 256 tokens over 680 codes, 30 heads of 64: 153 us; there a unit is six tiles long, and set-up, Q
//    and O cost a third of it. Looking at what the cubic gets (its result alone hides an overflow) is 2 to 3 % of these.
//  * Where scores are far from flat the reference moves more often: the long chunks take 756 us with queries 4 times as large
//    (scores of a standard deviation of 5), 918 us with 16 times; the codes 196 us with 4 times.
// 16-bit operands: bf16 for a bf16 cache (P rounded to bf16); fp16 for codes (exact), with queries scaled per row by a
// power of two as in the few-row kernel. Sums, maxima and O in fp32.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "stwq_paged.cuh"
#include "stwq_pattn.cuh"
#include "stwq_ptx.cuh"

using namespace stwq_ptx;

namespace {

constexpr int kRowWarps = 8, kLoadWarps = 3;   // and one that issues the products: 12 warps leave a thread 168 registers
constexpr int kThreads = 32 * (kRowWarps + kLoadWarps + 1);
constexpr int kKT = 128;                     // keys per tile
constexpr int kHalf = 128 * 128;             // bytes of 128 rows of 128 bytes
constexpr int kMaxStages = 4;
constexpr int kMaxSplit = 32;
constexpr int kPolyEvery = 4;                // one pair of exponentials in so many goes through the fma pipe instead of the ex2 unit
constexpr int kTmemCols = 512, kColS = 0, kColO = 256;
constexpr int kColMore = 128, kColSum = 384; // fp32 output: further terms of P (64 columns each), the fp32 sum of O

template <int NH>
struct Smem {
    static constexpr int stages = NH == 1 ? 4 : 2;
    static constexpr int tile = NH * kHalf;              // one Q, K or V tile
    static constexpr int offQ = 0;
    static constexpr int offV = 2 * tile;
    static constexpr int offK = offV + stages * tile;
    static constexpr int offBars = offK + stages * tile;
    // Key scales, a slot of 128 per tile. The loaders write slot j once the first product of tile j - stages is done, when
    // the row threads may still be reading that tile's: stages + 1 slots are alive at once.
    static constexpr int offScale = offBars + 512;
    static constexpr int slots = 8;
    static constexpr int offPre = offScale + slots * 512;               // first unit of each request [B + 1]
    static_assert(stages + 1 <= slots, "key-scale slots");
};

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel)
{
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(sel));
    return r;
}
__device__ __forceinline__ uint64_t add_f2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool live)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t codes_half2(uint32_t w, uint32_t sel)      // w: codes ^ 0x80
{
    const uint32_t x = prmt(w, 0x64646464u, sel), k = 0x64806480u;
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&k));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// D[128 x N] (+)= A B, kind::f16, fp32 accumulators; A from shared memory or from tensor memory. The whole warp comes here
// with the same values (they then live in uniform registers) and one elected lane issues.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile("{\n\t.reg .pred p, e;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile("{\n\t.reg .pred p, e;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void commit_one(uint32_t bar)
{
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
                 "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}
// MN-major operand, 128-byte swizzle: rows (the contraction index) of 64 elements, 8-row groups 1024 bytes apart,
// the next 64 elements of a row kHalf bytes further
__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr)
{
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)(kHalf >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// D fp32, A and B bf16 (1) or fp16 (0); bmn: B is MN-major
__device__ __forceinline__ uint32_t idesc_f16(int n, bool bf16, bool bmn)
{
    const uint32_t f = bf16 ? 1u : 0u;
    return (1u << 4) | (f << 7) | (f << 10) | ((bmn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
                   "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint64_t pack_u2(uint32_t lo, uint32_t hi) { return pack_f2(__uint_as_float(lo), __uint_as_float(hi)); }
__device__ __forceinline__ void unpack_u2(uint64_t v, uint32_t& lo, uint32_t& hi)
{
    float a, b;
    unpack_f2(v, a, b);
    lo = __float_as_uint(a);
    hi = __float_as_uint(b);
}
// 2^x on a pair without the ex2 unit: x = n + r with |r| <= 1/2 (adding 1.5 2^23 rounds to the integer), a cubic for 2^r
// (least maximum relative error, 7.5e-5: below a quarter of fp16's half step), n added to the exponent. x is cut at -126 (NaN too); from
// 128 on the exponent runs over into the sign, so the caller has to look at x as well as at the result.
__device__ __forceinline__ uint64_t exp2_poly(uint64_t x2)
{
    float x0, x1;
    unpack_f2(x2, x0, x1);
    const uint64_t x = pack_f2(fmaxf(x0, -126.0f), fmaxf(x1, -126.0f));
    const uint64_t t = add_f2(x, dup_f2(12582912.0f));
    const uint64_t r = fma_f2(add_f2(t, dup_f2(-12582912.0f)), dup_f2(-1.0f), x);
    uint64_t q = fma_f2(r, dup_f2(0.05517167f), dup_f2(0.24261113f));
    q = fma_f2(q, r, dup_f2(0.69326099f));
    q = fma_f2(q, r, dup_f2(0.99992807f));
    uint32_t t0, t1, q0, q1;
    unpack_u2(t, t0, t1);
    unpack_u2(q, q0, q1);
    return pack_u2((t0 << 23) + q0, (t1 << 23) + q1);
}
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c)           // NaN if any of them is
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// The bounded wait of the GEMM kernels behind a few polls that do not read the timer.
__device__ __forceinline__ bool wait_bar(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, unsigned long long limit_ns)
{
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
        if (mbar_try_wait(bar, parity)) return true;
    return mbar_wait(bar, parity, abort_flag, limit_ns);
}
__device__ __forceinline__ void rows_barrier() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

template <bool I8>
__device__ __forceinline__ uint32_t pack_p(float a, float c) { return I8 ? pack_f16(a, c) : pack_bf16(a, c); }
template <bool I8>
__device__ __forceinline__ float2 unpack_p(uint32_t w)
{
    return I8 ? __half22float2(*reinterpret_cast<const __half2*>(&w)) : make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
// O (d columns) and the blocks of P already written for this tile, times f. Rare, so kept out of the loop's code.
template <bool I8>
__device__ __noinline__ void rescale(uint32_t to, int d, uint32_t tp, int blocks, float f)
{
    uint32_t w[16];
    tmem_st_wait();                                       // the blocks of P were stored without a wait, and are read back here
#pragma unroll 1
    for (int cb = 0; cb < d; cb += 16) {
        tmem_ld16(to + cb, w);
        tmem_ld_wait();
#pragma unroll
        for (int k = 0; k < 16; ++k) w[k] = __float_as_uint(__uint_as_float(w[k]) * f);
        tmem_st16(to + cb, w);
    }
#pragma unroll 1
    for (int pb = 0; pb < blocks; ++pb) {
        tmem_ld16(tp + 16 * pb, w);
        tmem_ld_wait();
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const float2 v = unpack_p<I8>(w[k]);
            w[k] = pack_p<I8>(v.x * f, v.y * f);
        }
        tmem_st16(tp + 16 * pb, w);
    }
    tmem_st_wait();
}

template <bool I8, int NH, bool F32>
__global__ void __launch_bounds__(kThreads, 1) pattn_tiled_kernel(const PaParams p, const int sm_count)
{
    using L = Smem<NH>;
    constexpr int NST = L::stages;
    constexpr int kX = F32 ? 1 : 2;                       // tiles of 128 rows
    constexpr int kRows = 128 * kX;
    constexpr int kUnroll = I8 || F32 ? 1 : 2;            // the loops of all roles have to stay in the instruction cache together
    constexpr int kTerms = !F32 ? 1 : (I8 ? 2 : 3);       // 16-bit terms of P
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - raw);
    const uint32_t bars = base + L::offBars;
    auto bar_q = [&](int x) { return bars + 8u * x; };
    auto bar_kfull = [&](int s) { return bars + 8u * (2 + s); };
    auto bar_kempty = [&](int s) { return bars + 8u * (2 + kMaxStages + s); };
    auto bar_vfull = [&](int s) { return bars + 8u * (2 + 2 * kMaxStages + s); };
    auto bar_vempty = [&](int s) { return bars + 8u * (2 + 3 * kMaxStages + s); };
    auto bar_s = [&](int x) { return bars + 8u * (2 + 4 * kMaxStages + x); };
    auto bar_p = [&](int x) { return bars + 8u * (4 + 4 * kMaxStages + x); };
    auto bar_o = [&](int x) { return bars + 8u * (6 + 4 * kMaxStages + x); };
    const uint32_t bar_drain = bars + 8u * (8 + 4 * kMaxStages);
    uint32_t* misc = reinterpret_cast<uint32_t*>(smem + L::offBars + 256);
    uint32_t* tmem_slot = misc;
    volatile uint32_t* abort_flag = misc + 1;
    uint32_t* sm_last = misc + 2;
    int* wsum = reinterpret_cast<int*>(misc + 8);         // [13]
    int* pre = reinterpret_cast<int*>(smem + L::offPre);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;      // warp: uniform

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");     // the few-row kernel of the same call may start where there is room
    // barriers and tensor memory, while the lengths are on their way
    if (tid == 0) {
        for (int x = 0; x < 2; ++x) {
            mbar_init(bar_q(x), 4);
            mbar_init(bar_s(x), 1);
            mbar_init(bar_p(x), 4);
            mbar_init(bar_o(x), 1);
        }
        for (int s = 0; s < NST; ++s) {
            mbar_init(bar_kfull(s), I8 ? kLoadWarps : 32 * kLoadWarps);
            mbar_init(bar_kempty(s), 1);
            mbar_init(bar_vfull(s), I8 ? kLoadWarps : 32 * kLoadWarps);
            mbar_init(bar_vempty(s), 1);
        }
        mbar_init(bar_drain, 1);
        *abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    if (warp == kRowWarps + kLoadWarps) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tc_fence_before();
    }
    // ---- units of every request: key heads x tiles of 256 rows
    bool bad = false;
    auto units_of = [&](int b) -> int {
        const PaReq q = pa_request(p, b, bad);
        const int rows = q.n * p.g;
        return rows <= p.few_max || q.n <= 0 ? 0 : p.Hkv * ((rows + kRows - 1) / kRows);
    };
    {
        const int per = (p.B + kThreads - 1) / kThreads;
        const int b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
        int sum = 0;
        for (int b = b0; b < b1; ++b) sum += units_of(b);
        const int units0 = sum;                           // of the only request, where a thread has one
        int s = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += u;
        }
        if (lane == 31) wsum[warp] = s;
        __syncthreads();
        int at = s - sum;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) at += w < warp ? wsum[w] : 0;
        for (int b = b0; b < b1; ++b) {
            pre[b] = at;
            at += per == 1 ? units0 : units_of(b);
        }
        if (tid == kThreads - 1) pre[p.B] = at;
    }
    if (bad && blockIdx.x == 0) atomicOr(p.status, STWQ_DEV_PAGES);
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    auto free_tmem = [&]() {
        if (warp == kRowWarps + kLoadWarps) {
            __syncwarp();
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
        }
    };
    const int U = pre[p.B];
    const int nS = min(max(sm_count / max(U, 1), 1), kMaxSplit);        // ranges of keys per unit
    if ((int)blockIdx.x >= U * nS) {
        free_tmem();
        return;
    }
    const int unit = nS == 1 ? (int)blockIdx.x : (int)blockIdx.x / nS, split = (int)blockIdx.x - unit * nS;
    int b = 0;
    {
        int x0 = 0, x1 = p.B;
        while (x1 - x0 > 1) {
            const int m = (x0 + x1) >> 1;
            if (pre[m] <= unit) x0 = m;
            else x1 = m;
        }
        b = x0;                                           // requests without units share their start with the next one
    }
    const PaReq q = pa_request(p, b, bad);
    const int rows = q.n * p.g;
    const int nqt = (rows + kRows - 1) / kRows;
    const int ul = unit - pre[b];
    const int qt = nqt - 1 - ul / p.Hkv, hk = ul % p.Hkv; // late rows first: under a causal mask they see the most keys
    const int row0 = qt * kRows;
    // keys that the last row of tile x sees, and tiles of keys
    auto last_limit = [&](int x) -> int {
        const int last = min(rows, row0 + 128 * (x + 1)) - 1;
        if (last < row0 + 128 * x) return 0;
        return max(0, p.causal ? q.kv - q.n + last / p.g + 1 : q.kv);
    };
    const int tiles0 = (last_limit(0) + kKT - 1) / kKT, tiles1 = kX == 1 ? 0 : (last_limit(1) + kKT - 1) / kKT;
    const int tiles = max(tiles0, tiles1);
    // Ranges of the keys: a tile takes about 3000 cycles, adding up a part about 2000, so their number goes with the root
    const int eS = min(nS, max(1, (int)sqrtf(1.5f * (float)tiles)));
    if (split >= eS) {
        free_tmem();
        return;
    }
    const int t0 = eS == 1 ? 0 : (int)((uint32_t)tiles * (uint32_t)split / (uint32_t)eS);               // tiles < 2^24, eS <= 32
    const int t1 = eS == 1 ? tiles : (int)((uint32_t)tiles * (uint32_t)(split + 1) / (uint32_t)eS);
    const int nt0 = max(0, min(tiles0, t1) - t0), nt1 = max(0, min(tiles1, t1) - t0);
    const int n = max(nt0, nt1);

    const unsigned long long limit_ns = p.wait_limit_ns;
    const int d = p.d;

    if (warp == kRowWarps + kLoadWarps) {
        // ------------------------------------------------------------------------------------ MMA issuer
        if (n > 0) {
            const uint32_t id_s = idesc_f16(kKT, !I8, false), id_o = idesc_f16(d, !I8, true);
            const int ksteps = d / 16;
            // descriptors count in 16 bytes: steps are plain additions to the low word
            const uint64_t dq = make_smem_desc(base + L::offQ), dk = make_smem_desc(base + L::offK), dv = desc_mn(base + L::offV);
            auto qk = [&](int x, int s) {
                const uint64_t a = dq + (uint32_t)(x * (L::tile >> 4)), c = dk + (uint32_t)(s * (L::tile >> 4));
                const uint32_t to = tmem + kColS + 128 * x;
                auto step = [&](int k) { const uint32_t off = (uint32_t)((k >> 2) * kHalf + (k & 3) * 32) >> 4; mma_ss(to, a + off, c + off, id_s, k > 0 ? 1u : 0u); };
                if (ksteps == NH * 4) {
#pragma unroll
                    for (int k = 0; k < NH * 4; ++k) step(k);
                } else {
#pragma unroll 1
                    for (int k = 0; k < ksteps; ++k) step(k);
                }
            };
            auto pv = [&](int x, int s, uint32_t acc) {
                const uint64_t c = dv + (uint32_t)(s * (L::tile >> 4));
                const uint32_t to = tmem + kColO + 128 * x, a = tmem + kColS + 128 * x;
#pragma unroll
                for (int k = 0; k < kKT / 16; ++k) mma_ts(to, a + 8 * k, c + k * 128, id_o, k > 0 ? 1u : acc);
#pragma unroll
                for (int e = 1; e < kTerms; ++e)
#pragma unroll
                    for (int k = 0; k < kKT / 16; ++k) mma_ts(to, tmem + kColMore + 64 * (e - 1) + 8 * k, c + k * 128, id_o, 1u);
            };
            bool ok = true;
            const int nt[2] = {nt0, nt1};
            for (int x = 0; ok && x < 2; ++x)
                if (nt[x] > 0) ok = __all_sync(0xffffffffu, wait_bar(bar_q(x), 0u, abort_flag, limit_ns));
            ok = ok && __all_sync(0xffffffffu, wait_bar(bar_kfull(0), 0u, abort_flag, limit_ns));
            if (ok) {
                tc_fence_after();
                fence_async_smem();                       // what the loaders' copies wrote, for the tensor core's reads
                for (int x = 0; x < 2; ++x)
                    if (nt[x] > 0) {
                        qk(x, 0);
                        commit_one(bar_s(x));
                    }
                commit_one(bar_kempty(0));
            }
            for (int j = 0; ok && j < n; ++j) {
                const int sv = j % NST, sk = (j + 1) % NST;
                ok = __all_sync(0xffffffffu, wait_bar(bar_vfull(sv), (uint32_t)(j / NST) & 1u, abort_flag, limit_ns));
                if (ok && j + 1 < n) ok = __all_sync(0xffffffffu, wait_bar(bar_kfull(sk), (uint32_t)((j + 1) / NST) & 1u, abort_flag, limit_ns));
                fence_async_smem();
                for (int x = 0; ok && x < 2; ++x) {
                    if (j >= nt[x]) continue;
                    ok = __all_sync(0xffffffffu, wait_bar(bar_p(x), (uint32_t)j & 1u, abort_flag, limit_ns));
                    if (!ok) break;
                    tc_fence_after();
                    pv(x, sv, !F32 && j > 0 ? 1u : 0u);
                    if (j + 1 < nt[x]) {
                        qk(x, sk);                        // over S and P, behind the product that reads P
                        commit_one(bar_s(x));
                    } else commit_one(bar_o(x));
                }
                if (ok) {
                    commit_one(bar_vempty(sv));
                    if (j + 1 < n) commit_one(bar_kempty(sk));
                }
            }
            if (!ok) {                                    // giving up: products already issued must not outlive the tensor memory
                commit_one(bar_drain);
                const unsigned long long w0 = globaltimer_ns();
                while (!mbar_try_wait(bar_drain, 0u))
                    if (globaltimer_ns() - w0 > limit_ns) break;
            }
        }
    } else if (warp >= kRowWarps) {
        // ------------------------------------------------------------------------------------ loaders
        // Warp w copies the 16-key blocks w, w + 3 and w + 6 of a tile. A block lies in one page and is contiguous there: 16 d
        // elements, taken 16 bytes per lane; the swizzled destinations inside a block are the same for every block and
        // stay in registers. Page lookups: every 8 tiles a lane finds the address of one (tile, block) pair.
        const int lw = warp - kRowWarps;
        constexpr int es = I8 ? 1 : 2;
        constexpr int kP = NH * 2 * es;                   // pieces per lane and block
        const int nb = lw < 2 ? 3 : 2;                    // blocks of a tile
        const int ppk = d * es / 16, pieces = 16 * ppk;
        const int per_page = p.S / 16;
        const int64_t row_bytes = (int64_t)d * es, page_bytes = row_bytes * p.S;
        const int32_t* trow = p.table + (int64_t)b * p.W;
        uint32_t dsto[kP];                                // destination of the lane's pieces, from the block's first row
        int keyo[kP];                                     // their key in the block
#pragma unroll
        for (int k = 0; k < kP; ++k) {
            const int x = lane + 32 * k, key = x / ppk, c = (x - key * ppk) * (I8 ? 2 : 1);
            keyo[k] = x < pieces ? key : 1 << 20;
            dsto[k] = (uint32_t)((c >> 3) * kHalf + key * 128 + (((c & 7) ^ (key & 7)) << 4));
        }
        bool ok = true;
        // byte offset in the pool of block lw + 3 (lane & 3) of tile j0 + lane / 4
        auto find_blocks = [&](int j0) -> int64_t {
            const int b16 = (t0 + j0 + (lane >> 2)) * 8 + lw + 3 * (lane & 3);
            int id = 0, off = 0;
            if (j0 + (lane >> 2) < n && (lane & 3) < nb && b16 * 16 < q.kv) {
                const int pg = b16 / per_page;
                off = b16 - pg * per_page;
                id = __ldg(trow + pg);
                if (id < 0 || id >= p.n_pages) {
                    atomicOr(p.status, STWQ_DEV_PAGES);
                    id = 0;
                }
            }
            return ((int64_t)id * p.Hkv + hk) * page_bytes + off * 16 * row_bytes;
        };
        auto wait_stage = [&](bool is_v, int j) -> bool {
            if (j < NST) return true;
            const int s = j % NST;
            return wait_bar(is_v ? bar_vempty(s) : bar_kempty(s), (uint32_t)(j / NST + 1) & 1u, abort_flag, limit_ns);
        };
        int64_t blocks = find_blocks(0), blocks_next = find_blocks(8);
        auto block_at = [&](int j, int h) -> int64_t { return __shfl_sync(0xffffffffu, blocks, 4 * (j & 7) + h); };
        auto advance = [&](int j) {                       // before the first use of tile j
            if ((j & 7) == 0 && j > 0) {
                blocks = blocks_next;
                blocks_next = find_blocks(j + 8);
            }
        };
        if (!I8) {
            for (int i = 0; i < 2 * n; ++i) {
                const int j = i >> 1;
                const bool is_v = i & 1;
                if (!is_v) advance(j);
                ok = wait_stage(is_v, j);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t dst0 = base + (is_v ? L::offV : L::offK) + (j % NST) * L::tile;
                const uint8_t* pool = reinterpret_cast<const uint8_t*>(is_v ? p.Vp : p.Kp);
#pragma unroll
                for (int h = 0; h < 3; ++h) {
                    if (h == nb) break;
                    const uint8_t* src = pool + block_at(j, h) + lane * 16;
                    const int first = (lw + 3 * h) * 16;
                    const int left = q.kv - (t0 + j) * kKT - first;       // keys of the block that exist
                    const uint32_t dst = dst0 + first * 128;
                    if (left >= 16 && pieces == 32 * kP) {
#pragma unroll
                        for (int k = 0; k < kP; ++k) cp_async16(dst + dsto[k], src + k * 512, true);
                    } else {
#pragma unroll
                        for (int k = 0; k < kP; ++k)
                            if (keyo[k] < 16) cp_async16(dst + dsto[k], keyo[k] < left ? src + k * 512 : pool, keyo[k] < left);
                    }
                }
                // the lane's arrival on the stage's barrier comes when its copies have landed
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(is_v ? bar_vfull(j % NST) : bar_kfull(j % NST)) : "memory");
            }
            asm volatile("cp.async.wait_all;" ::: "memory");       // nothing lands after the CTA has given up
        } else {
            // codes: the bytes of the next loads are on their way in registers while this one is widened (kDeep loads of
            // 8 or 16 KB per CTA cover the latency of HBM)
            constexpr int kDeep = 2;
            const bool whole = pieces == 32 * kP;         // d fills the lanes
            const int n_full = q.kv / kKT - t0;           // tiles before this one have all their keys
            uint4 buf[kDeep][3][kP];
            float sk[kDeep][2];
            auto fetch = [&](int i, uint4 (&to)[3][kP], float (&sc)[2]) {
                const int j = i >> 1;
                if (!(i & 1)) advance(j);
                const uint8_t* pool = reinterpret_cast<const uint8_t*>((i & 1) ? p.Vp : p.Kp);
#pragma unroll
                for (int h = 0; h < 3; ++h) {
                    if (h == nb) break;
                    const uint8_t* src = pool + block_at(j, h) + lane * 16;
                    if (whole && j < n_full) {
#pragma unroll
                        for (int k = 0; k < kP; ++k) to[h][k] = __ldg(reinterpret_cast<const uint4*>(src + k * 512));
                    } else {
                        const int left = min(q.kv - (t0 + j) * kKT - (lw + 3 * h) * 16, 16);
#pragma unroll
                        for (int k = 0; k < kP; ++k) {
                            to[h][k] = make_uint4(0u, 0u, 0u, 0u);
                            if (keyo[k] < left) to[h][k] = __ldg(reinterpret_cast<const uint4*>(src + k * 512));
                        }
                    }
                }
                if (!(i & 1)) {
                    const int kj = (t0 + j) * kKT + lw * 32 + lane;
                    sc[0] = kj < q.kv ? __ldg(p.s_k + kj) : 0.0f;
                    if (lw == 0) sc[1] = kj + 96 < q.kv ? __ldg(p.s_k + kj + 96) : 0.0f;
                }
            };
            auto widen = [&](const uint4& x, uint32_t at) {
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                uint32_t v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t c = w[e] ^ 0x80808080u;
                    v[2 * e] = codes_half2(c, 0x4140u);
                    v[2 * e + 1] = codes_half2(c, 0x4342u);
                }
                st_shared_v4(at, v[0], v[1], v[2], v[3]);
                st_shared_v4(at ^ 16u, v[4], v[5], v[6], v[7]);            // the neighbouring piece of the swizzled row
            };
#pragma unroll
            for (int u = 0; u < kDeep; ++u)
                if (u < 2 * n) fetch(u, buf[u], sk[u]);
            for (int i0 = 0; ok && i0 < 2 * n; i0 += kDeep) {
#pragma unroll
                for (int u = 0; u < kDeep; ++u) {
                    const int i = i0 + u, j = i >> 1;
                    const bool is_v = i & 1;
                    if (i >= 2 * n) break;
                    ok = wait_stage(is_v, j);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    const uint32_t dst0 = base + (is_v ? L::offV : L::offK) + (j % NST) * L::tile;
                    if (!is_v) {
                        float* dst = reinterpret_cast<float*>(smem + L::offScale) + (j & (L::slots - 1)) * 128 + lw * 32 + lane;
                        dst[0] = sk[u][0];
                        if (lw == 0) dst[96] = sk[u][1];
                    }
#pragma unroll
                    for (int h = 0; h < 3; ++h) {
                        if (h == nb) break;
                        const uint32_t dst = dst0 + (lw + 3 * h) * 16 * 128;
                        if (whole) {
#pragma unroll
                            for (int k = 0; k < kP; ++k) widen(buf[u][h][k], dst + dsto[k]);
                        } else {
#pragma unroll
                            for (int k = 0; k < kP; ++k)
                                if (keyo[k] < 16) widen(buf[u][h][k], dst + dsto[k]);
                        }
                    }
                    __syncwarp();                         // the proxy fence is the issuer's: here it would also wait for the loads in flight
                    if (lane == 0) mbar_arrive(is_v ? bar_vfull(j % NST) : bar_kfull(j % NST));
                    if (i + kDeep < 2 * n) fetch(i + kDeep, buf[u], sk[u]);
                }
            }
        }
    } else {
        // ------------------------------------------------------------------------------------ one thread per row
        const int x = warp >> 2;                          // tile
        const int rl = tid & 127;                         // row of the tile
        const int row = row0 + 128 * x + rl;
        const bool live = x < kX && row < rows;
        const int ti = live ? row / p.g : 0, hd = hk * p.g + (live ? row - ti * p.g : 0);
        const int nt = x == 0 ? nt0 : nt1;
        const int vis = !live ? 0 : max(0, p.causal ? q.kv - q.n + ti + 1 : q.kv);        // keys this row sees
        float inv = 1.0f;
        // the 16-byte pieces of the warp's 32 rows of d 16-bit elements, in the order of the rows: body(row, piece)
        const int ppr = d / 8;
        auto walk_rows = [&](auto&& body) {
            if (ppr == NH * 8) {
#pragma unroll
                for (int k = 0; k < NH * 8; ++k) body(lane / (NH * 8) + k * (4 / NH), lane % (NH * 8));
                return;
            }
            int rw = lane / ppr, c = lane - rw * ppr;
            const int dr = 32 / ppr, dc = 32 - dr * ppr;
            for (int k = 0; k < ppr; ++k) {               // 32 ppr pieces over 32 lanes
                body(rw, c);
                rw += dr;
                c += dc;
                if (c >= ppr) {
                    c -= ppr;
                    ++rw;
                }
            }
        };
        if (nt > 0) {
            // ---- the warp's 32 rows of Q, swizzled: lanes walk along the rows
            const int64_t qoff = live ? (int64_t)(q.t0 + ti) * p.q_ts + (int64_t)hd * p.q_hs : -1;
            const uint32_t qrow = base + L::offQ + x * L::tile + (rl & ~31) * 128;
            walk_rows([&](int rw, int c) {
                const int64_t off = __shfl_sync(0xffffffffu, qoff, rw);
                cp_async16(qrow + (c >> 3) * kHalf + rw * 128 + (((c & 7) ^ (rw & 7)) << 4),
                           reinterpret_cast<const __nv_bfloat16*>(p.Q) + max(off, (int64_t)0) + c * 8, off >= 0);
            });
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (I8) {
                // each thread turns its own row into fp16 under a power of two
                __syncwarp();
                const uint32_t mine = qrow + lane * 128;
                auto piece = [&](int c) { return mine + (c >> 3) * kHalf + (((c & 7) ^ (lane & 7)) << 4); };
                float mx = 0.0f;
                uint4 v[NH * 8];
#pragma unroll
                for (int c = 0; c < NH * 8; ++c) v[c] = c < d / 8 ? ld_shared_v4(piece(c)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int c = 0; c < NH * 8; ++c) {
                    const uint32_t w[4] = {v[c].x, v[c].y, v[c].z, v[c].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        mx = max3(mx, fabsf(__uint_as_float(w[e] << 16)), fabsf(__uint_as_float(w[e] & 0xffff0000u)));
                }
                int e = (int)(__float_as_uint(mx) >> 23) - 127;
                e = mx > 0.0f && mx < INFINITY ? max(e, -100) : 13;
                const float up = __uint_as_float((uint32_t)(13 - e + 127) << 23);
                inv = __uint_as_float((uint32_t)(e - 13 + 127) << 23);
#pragma unroll
                for (int c = 0; c < NH * 8; ++c)
                    if (c < d / 8) {
                        uint32_t w[4] = {v[c].x, v[c].y, v[c].z, v[c].w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) w[k] = pack_f16(__uint_as_float(w[k] << 16) * up, __uint_as_float(w[k] & 0xffff0000u) * up);
                        st_shared_v4(piece(c), w[0], w[1], w[2], w[3]);
                    }
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_q(x));
        }
        const float cc = p.scale * kPaLog2e * inv;        // scores in units of log2
        const uint64_t cc2 = dup_f2(cc);
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t ts = tmem + kColS + 128 * x + lanes, to = tmem + kColO + 128 * x + lanes;
        const int min_vis = __reduce_min_sync(0xffffffffu, live ? vis : 0x7fffffff);
        float m = vis > 0 ? -INFINITY : 0.0f, l = 0.0f;   // a row that sees nothing needs no reference: its sum stays next to nothing
        float m_sum = -INFINITY;                          // the reference that the fp32 sum of O stands against
        auto add_up = [&](bool more) {                     // sum = sum 2^(m_sum - m) + O
            const float f = more && m > -INFINITY ? ex2_approx(m_sum - m) : 0.0f;
            for (int cb = 0; cb < d; cb += 16) {
                uint32_t w[16], a[16];
                tmem_ld16(to + cb, w);
                if (more) tmem_ld16(tmem + kColSum + lanes + cb, a);
                tmem_ld_wait();
                if (more) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) w[k] = __float_as_uint(fmaf(__uint_as_float(a[k]), f, __uint_as_float(w[k])));
                }
                tmem_st16(tmem + kColSum + lanes + cb, w);
            }
            tmem_st_wait();
        };
        bool ok = true;
        for (int j = 0; j < nt; ++j) {
            ok = wait_bar(bar_s(x), (uint32_t)j & 1u, abort_flag, limit_ns);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const int key0 = (t0 + j) * kKT;
            const bool masked = key0 + kKT > min_vis;     // uniform over the warp
            const float4* sks = reinterpret_cast<const float4*>(smem + L::offScale) + (j & (L::slots - 1)) * 32;
            uint32_t v[2][32];                            // 64 scores at a time
            // key scales and mask on the 32 scores h of part qd
            auto scores = [&](int qd, int h) {
                if (I8) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float4 f = sks[qd * 16 + h * 8 + k];
                        unpack_u2(mul_f2(pack_u2(v[h][4 * k], v[h][4 * k + 1]), pack_f2(f.x, f.y)), v[h][4 * k], v[h][4 * k + 1]);
                        unpack_u2(mul_f2(pack_u2(v[h][4 * k + 2], v[h][4 * k + 3]), pack_f2(f.z, f.w)), v[h][4 * k + 2], v[h][4 * k + 3]);
                    }
                }
                if (masked) {
                    const int seen = vis - key0 - 64 * qd - 32 * h;
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (k >= seen) v[h][k] = 0xff800000u;             // -Inf
                }
            };
            auto maximum = [&](int h) -> float {
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int k = 0; k < 32; k += 2) mx[(k >> 1) & 3] = max3(mx[(k >> 1) & 3], __uint_as_float(v[h][k]), __uint_as_float(v[h][k + 1]));
                return fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
            };
            if (F32 && j > 0) {                           // the product of the tile before is done
                add_up(j > 1);
                m_sum = m;
            }
            float tile_max = -INFINITY;                   // fp32 output: known before the first exponential, so no term is rescaled
            if (F32) {
#pragma unroll 1
                for (int qd = 0; qd < 2; ++qd) {
                    tmem_ld32(ts + 64 * qd, v[0]);
                    tmem_ld32(ts + 64 * qd + 32, v[1]);
                    tmem_ld_wait();
                    scores(qd, 0);
                    scores(qd, 1);
                    tile_max = max3(tile_max, maximum(0), maximum(1));
                }
            }
            tmem_ld32(ts, v[0]);
            tmem_ld32(ts + 32, v[1]);
#pragma unroll(kUnroll)
            for (int qd = 0; qd < 2; ++qd) {
                tmem_ld_wait();
                scores(qd, 0);
                scores(qd, 1);
                // The exponentials are taken against the reference as it stands. Only when some row has none yet, or its sum
                // over these 64 keys shows that a score exceeded it by more than the slack, are the scores read again, the
                // reference moved to their maximum, and what was summed and written so far scaled down to it.
                bool move = F32 ? qd == 0 : __any_sync(0xffffffffu, m == -INFINITY);
                constexpr int kHeld = F32 ? 1 : 2;        // halves kept until the sum is known to be fine
                uint32_t w[kHeld][kTerms][16];
                auto store_p = [&](int h) {               // over columns whose scores have been read
                    tmem_st16(ts + 32 * qd + 16 * h, w[h % kHeld][0]);
#pragma unroll
                    for (int e = 1; e < kTerms; ++e) tmem_st16(tmem + kColMore + lanes + 64 * (e - 1) + 32 * qd + 16 * h, w[h % kHeld][e]);
                };
                float part, hi;                           // sum; largest argument of the cubic, whose result means nothing from 2^128 on
                for (int pass = 0;; ++pass) {
                    if (move) {
                        if (!F32 && pass > 0) {          // the registers hold the next scores already
                            tmem_ld_wait();
                            tmem_ld32(ts + 64 * qd, v[0]);
                            tmem_ld32(ts + 64 * qd + 32, v[1]);
                            tmem_ld_wait();
                            scores(qd, 0);
                            scores(qd, 1);
                        }
                        const float mx = cc * (F32 ? tile_max : fmaxf(maximum(0), maximum(1)));            // cc > 0
                        const float mn = fmaxf(m, mx);
                        const float f = mn == -INFINITY ? 1.0f : ex2_approx(m - mn);
                        m = mn;
                        l *= f;
                        if (!F32) rescale<I8>(to, j > 0 ? d : 0, ts, 2 * qd, f);
                    }
                    const float mm = m == -INFINITY ? 0.0f : m - (I8 ? 4.0f : 0.0f);   // fp16: four octaves up keep small probabilities' bits
                    const uint64_t negm2 = dup_f2(-mm);
                    uint64_t l2[2] = {0ull, 0ull};        // (0, 0)
                    hi = -INFINITY;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            const uint64_t e2 = fma_f2(pack_u2(v[h][2 * k], v[h][2 * k + 1]), cc2, negm2);
                            float a, c;
                            unpack_f2(e2, a, c);
                            if (!F32 && k % kPolyEvery == kPolyEvery - 1) {
                                hi = max3_nan(hi, a, c);
                                unpack_f2(exp2_poly(e2), a, c);
                            } else {
                                a = ex2_approx(a);
                                c = ex2_approx(c);
                            }
                            l2[k & 1] = add_f2(l2[k & 1], pack_f2(a, c));
#pragma unroll
                            for (int e = 0; e < kTerms; ++e) {
                                w[h % kHeld][e][k] = pack_p<I8>(a, c);
                                if (e + 1 < kTerms) {
                                    const float2 r = unpack_p<I8>(w[h % kHeld][e][k]);
                                    a -= r.x;
                                    c -= r.y;
                                }
                            }
                        }
                        if (qd == 0) tmem_ld32(ts + 64 + 32 * h, v[h]);    // the next scores into the registers just used up
                        if (F32) store_p(h);
                    }
                    float la, lb;
                    unpack_f2(add_f2(l2[0], l2[1]), la, lb);
                    part = la + lb;
                    if (F32 || pass > 0) break;
                    move = __any_sync(0xffffffffu, !(part <= (I8 ? 16.0f : 1.0f) * 1024.0f) || !(hi <= (I8 ? 14.0f : 10.0f)));
                    if (!move) break;
                }
                if (!F32 && move && hi != hi) part = hi;  // a NaN that only the cubic saw
                l += part;
                if (!F32) {
                    store_p(0);
                    store_p(1);
                }
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_p(x));
        }
        // ---- O
        if (ok && nt > 0) {
            ok = wait_bar(bar_o(x), 0u, abort_flag, limit_ns);
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
        }
        auto write16 = [&](int cb, float (&o)[16], float rl_sum) {       // 16 channels of the row
            // no visible key: zeros. The sum of a row with a score above -Inf is about 1 or more, and scores at -Inf add at most
            // 2^-126 each: a row that sees nothing else is 0 / 0
            const float inv_l = rl_sum < 5.4e-20f ? __uint_as_float(0x7fffffffu) : __fdividef(1.0f, rl_sum);
#pragma unroll
            for (int k = 0; k < 16; ++k) o[k] = vis > 0 ? o[k] * inv_l : 0.0f;
            if (I8) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float4 f = __ldg(reinterpret_cast<const float4*>(p.s_v + (int64_t)hk * d + cb) + k);
                    o[4 * k] *= f.x; o[4 * k + 1] *= f.y; o[4 * k + 2] *= f.z; o[4 * k + 3] *= f.w;
                }
            }
            const int64_t at = (int64_t)(q.t0 + ti) * p.o_ts + (int64_t)hd * p.o_hs + cb;
            if (!F32) {                                   // into the row's place in the Q tile, which no product reads any more
                const uint32_t mine = base + L::offQ + x * L::tile + rl * 128 + (cb >> 6) * kHalf;
                const int c = (cb >> 3) & 7;
                st_shared_v4(mine + ((c ^ (rl & 7)) << 4), pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]), pack_bf16(o[4], o[5]), pack_bf16(o[6], o[7]));
                st_shared_v4(mine + (((c + 1) ^ (rl & 7)) << 4), pack_bf16(o[8], o[9]), pack_bf16(o[10], o[11]), pack_bf16(o[12], o[13]),
                             pack_bf16(o[14], o[15]));
            } else {
                float4* dst = reinterpret_cast<float4*>(reinterpret_cast<float*>(p.O) + at);
#pragma unroll
                for (int k = 0; k < 4; ++k) dst[k] = make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
            }
        };
        auto store_rows = [&]() {                         // bf16 output: from there to memory, lanes walking along the rows
            if (F32) return;
            __syncwarp();
            const int64_t ooff = live ? (int64_t)(q.t0 + ti) * p.o_ts + (int64_t)hd * p.o_hs : -1;
            const uint32_t orow = base + L::offQ + x * L::tile + (rl & ~31) * 128;
            walk_rows([&](int rw, int c) {
                const int64_t off = __shfl_sync(0xffffffffu, ooff, rw);
                const uint4 v = ld_shared_v4(orow + (c >> 3) * kHalf + rw * 128 + (((c & 7) ^ (rw & 7)) << 4));
                if (off >= 0) *(reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.O) + off) + c) = v;
            });
        };
        constexpr int DP = NH * 64;
        const int64_t part_f4 = (int64_t)(DP / 4) * 256 + 128;           // float4s of a partial result: O, then (m, l)
        float4* part = reinterpret_cast<float4*>(p.part) + ((int64_t)unit * nS + split) * part_f4;
        const int pr = 128 * x + rl;
        if (ok) {
            for (int cb = 0; cb < d; cb += 16) {
                uint32_t w[16];
                float o[16];
                if (nt > 0) {
                    tmem_ld16(to + cb, w);
                    tmem_ld_wait();
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] = nt > 0 ? __uint_as_float(w[k]) : 0.0f;
                if (F32 && nt > 1) {
                    const float f = m > -INFINITY ? ex2_approx(m_sum - m) : 0.0f;
                    tmem_ld16(tmem + kColSum + lanes + cb, w);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 16; ++k) o[k] = fmaf(__uint_as_float(w[k]), f, o[k]);
                }
                if (eS == 1) {
                    if (live || !F32) write16(cb, o, l);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) __stcg(part + (cb / 4 + k) * 256 + pr, make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]));
                }
            }
            if (eS == 1) store_rows();
        }
        if (eS > 1) {
            float2* ml = reinterpret_cast<float2*>(part + (DP / 4) * 256);
            __stcg(ml + pr, make_float2(m, l));
            __threadfence();
            rows_barrier();
            if (tid == 0) {
                const uint32_t k = atomicAdd(p.counters + unit, 1u);
                *sm_last = k == (uint32_t)(eS - 1) ? 1u : 0u;
                if (*sm_last) p.counters[unit] = 0u;      // zero again for the next call
                __threadfence();
            }
            rows_barrier();
            if (*sm_last && x < kX) {
                const float4* p0 = reinterpret_cast<const float4*>(p.part) + (int64_t)unit * nS * part_f4;
                float M = -INFINITY, Ls = 0.0f;
                float* fs = reinterpret_cast<float*>(smem + L::offV);    // [eS][256]: the operand tiles are no longer needed
#pragma unroll 8
                for (int s = 0; s < eS; ++s) {
                    const float2 v = __ldcg(reinterpret_cast<const float2*>(p0 + s * part_f4 + (DP / 4) * 256) + pr);
                    M = fmaxf(M, v.x);
                }
#pragma unroll 8
                for (int s = 0; s < eS; ++s) {
                    const float2 v = __ldcg(reinterpret_cast<const float2*>(p0 + s * part_f4 + (DP / 4) * 256) + pr);
                    const float f = M == -INFINITY ? 0.0f : ex2_approx(v.x - M);
                    fs[s * 256 + pr] = f;
                    Ls = fmaf(f, v.y, Ls);
                }
                // 64 channels at a time: sixteen loads in flight per part (the latency of L2 is what this costs)
#pragma unroll 1
                for (int hb = 0; hb < d; hb += 64) {
                    float o[64];
#pragma unroll
                    for (int k = 0; k < 64; ++k) o[k] = 0.0f;
#pragma unroll 1
                    for (int s = 0; s < eS; ++s) {
                        const float f = fs[s * 256 + pr];
                        const float4* src = p0 + s * part_f4 + (hb / 4) * 256 + pr;
                        float4 v[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) v[k] = hb + 4 * k < d ? __ldcg(src + k * 256) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            o[4 * k] = fmaf(f, v[k].x, o[4 * k]);
                            o[4 * k + 1] = fmaf(f, v[k].y, o[4 * k + 1]);
                            o[4 * k + 2] = fmaf(f, v[k].z, o[4 * k + 2]);
                            o[4 * k + 3] = fmaf(f, v[k].w, o[4 * k + 3]);
                        }
                    }
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (hb + 16 * c < d && (live || !F32)) {
                            float o16[16];
#pragma unroll
                            for (int k = 0; k < 16; ++k) o16[k] = o[16 * c + k];
                            write16(hb + 16 * c, o16, Ls);
                        }
                }
                store_rows();
            }
        }
    }
    // ---- teardown
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && *abort_flag) atomicOr(p.status, STWQ_DEV_TIMEOUT);
    tc_fence_after();
    free_tmem();
}

template <bool I8, int NH, bool F32>
int launch_as(stwq_ctx* ctx, const PaParams& p, unsigned grid, cudaStream_t st)
{
    auto kern = pattn_tiled_kernel<I8, NH, F32>;
    int smem = Smem<NH>::offPre + (p.B + 1) * 4 + 1024;
    if (smem < 116 * 1024) smem = 116 * 1024;             // all of tensor memory: one CTA per SM
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024);
    if (e != cudaSuccess) return stwq_cuda_fail(ctx, e);
    kern<<<grid, kThreads, smem, st>>>(p, ctx->sm_count);
    ctx->launches += 1;
    e = cudaGetLastError();
    return e == cudaSuccess ? STWQ_OK : stwq_cuda_fail(ctx, e);
}

template <bool I8, int NH>
int launch(stwq_ctx* ctx, const PaParams& p, unsigned grid, cudaStream_t st)
{
    return p.out_bf16 ? launch_as<I8, NH, false>(ctx, p, grid, st) : launch_as<I8, NH, true>(ctx, p, grid, st);
}

}  // namespace

size_t stwq_pattn_tiled_part_bytes(const stwq_ctx* ctx, int d)
{
    const int DP = d <= 64 ? 64 : 128;
    return (size_t)ctx->sm_count * ((size_t)(DP / 4) * 256 + 128) * 16;      // only with units x ranges <= SMs
}

int stwq_launch_pattn_tiled(stwq_ctx* ctx, const PaParams& p, cudaStream_t st)
{
    // units: at most ceil(rows / unit) per request and key head, rows adding up to T g
    int64_t grid = (int64_t)p.Hkv * ((p.T * p.g + (p.out_bf16 ? 255 : 127)) / (p.out_bf16 ? 256 : 128) + p.B);
    if (grid < ctx->sm_count) grid = ctx->sm_count;
    if (grid > 0x7fffffff) return STWQ_ERR_DIM;
    const unsigned gx = (unsigned)grid;
    if (p.d <= 64) return p.s_k ? launch<true, 1>(ctx, p, gx, st) : launch<false, 1>(ctx, p, gx, st);
    return p.s_k ? launch<true, 2>(ctx, p, gx, st) : launch<false, 2>(ctx, p, gx, st);
}
