// The pass between two linears of a transformer block: residual sum, gate, norms, modulation, codes (block_norm).
//
// For a row of C channels, in fp32:
//     h' = h + r g (Npost(o) wp + bp),   y = (Npre(h') w + b) (1 + scale) + shift,
//     N: x / sqrt(mean(x^2) + eps), or (x - m) / sqrt(mean((x - m)^2) + eps) with m = mean(x), or x
//     out: y, y (1/s_ch), or the codes clamp(round((y rc) rt)), rc = 1/s_ch, rt = 1/s_tok[pos]
// Each row is read once: its 16-byte pieces are copied asynchronously into shared memory while the rows before it are worked on, and
// its channels stay in registers from there on. A mean and a sum of squares are one reduction each over the threads of the row; the
// squares are those of the centred values. Vectors of C channels (weights, gate, scale, shift) come from L1 and L2.
// Bound: HBM asks for |h| + |o| in, |h'| + |y| out. 65536 rows of 1280 (fp32 stream, bf16 branch and output) take 169 us, 6.0 TB/s, 0.91 of
// the measured copy rate; with everything in bf16 the phases of a row, one behind the other, which 16 warps of up to 128 registers on an SM hide
// in part (some 25 instructions per channel and lane, issue slots half busy): 8192 rows of 1920 30 us, 4.2 TB/s; 20000 of 1024 with two weighted norms 38 us, 4.4 TB/s.
#include <cuda_bf16.h>

#include "stwq_internal.cuh"
#include "stwq_paged.cuh"
#include "stwq_ptx.cuh"

using namespace stwq_ptx;       // packed fp32 arithmetic

namespace {

constexpr int kMaxC = 16384;
constexpr int kMaxThreads = 512;           // of one row
constexpr int kTeams = 4;                  // rows a block works on at a time, where a warp holds a row
constexpr int kMaxRows = 32;               // rows of a team in turn: a lane keeps the ids of one

struct BnParams {
    const void *H, *O, *gate, *scale, *shift;
    void *Ho, *Y;
    int64_t ldh, ldo, ldc, ldho, ldy, M;
    int C, G, P, y_dtype, post, pre, qmin, qmax, rows, depth;
    const int32_t *cond, *pos;
    const float *wp, *bp, *w, *b, *s_ch, *s_tok;
    float res_scale, eps, inv_C;
    uint32_t* status;
};

// Eight channels. Two fp32 values per instruction where there is one for it; each half rounds as the scalar instruction does.
struct F8 {
    uint64_t p[4];
    __device__ __forceinline__ void fill(float v)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = dup_f2(v);
    }
    template <bool BF>
    __device__ __forceinline__ void widen(const uint4& a, const uint4& b)
    {
        if (BF) {
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = pack_f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
        } else {
            p[0] = pack_f2(__uint_as_float(a.x), __uint_as_float(a.y));
            p[1] = pack_f2(__uint_as_float(a.z), __uint_as_float(a.w));
            p[2] = pack_f2(__uint_as_float(b.x), __uint_as_float(b.y));
            p[3] = pack_f2(__uint_as_float(b.z), __uint_as_float(b.w));
        }
    }
    template <bool BF>
    __device__ __forceinline__ void store(char* at) const
    {
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack_f2(p[i], v[2 * i], v[2 * i + 1]);
        if (BF) *reinterpret_cast<uint4*>(at) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
        else {
            reinterpret_cast<float4*>(at)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(at)[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    }
};
__device__ __forceinline__ uint64_t add_f2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
#define STWQ_EACH(v) _Pragma("unroll") for (int v = 0; v < VPT; ++v)
#define STWQ_PAIRS(i) _Pragma("unroll") for (int i = 0; i < 4; ++i)

// A warp holds VPT vectors of 256 consecutive channels of a row, a lane eight channels of each: vector v of a lane starts
// 256 v channels behind its first. on[v]: whether it lies in the row.
template <int VPT, bool BF>
struct Side {                              // of a vector of C channels that no call writes, as it lies in memory
    uint4 q[VPT][BF ? 1 : 2];
    // KEEP false: an ordinary load, which the compiler does not carry from row to row in registers (that costs more by the warps it displaces)
    template <bool KEEP>
    __device__ __forceinline__ void load(const void* lane0, const bool (&on)[VPT])
    {
        STWQ_EACH(v)
#pragma unroll
            for (int i = 0; i < (BF ? 1 : 2); ++i) {
                const uint4* src = reinterpret_cast<const uint4*>(lane0) + v * (BF ? 32 : 64) + i;
                q[v][i] = make_uint4(0u, 0u, 0u, 0u);         // left undefined it would live from row to row
                if (on[v]) {
                    if (KEEP) q[v][i] = __ldg(src);
                    else asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q[v][i].x), "=r"(q[v][i].y), "=r"(q[v][i].z), "=r"(q[v][i].w) : "l"(src) : "memory");
                }
            }
    }
    __device__ __forceinline__ F8 get(int v) const
    {
        F8 x;
        x.widen<BF>(q[v][0], q[v][BF ? 0 : 1]);
        return x;
    }
};

// A warp's part of a row in shared memory, copied 16 bytes at a time: lane l copies piece 32 i + l. bf16: a piece is a lane's
// vector; fp32: pieces 2l and 2l + 1 are, and every other four lanes' pieces change places, so that reads of eight lanes do not meet.
template <int VPT, bool BF>
struct Slot {
    static constexpr int kBytes = VPT * (BF ? 512 : 1024);       // of a warp
    // `row`: the warp's first channel; `left`: bytes from there to the end of the row
    __device__ __forceinline__ static void fetch(uint32_t slot, const char* row, int left, int lane)
    {
#pragma unroll
        for (int i = 0; i < kBytes / 512; ++i) {
            const int at = i * 512 + 16 * lane;
            const uint32_t to = slot + i * 512 + 16 * (BF ? lane : lane ^ ((lane >> 3) & 1));
            if (at < left) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(row + at) : "memory");
        }
    }
    __device__ __forceinline__ static F8 read(const char* slot, int v, int lane)
    {
        F8 x;
        const uint4* q = reinterpret_cast<const uint4*>(slot) + v * (BF ? 32 : 64);
        if (BF) {
            const uint4 a = q[lane];
            x.widen<BF>(a, a);
        } else {
            const int turned = (lane >> 2) & 1;
            x.widen<BF>(q[2 * lane + turned], q[2 * lane + 1 - turned]);
        }
        return x;
    }
};

// The sum over a row, in all its threads, added in a fixed order. The two sets of `red` are used in turn: no warp writes a set
// again before all have passed the barrier of the other.
template <bool MULTI>
__device__ __forceinline__ float row_sum(uint64_t v2, float (*red)[kMaxThreads / 32], int& turn)
{
    float a, b;
    unpack_f2(v2, a, b);
    float v = a + b;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (!MULTI) return v;
    float* set = red[turn];
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) set[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.0f;
    for (int i = 0; i < (int)(blockDim.x >> 5); i += 4) {          // sets are padded with zeros
        const float4 q = *reinterpret_cast<const float4*>(set + i);
        s += (q.x + q.y) + (q.z + q.w);
    }
    return s;
}

// x <- N(x) w + b. Channels beyond the row hold zeros before, and anything after.
template <int VPT, bool MULTI>
__device__ __forceinline__ void normalise(F8 (&x)[VPT], const bool (&on)[VPT], int kind, const float* w, const float* b, int lane0, const BnParams& p,
                                          float (*red)[kMaxThreads / 32], int& turn)
{
    if (kind == STWQ_NORM_LAYER) {
        uint64_t s = dup_f2(0.0f);
        STWQ_EACH(v) STWQ_PAIRS(i) s = add_f2(s, x[v].p[i]);
        const uint64_t m = dup_f2(-row_sum<MULTI>(s, red, turn) * p.inv_C);
        STWQ_EACH(v) if (on[v]) STWQ_PAIRS(i) x[v].p[i] = add_f2(x[v].p[i], m);
    }
    if (kind != STWQ_NORM_NONE) {
        uint64_t q = dup_f2(0.0f);
        STWQ_EACH(v) STWQ_PAIRS(i) q = fma_f2(x[v].p[i], x[v].p[i], q);
        const uint64_t r = dup_f2(rsqrtf(fmaf(row_sum<MULTI>(q, red, turn), p.inv_C, p.eps)));
        STWQ_EACH(v) STWQ_PAIRS(i) x[v].p[i] = mul_f2(x[v].p[i], r);
    }
    if (w != nullptr) {
        Side<VPT, false> f;
        f.template load<false>(w + lane0, on);
        STWQ_EACH(v) {
            const F8 a = f.get(v);
            STWQ_PAIRS(i) x[v].p[i] = mul_f2(x[v].p[i], a.p[i]);
        }
    }
    if (b != nullptr) {
        Side<VPT, false> f;
        f.template load<false>(b + lane0, on);
        STWQ_EACH(v) {
            const F8 a = f.get(v);
            STWQ_PAIRS(i) x[v].p[i] = add_f2(x[v].p[i], a.p[i]);
        }
    }
}

// A team (a warp, or with MULTI the warps of a block) goes through its rows with the next `depth` on their way into its slots
// (two, or one where two do not fit).
template <int VPT, bool MULTI, bool HB, bool OB, bool CB>
__global__ void __launch_bounds__(MULTI ? kMaxThreads : 32 * kTeams, MULTI ? (VPT == 1 ? 2 : 1) : VPT == 1 ? 8 : 4) block_norm_kernel(const BnParams p)
{
    __shared__ __align__(16) float red[2][kMaxThreads / 32];
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int teams = MULTI ? 1 : kTeams, me = MULTI ? 0 : warp;
    const int first = MULTI ? warp * (256 * VPT) : 0, lane0 = first + 8 * lane;   // first channel of the warp, of the lane
    const int slot_bytes = Slot<VPT, HB>::kBytes + (p.O != nullptr ? Slot<VPT, OB>::kBytes : 0);
    char* slots = smem + warp * p.depth * slot_bytes;
    float* rc = reinterpret_cast<float*>(smem + warps * p.depth * slot_bytes);    // [C] 1 / s_ch
    if (MULTI && threadIdx.x < 2 * (kMaxThreads / 32)) (&red[0][0])[threadIdx.x] = 0.0f;
    if (p.s_ch != nullptr)
#pragma unroll 4
        for (int i = threadIdx.x; i < p.C / 4; i += blockDim.x) {
            const float4 f = __ldg(reinterpret_cast<const float4*>(p.s_ch) + i);
            reinterpret_cast<float4*>(rc)[i] = make_float4(__frcp_rn(f.x), __frcp_rn(f.y), __frcp_rn(f.z), __frcp_rn(f.w));
        }
    bool on[VPT];
    STWQ_EACH(v) on[v] = lane0 + 256 * v < p.C;
    int turn = 0;

    // a block's rows are consecutive, its teams take them in turn; a lane keeps what goes with one row of its team: bit or lane j, row j
    const int64_t row0 = (int64_t)blockIdx.x * p.rows * teams + me, my_row = row0 + (int64_t)lane * teams;
    const bool mine = lane < p.rows && my_row < p.M, codes = p.y_dtype == STWQ_OUT_INT8;
    const int my_pos = mine && p.pos != nullptr ? p.pos[my_row] : 0;
    int my_cond = mine && p.cond != nullptr ? p.cond[my_row] : 0;
    const uint32_t live = __ballot_sync(0xffffffffu, mine && my_pos != -1);       // not behind the last row, not padding
    const uint32_t bad_g = __ballot_sync(0xffffffffu, mine && my_pos != -1 && (my_cond < 0 || my_cond >= p.G));
    const uint32_t bad_y = bad_g | __ballot_sync(0xffffffffu, mine && codes && my_pos != -1 && (my_pos < 0 || my_pos >= p.P));
    if (bad_y != 0u && lane0 == 0) atomicOr(p.status, STWQ_DEV_POS_RANGE);
    if ((bad_g >> lane) & 1u) my_cond = 0;
    const float my_rt = codes && mine && my_pos >= 0 && my_pos < p.P ? __frcp_rn(p.s_tok[my_pos]) : 1.0f;

    // running addresses: of the next row to fetch, of the row at hand
    constexpr int kH = HB ? 2 : 4, kO = OB ? 2 : 4;
    const char* h_next = reinterpret_cast<const char*>(p.H) + (row0 * p.ldh + first) * kH;
    const char* o_next = reinterpret_cast<const char*>(p.O) + (row0 * p.ldo + first) * kO;
    char* ho = reinterpret_cast<char*>(p.Ho) + (row0 * p.ldho + lane0) * kH;
    const int y_bytes = codes ? 1 : p.y_dtype == STWQ_OUT_BF16 ? 2 : 4;
    char* y = reinterpret_cast<char*>(p.Y) + (row0 * p.ldy + lane0) * y_bytes;
    const int64_t h_step = p.ldh * teams * kH, o_step = p.ldo * teams * kO, ho_step = p.ldho * teams * kH, y_step = p.ldy * teams * y_bytes;
    uint32_t to = smem_u32(slots), coming = live;                 // where the next row goes; bit 0: whether it is a live one
    const uint32_t flip = p.depth > 1 ? to ^ (to + slot_bytes) : 0u;
    auto fetch = [&]() {
        if (coming & 1u) {
            Slot<VPT, HB>::fetch(to, h_next, (p.C - first) * kH, lane);
            if (p.O != nullptr) Slot<VPT, OB>::fetch(to + Slot<VPT, HB>::kBytes, o_next, (p.C - first) * kO, lane);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        coming >>= 1;
        h_next += h_step;
        o_next += o_step;
        to ^= flip;
    };
    // what no row fills stays zero
    for (int i = lane; i < p.depth * slot_bytes / 16; i += 32) reinterpret_cast<uint4*>(slots)[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncwarp();
    fetch();
    if (p.depth > 1) fetch();
    if (MULTI || p.s_ch != nullptr) __syncthreads();

    const char* slot = slots;
    const int slot_step = p.depth > 1 ? slot_bytes : 0;
#pragma unroll 1
    for (int j = 0; j < 32 && (live >> j) != 0u; ++j, ho += ho_step, y += y_step) {
        const char* here = slot + (j & 1) * slot_step;
        if (!((live >> j) & 1u)) {                                // the same in all threads of the team
            fetch();
            continue;
        }
        const int64_t side = (__shfl_sync(0xffffffffu, my_cond, j) * p.ldc + lane0) * (CB ? 2 : 4);
        Side<VPT, CB> gate;
        if (p.gate != nullptr) gate.template load<true>(reinterpret_cast<const char*>(p.gate) + side, on);
        if (p.depth > 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();                                             // the pieces that other lanes copied
        F8 h[VPT];
        STWQ_EACH(v) h[v] = Slot<VPT, HB>::read(here, v, lane);
        if (p.O != nullptr) {
            F8 o[VPT];
            STWQ_EACH(v) o[v] = Slot<VPT, OB>::read(here + Slot<VPT, HB>::kBytes, v, lane);
            normalise<VPT, MULTI>(o, on, p.post, p.wp, p.bp, lane0, p, red, turn);
            const uint64_t f = dup_f2(p.res_scale);
            if (p.gate != nullptr)
                STWQ_EACH(v)
                {
                    const F8 g = gate.get(v);
                    STWQ_PAIRS(i) o[v].p[i] = mul_f2(o[v].p[i], g.p[i]);
                }
            if (!((bad_g >> j) & 1u)) STWQ_EACH(v) if (on[v]) STWQ_PAIRS(i) h[v].p[i] = fma_f2(f, o[v].p[i], h[v].p[i]);
            if (p.Ho != nullptr) STWQ_EACH(v) if (on[v]) h[v].template store<HB>(ho + v * 256 * kH);
        }
        __syncwarp();                                             // all lanes have read the slot
        fetch();
        if (p.Y == nullptr) continue;
        Side<VPT, CB> scale, shift;
        if (p.scale != nullptr) scale.template load<true>(reinterpret_cast<const char*>(p.scale) + side, on);
        if (p.shift != nullptr) shift.template load<true>(reinterpret_cast<const char*>(p.shift) + side, on);
        normalise<VPT, MULTI>(h, on, p.pre, p.w, p.b, lane0, p, red, turn);
        if (p.scale != nullptr) {
            const uint64_t one = dup_f2(1.0f);
            STWQ_EACH(v)
            {
                const F8 a = scale.get(v);
                STWQ_PAIRS(i) h[v].p[i] = mul_f2(h[v].p[i], add_f2(a.p[i], one));
            }
        }
        if (p.shift != nullptr)
            STWQ_EACH(v)
            {
                const F8 a = shift.get(v);
                STWQ_PAIRS(i) h[v].p[i] = add_f2(h[v].p[i], a.p[i]);
            }
        if (p.s_ch != nullptr)
            STWQ_EACH(v) if (on[v])
            {
                const uint4* q = reinterpret_cast<const uint4*>(rc + lane0 + 256 * v);
                F8 a;
                a.widen<false>(q[0], q[1]);
                STWQ_PAIRS(i) h[v].p[i] = mul_f2(h[v].p[i], a.p[i]);
            }
        if ((bad_y >> j) & 1u) STWQ_EACH(v) h[v].fill(0.0f);
        if (codes) {
            const uint64_t rt = dup_f2(__shfl_sync(0xffffffffu, my_rt, j));
            STWQ_EACH(v) if (on[v])
            {
                uint32_t w[2] = {0u, 0u};
                STWQ_PAIRS(i)
                {
                    float u0, u1;
                    unpack_f2(mul_f2(h[v].p[i], rt), u0, u1);
                    w[i >> 1] |= ((uint32_t)(stwq_code(u0, p.qmin, p.qmax) & 0xFF) | (uint32_t)(stwq_code(u1, p.qmin, p.qmax) & 0xFF) << 8) << (16 * (i & 1));
                }
                *reinterpret_cast<uint2*>(y + 256 * v) = make_uint2(w[0], w[1]);
            }
        } else if (y_bytes == 2) STWQ_EACH(v) { if (on[v]) h[v].template store<true>(y + 512 * v); }
        else STWQ_EACH(v) { if (on[v]) h[v].template store<false>(y + 1024 * v); }
    }
}

template <int VPT, bool MULTI, bool HB, bool OB, bool CB>
int launch_bn(stwq_ctx* ctx, BnParams& p, int threads, cudaStream_t st)
{
    const int teams = MULTI ? 1 : kTeams, block = MULTI ? threads : 32 * kTeams;
    const int slot = (block / 32) * (Slot<VPT, HB>::kBytes + (p.O != nullptr ? Slot<VPT, OB>::kBytes : 0));
    const size_t side = p.s_ch != nullptr ? (size_t)p.C * 4 : 0;
    p.depth = (size_t)2 * slot + side <= 220 * 1024 ? 2 : 1;
    const size_t smem = (size_t)p.depth * slot + side;
    auto kern = block_norm_kernel<VPT, MULTI, HB, OB, CB>;
    cudaError_t e = cudaSuccess;
    if (smem > 40 * 1024) e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024);
    if (e != cudaSuccess) return stwq_cuda_fail(ctx, e);
    // Rows per team: whole waves of the blocks that fit an SM, by shared memory and registers (64 or up to 128 a thread)
    int64_t fit = (int64_t)(200 * 1024 / (smem + 1024));
    const int threads_fit = VPT == 1 ? 1024 : 512;
    if (fit > threads_fit / block) fit = threads_fit / block;
    if (fit < 1) fit = 1;
    const int64_t slots = fit * ctx->sm_count * teams, waves = (p.M + slots * kMaxRows - 1) / (slots * kMaxRows);
    p.rows = (int)((p.M + slots * waves - 1) / (slots * waves));
    const int64_t blocks = (p.M + (int64_t)p.rows * teams - 1) / ((int64_t)p.rows * teams);
    kern<<<(unsigned)blocks, block, smem, st>>>(p);
    ctx->launches += 1;
    e = cudaGetLastError();
    return e == cudaSuccess ? STWQ_OK : stwq_cuda_fail(ctx, e);
}

// Vectors per thread: with few rows one (a row is done soonest); else two or three, whichever leaves fewer lanes without channels, three
// where they are equal (8192 rows of 1920: 29 us with 2, 31 with 3, 37 with 4; 65536 of 1280: 189, 169, 169); four where 16 warps need them.
template <bool HB, bool OB, bool CB>
int launch_bn_any(stwq_ctx* ctx, BnParams& p, cudaStream_t st)
{
    const int warps = (p.C / 8 + 31) / 32;                // with one vector per thread
    if (warps == 1) return launch_bn<1, false, HB, OB, CB>(ctx, p, 32, st);
    if (p.M <= 2 * ctx->sm_count && warps <= kMaxThreads / 32) return launch_bn<1, true, HB, OB, CB>(ctx, p, 32 * warps, st);
    if (warps == 2) return launch_bn<2, false, HB, OB, CB>(ctx, p, 32, st);
    if (warps == 3) return launch_bn<3, false, HB, OB, CB>(ctx, p, 32, st);
    const int t2 = (warps + 1) / 2, t3 = (warps + 2) / 3;
    if (t2 <= kMaxThreads / 32 && 2 * t2 < 3 * t3) return launch_bn<2, true, HB, OB, CB>(ctx, p, 32 * t2, st);
    if (t3 <= kMaxThreads / 32) return launch_bn<3, true, HB, OB, CB>(ctx, p, 32 * t3, st);
    return launch_bn<4, true, HB, OB, CB>(ctx, p, 32 * ((warps + 3) / 4), st);
}

// A matrix of rows: M rows of `width` bytes, `pitch` bytes apart.
struct Rows {
    const char* at;
    int64_t width, pitch;
};
// Whether two of them share a byte (rows of one pitch may lie side by side in one buffer).
bool share(const Rows& a, const Rows& b, int64_t M)
{
    if (a.at == nullptr || b.at == nullptr) return false;
    const char *ea = a.at + (M - 1) * a.pitch + a.width, *eb = b.at + (M - 1) * b.pitch + b.width;
    if (ea <= b.at || eb <= a.at) return false;
    if (a.pitch != b.pitch || M == 1) return true;
    int64_t d = (b.at - a.at) % a.pitch;
    if (d < 0) d += a.pitch;
    return d < a.width || d + b.width > a.pitch;
}
bool same(const Rows& a, const Rows& b, int64_t M) { return a.at == b.at && a.width == b.width && (a.pitch == b.pitch || M == 1); }

}  // namespace

extern "C" int block_norm(stwq_ctx* ctx, const void* H, int64_t ldh, int h_dtype, const void* O, int64_t ldo, int o_dtype, int64_t M,
                          int C, const int32_t* cond_ids, int G, const void* gate, const void* scale, const void* shift, int64_t ldc,
                          int c_dtype, int post_norm, const float* w_post, const float* b_post, float res_scale, int pre_norm,
                          const float* w_pre, const float* b_pre, float eps, void* Hout, int64_t ldho, const int32_t* pos_ids,
                          const float* s_ch, const float* s_tok, int P, int bits, void* Y, int64_t ldy, int y_dtype, void* stream)
{
    if (!ctx || !H || (!Hout && !Y) || (Hout && !O)) return STWQ_ERR_NULL;
    if (M <= 0 || M > 0x7fffffff || C <= 0 || C > kMaxC) return STWQ_ERR_DIM;
    auto real = [](int t) { return t == STWQ_OUT_F32 || t == STWQ_OUT_BF16; };
    auto kind = [](int n) { return n == STWQ_NORM_NONE || n == STWQ_NORM_RMS || n == STWQ_NORM_LAYER; };
    const bool cond = gate || scale || shift;
    if (!real(h_dtype) || (O && !real(o_dtype)) || (cond && !real(c_dtype)) || !kind(post_norm) || !kind(pre_norm)) return STWQ_ERR_BITS;
    if (Y && !real(y_dtype) && y_dtype != STWQ_OUT_INT8) return STWQ_ERR_BITS;
    if (!(eps >= 0.0f) || (cond && G <= 0)) return STWQ_ERR_DIM;
    const bool codes = Y && y_dtype == STWQ_OUT_INT8;
    if (codes) {
        if (!pos_ids || !s_tok) return STWQ_ERR_NULL;
        if (bits != 8 && bits != 6) return STWQ_ERR_BITS;
        if (P <= 0) return STWQ_ERR_DIM;
    }
    const int eh = h_dtype == STWQ_OUT_F32 ? 4 : 2, eo = o_dtype == STWQ_OUT_F32 ? 4 : 2, ec = c_dtype == STWQ_OUT_F32 ? 4 : 2;
    const int ey = codes ? 1 : (y_dtype == STWQ_OUT_F32 ? 4 : 2);
    if (ldh < C || (O && ldo < C) || (Hout && ldho < C) || (Y && ldy < C) || (cond && G > 1 && ldc < C)) return STWQ_ERR_DIM;
    if (ldh > (1ll << 40) || (O && ldo > (1ll << 40)) || (Hout && ldho > (1ll << 40)) || (Y && ldy > (1ll << 40))) return STWQ_ERR_DIM;
    if ((C & 7) != 0 || ldh * eh % 16 != 0 || (O && ldo * eo % 16 != 0) || (Hout && ldho * eh % 16 != 0) ||
        (Y && ldy * ey % (codes ? 8 : 16) != 0) || (cond && G > 1 && ldc * ec % 16 != 0))
        return STWQ_ERR_ALIGN;
    const void* ptrs[] = {H, O, gate, scale, shift, w_post, b_post, w_pre, b_pre, Hout, s_ch, codes ? nullptr : Y};
    for (const void* q : ptrs)
        if (!stwq_aligned16(q)) return STWQ_ERR_ALIGN;
    if (codes && (reinterpret_cast<uintptr_t>(Y) & 7u) != 0) return STWQ_ERR_ALIGN;
    // outputs may replace a row operand exactly, thread by thread; any other overlap would be read by one row after another wrote it
    auto rows = [](const void* q, int64_t width, int64_t pitch) { return Rows{static_cast<const char*>(q), width, pitch}; };
    const Rows rh = rows(H, (int64_t)C * eh, ldh * eh), ro = rows(O, (int64_t)C * eo, ldo * eo), rho = rows(Hout, (int64_t)C * eh, ldho * eh),
               ry = rows(Y, (int64_t)C * ey, ldy * ey);
    if ((share(rho, rh, M) && !same(rho, rh, M)) || share(rho, ro, M) || share(rho, ry, M) || (share(ry, rh, M) && !same(ry, rh, M)) ||
        (share(ry, ro, M) && !same(ry, ro, M)))
        return STWQ_ERR_ALIGN;

    BnParams p = {};
    p.H = H; p.O = O; p.gate = O ? gate : nullptr; p.scale = scale; p.shift = shift; p.Ho = Hout; p.Y = Y;
    p.ldh = ldh; p.ldo = ldo; p.ldc = cond ? ldc : 0; p.ldho = ldho; p.ldy = ldy; p.M = M;
    p.C = C; p.G = cond ? G : 1; p.P = P;
    p.y_dtype = Y ? y_dtype : STWQ_OUT_F32;
    p.post = post_norm; p.pre = pre_norm;
    p.qmax = (1 << (bits == 6 ? 5 : 7)) - 1;
    p.qmin = -p.qmax - 1;
    p.cond = cond ? cond_ids : nullptr; p.pos = pos_ids;
    p.wp = w_post; p.bp = b_post; p.w = w_pre; p.b = b_pre; p.s_ch = s_ch; p.s_tok = s_tok;
    p.res_scale = res_scale; p.eps = eps; p.inv_C = 1.0f / (float)C;
    p.status = ctx->d_status;
    StwqDevGuard dev(ctx->device);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool hb = h_dtype == STWQ_OUT_BF16, ob = !O || o_dtype == STWQ_OUT_BF16, cb = !cond || c_dtype == STWQ_OUT_BF16;
    switch (4 * hb + 2 * ob + cb) {
        case 0: return launch_bn_any<false, false, false>(ctx, p, st);
        case 1: return launch_bn_any<false, false, true>(ctx, p, st);
        case 2: return launch_bn_any<false, true, false>(ctx, p, st);
        case 3: return launch_bn_any<false, true, true>(ctx, p, st);
        case 4: return launch_bn_any<true, false, false>(ctx, p, st);
        case 5: return launch_bn_any<true, false, true>(ctx, p, st);
        case 6: return launch_bn_any<true, true, false>(ctx, p, st);
        default: return launch_bn_any<true, true, true>(ctx, p, st);
    }
}
