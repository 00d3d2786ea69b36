// Few-row products with 4-bit weights and a scale per group of input channels (linear_w4g), and the fold that makes
// the weights (gps_fold_group4).
//
//     Y[m,n] = act(sum_g s[n,g] sum_{k in g} X[m,k] c[n,k] + bias[n])
//
// HBM asks for N K / 2 bytes of codes, read once. The codes are the A operand (16 rows of n) of mma.sync m16n8k16, the activations the
// B operand (8 tokens): up to 8 rows of X cost what one costs. tcgen05 would need the codes widened into shared memory first; here a
// word of eight codes becomes four bf16 pairs in registers by a shift, a mask and one subtraction each (0x3e00 | (nibble ^ 8) is 2^-3 +
// (code + 8) 2^-10 as bf16; less 2^-3 + 2^-7 it is code 2^-10, exactly). The 2^-10 keeps 128 codes times the largest activation
// inside fp32; it leaves the result at the end (bits below 2^-126 are lost).
// A second kernel, further down, takes more rows than a tile or two of eight, and fp32 ones from four on where it is sooner done.
// A chunk is 128 input channels: 64 bytes of codes of each row, copied asynchronously into a ring of stages that every warp has for
// itself, with the chunk's activations beside them. The order in which channels meet in a product does not matter as long as both
// operands keep it. Where a group is a multiple of 128 channels, a lane takes 16 bytes of a row (32 channels), the chunk's products
// share a scale, and the chunk's fp32 sum is scaled once. Finer groups (a multiple of 32): the four lanes of a row take the four words
// of one group's 16 bytes together, two products per group, and the sum of each group is scaled.
// fp32 activations enter as three bf16 parts, cut off bit by bit (8 + 8 + 8 bits: exact), the smallest first.
// The warps of a block take different chunks of the same output channels, or different channels; the sums of those that split K meet
// in shared memory and are added in warp order. Where they fit, the activations of a block lie in shared memory as operands from the
// start: the cutting and pairing is done once, not once per tile.
// What bounds it: with many output channels three things of similar length that 16 warps of up to 128 registers do not hide behind each
// other: the copies, the widening on a half-rate pipe, the products (some 320 instructions per 2 KB of codes, issue slots 0.55 busy): 4 x 4096 > 128000, groups of 128, 75 us, 3.6 TB/s, 0.56 of the measured copy rate
// (65 us from L2 alone, 65 without the widening or without the products). Few channels: launch, first bytes, the exchange: 1 x 2048 >
// 8192 6.6 us, 8 x 8192 > 2048 in groups of 64 8.3 us. fp32 activations take three products: 13 x 1920 > 5760 in groups of 32 10.2 us.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <cstdint>

#include "stwq_internal.cuh"
#include "stwq_paged.cuh"
#include "stwq_ptx.cuh"

namespace cg = cooperative_groups;
using namespace stwq_ptx;       // activations of the epilogue

namespace {

constexpr int kMaxRows = 64;               // of X
constexpr int kMaxWarps = 16;

// ------------------------------------------------------------------------------------------ fold
// One warp per group: abs-max, scale, codes.
template <typename ST>
__global__ void __launch_bounds__(256) fold_group4_kernel(const float* __restrict__ W, int64_t groups, int K, const float* __restrict__ s_ch,
                                                          int group, uint8_t* __restrict__ Wp, ST* __restrict__ s_g)
{
    const int lane = threadIdx.x & 31, per_row = K / group;
    for (int64_t gi = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); gi < groups; gi += (int64_t)gridDim.x * 8) {
        const int64_t n = gi / per_row;
        const int k0 = (int)(gi - n * per_row) * group;
        const float2* w = reinterpret_cast<const float2*>(W + n * K + k0);
        const float2* c = reinterpret_cast<const float2*>(s_ch + k0);
        float a = 0.0f;
        for (int i = lane; i < group / 2; i += 32) {
            const float2 v = w[i], f = s_ch ? c[i] : make_float2(1.0f, 1.0f);
            a = fmaxf(a, fmaxf(fabsf(__fmul_rn(v.x, f.x)), fabsf(__fmul_rn(v.y, f.y))));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
        const ST s = static_cast<ST>(stwq_delta(a, 4));
        const float d = static_cast<float>(s);
        if (lane == 0) s_g[gi] = s;
        for (int i = lane; i < group / 2; i += 32) {
            const float2 v = w[i], f = s_ch ? c[i] : make_float2(1.0f, 1.0f);
            const int lo = stwq_code(__fdiv_rn(__fmul_rn(v.x, f.x), d), -8, 7), hi = stwq_code(__fdiv_rn(__fmul_rn(v.y, f.y), d), -8, 7);
            Wp[(n * K + k0) / 2 + i] = (uint8_t)((lo & 15) | ((hi & 15) << 4));
        }
    }
}

// ------------------------------------------------------------------------------------------ products
struct W4Params {
    const void* X;
    int64_t ldx;
    int M, K, N, per_row, chunks, tiles, stages;
    int side_log;                           // warps that hold different output channels of a tile, as a power of two; the others split K
    uint32_t group32, magic;                // 32-channel units per group, and ceil(2^32 / that): i / group32 = umulhi(i, magic) for i < 2^12
    const uint8_t* Wp;
    const void* s_g;
    int s_bf;
    const float* bias;
    int act, y_bf;
    void* Y;
};

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the first product of a sum
__device__ __forceinline__ void mma_bf16_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
// Nibbles q and q + 4 of a word as a pair of bf16: the codes times 2^-10.
__device__ __forceinline__ uint32_t codes2(uint32_t w, int q)
{
    uint32_t t;                                           // (w & mask) ^ bias in one operation
    asm("lop3.b32 %0, %1, %2, %3, 0x6a;" : "=r"(t) : "r"(w >> (4 * q)), "r"(0x000f000fu), "r"(0x3e083e08u));
    const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&t), __float2bfloat162_rn(0.1328125f));
    return *reinterpret_cast<const uint32_t*>(&v);
}
// The activations as the other linears have them. z Phi(z) of an infinite z: Inf, and -Inf * 0 = NaN.
__device__ __forceinline__ float activate(float z, int act)
{
    if (act == STWQ_ACT_NONE) return z;
    if (act == STWQ_ACT_GELU_ERF) return fabsf(z) == INFINITY ? z * (z > 0.0f ? 1.0f : 0.0f) : apply_act<STWQ_ACT_GELU_ERF>(z);
    return act == STWQ_ACT_GELU_TANH ? apply_act<STWQ_ACT_GELU_TANH>(z) : apply_act<STWQ_ACT_GELU_FAST>(z);
}
// 16 bytes into shared memory; zeros where `in` is false
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool in)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint4 lds128(const char* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// A warp's stage: 16 RT rows of 64 bytes of codes, 8 MT rows of 128 activations. 16-byte pieces change places within a row so that
// the lanes of a read do not meet in a bank (`row`: of the codes or of the activations; `p`: piece).
template <bool FINE>
__device__ __forceinline__ int code_piece(int row, int p) { return FINE ? p ^ ((row >> 1) & 3) : p; }
template <bool XF, bool FINE>
__device__ __forceinline__ int x_piece(int row, int p)
{
    if (FINE) return XF ? p ^ (row & 1) : p ^ ((row & 1) << 2);
    return XF ? p ^ (((p >> 3) & 3) | ((row & 1) << 2)) : p ^ (((p >> 3) & 1) | ((row & 1) << 1));
}
template <int RT, int MT, bool XF, bool RES>
struct Stage {
    static constexpr int kCodes = RT * 1024, kRow = XF ? 512 : 256, kBytes = kCodes + (RES ? 0 : MT * 8 * kRow);
};

// Where a lane's copies of codes come from: 16-byte piece t of rows g, g + 8, ... of a tile of 16 RT output channels. Rows behind the
// last output channel repeat it.
template <int RT>
struct CodeFeed {
    const uint8_t* row[RT * 2];
    int tile, chunk, slot;
    __device__ __forceinline__ CodeFeed() : slot(0) {}
    __device__ __forceinline__ void enter(const W4Params& p, int to_tile, int side, int first, int g, int t)
    {
        tile = to_tile;
        chunk = first;
#pragma unroll
        for (int i = 0; i < RT * 2; ++i) {
            const int n = min(((to_tile << p.side_log) + side) * (RT * 16) + i * 8 + g, p.N - 1);
            row[i] = p.Wp + (int64_t)n * (p.K >> 1) + t * 16;
        }
    }
    template <bool FINE>
    __device__ __forceinline__ void copy(const W4Params& p, uint32_t to, int g, int t) const
    {
        const bool in = chunk * 128 + t * 32 < p.K;      // else zeros; the address stays inside the row
        const int at = in ? chunk * 64 : -16 * t;
#pragma unroll
        for (int i = 0; i < RT * 2; ++i) copy16(to + (uint32_t)((i * 8 + g) * 64 + code_piece<FINE>(i * 8 + g, t) * 16), row[i] + at, in);
    }
};
// The same for the activations: piece q of rows r, r + kStep, ... of the tokens at hand.
template <int MT, bool XF, bool FINE>
struct XFeed {
    static constexpr int kRow = XF ? 512 : 256, kPieces = kRow / 16, kPer = XF ? 4 : 8, kStep = 32 / kPieces, kSize = XF ? 4 : 2;
    const char* base;                                     // of row r
    int64_t step;
    int r, q;
    __device__ __forceinline__ void enter(const W4Params& p, int m0, int lane)
    {
        r = lane / kPieces;
        q = lane % kPieces;
        step = p.ldx * (kStep * kSize);
        base = reinterpret_cast<const char*>(p.X) + (m0 + r) * p.ldx * kSize;
    }
    __device__ __forceinline__ void copy(const W4Params& p, uint32_t to, int chunk, int rows) const
    {
        const int k = chunk * 128 + q * kPer;
        const bool in = k < p.K;
        const char* src = base + (in ? k * kSize : 0);
#pragma unroll
        for (int i = 0; i < MT * 8 / kStep; ++i) {
            const int row = i * kStep + r;
            if (row < rows) copy16(to + (uint32_t)(row * kRow + x_piece<XF, FINE>(row, q) * 16), src + i * step, in);
        }
    }
};
// Scales of a chunk. FINE: a lane loads those of its 32 channels for its 2 RT rows. Else the four lanes of a row have the same ones, and
// lane t loads those of row t of the 2 RT.
template <int RT, bool FINE>
struct Scales {
    static constexpr int kN = FINE ? 2 * RT : 1;
    const char* row[kN];
    int tile, chunk;
    __device__ __forceinline__ void enter(const W4Params& p, int to_tile, int side, int first, int g, int t)
    {
        tile = min(to_tile, p.tiles - 1);                 // beyond the last one nothing uses what is loaded
        chunk = min(first, p.chunks - 1);
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int n = min(((tile << p.side_log) + side) * (RT * 16) + (FINE ? i : t % (2 * RT)) * 8 + g, p.N - 1);
            row[i] = reinterpret_cast<const char*>(p.s_g) + (((int64_t)n * p.per_row) << (p.s_bf ? 1 : 2));
        }
    }
    // the scales of the chunk at hand, and on to this warp's next
    __device__ __forceinline__ void load(const W4Params& p, int side, int first, int step, int g, int t, float (&s)[kN])
    {
        const int unit = min(chunk * 4 + (FINE ? t : 0), p.K / 32 - 1), gi = p.group32 == 1u ? unit : (int)__umulhi((uint32_t)unit, p.magic);
        if (p.s_bf) {
#pragma unroll
            for (int i = 0; i < kN; ++i) s[i] = __uint_as_float((uint32_t)__ldg(reinterpret_cast<const unsigned short*>(row[i]) + gi) << 16);
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i) s[i] = __ldg(reinterpret_cast<const float*>(row[i]) + gi);
        }
        chunk += step;
        if (chunk >= p.chunks) enter(p, tile + (int)gridDim.x, side, first, g, t);
    }
    // of row half h of tile r and (FINE) group i of the chunk
    __device__ __forceinline__ static float get(const float (&s)[kN], int r, int h, int i, int lane)
    {
        return __shfl_sync(0xffffffffu, s[FINE ? 2 * r + h : 0], (lane & ~3) | (FINE ? i : 2 * r + h));
    }
};

// Eight activations as B operands of two products: pairs of channels (0,4), (1,5), (2,6), (3,7); fp32 ones as three such sets, the top,
// middle and bottom 8 bits of the significands. An infinity stands in the first part alone; the rest of a NaN is one again, since its
// first 16 bits may be those of an infinity.
__device__ __forceinline__ uint4 pairs_bf16(const uint4& x)
{
    return make_uint4(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632), __byte_perm(x.y, x.w, 0x5410), __byte_perm(x.y, x.w, 0x7632));
}
__device__ __forceinline__ void pairs_f32(const uint4& u, const uint4& v, uint4 (&b)[3])
{
    const uint32_t x[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        r[e] = __uint_as_float(x[e]) - __uint_as_float(x[e] & 0xffff0000u);
        if (fabsf(__uint_as_float(x[e])) == INFINITY) r[e] = 0.0f;
    }
    b[0] = make_uint4(__byte_perm(x[0], x[4], 0x7632), __byte_perm(x[1], x[5], 0x7632), __byte_perm(x[2], x[6], 0x7632), __byte_perm(x[3], x[7], 0x7632));
#pragma unroll
    for (int k = 1; k < 3; ++k) {
        uint32_t y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            y[e] = __float_as_uint(r[e]);
            if (k == 1) r[e] -= __uint_as_float(y[e] & 0xffff0000u);
        }
        b[k] = make_uint4(__byte_perm(y[0], y[4], 0x7632), __byte_perm(y[1], y[5], 0x7632), __byte_perm(y[2], y[6], 0x7632), __byte_perm(y[3], y[7], 0x7632));
    }
}

// RT: tiles of 16 output channels, MT: tiles of 8 tokens; XF: X is fp32; FINE: groups that are no multiple of 128; RES: all activations
// lie in shared memory as operands from the start, else those of a chunk come with its codes.
// A block goes through tiles of 16 RT output channels; its warps take the chunks of 128 input channels in turn, each with its own
// ring of stages that runs on over the end of a tile.
template <int RT, int MT, bool XF, bool FINE, bool RES>
__global__ void __launch_bounds__(32 * kMaxWarps, 1) linear_w4g_kernel(const W4Params p)
{
    using S = Stage<RT, MT, XF, RES>;
    constexpr int kCols = MT * 8, kRows = RT * 16, kParts = XF ? 3 : 1;
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int g = lane >> 2, t = lane & 3;
    // this warp's output channels within a tile, its first chunk, and the step to the next
    const int side = warp & ((1 << p.side_log) - 1), first = warp >> p.side_log, step = warps >> p.side_log;
    const int m0 = blockIdx.y * kCols, m_here = min(p.M - m0, kCols);
    char* ring = smem + warp * p.stages * S::kBytes;
    // two sets of [step][kCols][channels of a tile], used in turn
    float* part = reinterpret_cast<float*>(smem + warps * p.stages * S::kBytes);
    uint4* resident = reinterpret_cast<uint4*>(part + 2 * warps * kRows * kCols);  // [chunk][word][part][token][t]
    if (!RES) {                                           // rows of activations that no copy fills stay zero
        for (int i = lane; i < p.stages * S::kBytes / 16; i += 32) reinterpret_cast<uint4*>(ring)[i] = make_uint4(0u, 0u, 0u, 0u);
        __syncwarp();
    }
    CodeFeed<RT> feed;
    feed.enter(p, (int)blockIdx.x, side, first, g, t);
    XFeed<MT, XF, FINE> xfeed;
    if (!RES) xfeed.enter(p, m0, lane);
    const uint32_t ring_u = smem_u32(ring);
    // copies of the next chunk of this warp, `stages` - 1 ahead of the products; a group even where there is none
    auto copy = [&]() {
        if (feed.tile < p.tiles && feed.chunk < p.chunks) {
            const uint32_t to = ring_u + (uint32_t)(feed.slot * S::kBytes);
            feed.template copy<FINE>(p, to, g, t);
            if (!RES) xfeed.copy(p, to + S::kCodes, feed.chunk, m_here);
            feed.slot = feed.slot + 1 < p.stages ? feed.slot + 1 : 0;
            feed.chunk += step;
            if (feed.chunk >= p.chunks) feed.enter(p, feed.tile + (int)gridDim.x, side, first, g, t);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll 1
    for (int i = 1; i < p.stages; ++i) copy();
    // scales of this lane's rows and channels, loaded two chunks ahead
    Scales<RT, FINE> scales;
    constexpr int kS = Scales<RT, FINE>::kN;
    scales.enter(p, (int)blockIdx.x, side, first, g, t);
    float s0[kS], s1[kS];
    scales.load(p, side, first, step, g, t, s0);
    scales.load(p, side, first, step, g, t, s1);
    // columns of absent tokens repeat the last one's operands: nothing reads them
    int b_lane[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) b_lane[j] = min(j * 8 + g, m_here - 1) * 4 + t;
    if (RES) {
        // words ci = 4 chunk + i of the tokens; eight rows of four lanes take as many words at once as there are tokens less
        const int shift = m_here > 4 ? 3 : m_here > 2 ? 2 : m_here > 1 ? 1 : 0, per = 8 >> shift;
        constexpr int kAtOnce = XF ? 4 : 8;               // words in flight per lane
        for (int token = g & ((1 << shift) - 1); token < m_here; token += 8)
        for (int c0 = warp * per + (g >> shift); c0 < p.chunks * 4; c0 += kAtOnce * warps * per) {
            uint4 u[kAtOnce], v[XF ? kAtOnce : 1];
#pragma unroll
            for (int n = 0; n < kAtOnce; ++n) {
                const int ci = c0 + n * warps * per, k = (ci >> 2) * 128 + 8 * (FINE ? 4 * (ci & 3) + t : 4 * t + (ci & 3));
                u[n] = make_uint4(0u, 0u, 0u, 0u);
                if (XF) v[XF ? n : 0] = make_uint4(0u, 0u, 0u, 0u);
                if (k < p.K) {
                    const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p.X) + ((m0 + token) * p.ldx + k) * (XF ? 4 : 2));
                    u[n] = __ldg(src);
                    if (XF) v[XF ? n : 0] = __ldg(src + 1);
                }
            }
#pragma unroll
            for (int n = 0; n < kAtOnce; ++n) {
                const int ci = c0 + n * warps * per;
                if (ci >= p.chunks * 4) continue;
                uint4 b[3], *to = resident + (ci * kParts * m_here + token) * 4 + t;
                if (XF) pairs_f32(u[n], v[XF ? n : 0], b);
                else b[0] = pairs_bf16(u[n]);
#pragma unroll
                for (int q = 0; q < kParts; ++q) to[q * 4 * m_here] = b[q];
            }
        }
        __syncthreads();
    }

    int slot = 0, turn = 0;
    for (int tile = blockIdx.x; tile < p.tiles; tile += gridDim.x, turn ^= 1) {
        // this thread's outputs of the tile, threadIdx.x, + blockDim.x, ..., share a channel: blockDim.x is a multiple of the tile's
        const int channels = kRows << p.side_log, n_out = tile * channels + (threadIdx.x & (channels - 1));
        const float bias = p.bias != nullptr && n_out < p.N ? __ldg(p.bias + n_out) : 0.0f;
        float acc[RT][MT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[r][j][i] = 0.0f;
#pragma unroll 1
        for (int c = first; c < p.chunks; c += step) {
            copy();
            if (p.stages == 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
            else asm volatile("cp.async.wait_group 2;" ::: "memory");
            __syncwarp();
            float now[kS];
#pragma unroll
            for (int i = 0; i < kS; ++i) {
                now[i] = s0[i];
                s0[i] = s1[i];
            }
            scales.load(p, side, first, step, g, t, s1);
            const char* codes = ring + slot * S::kBytes;
            const char* xs = codes + S::kCodes;
            const uint4* bs = resident + c * (16 * kParts) * m_here;
            uint4 w[RT][2];
            if (!FINE)
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h) w[r][h] = lds128(codes + (r * 16 + h * 8 + g) * 64 + t * 16);
            float sum[RT][MT][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {                 // 32 channels: word i of the four lanes, or (FINE) the four words of group i
                if (FINE || i == 0)
#pragma unroll
                    for (int r = 0; r < RT; ++r)
#pragma unroll
                        for (int j = 0; j < MT; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) sum[r][j][e] = 0.0f;
                uint32_t a[RT][2][4];
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    uint32_t v[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int row = r * 16 + h * 8 + g;
                        v[h] = FINE ? *reinterpret_cast<const uint32_t*>(codes + row * 64 + code_piece<FINE>(row, i) * 16 + t * 4) : word_of(w[r][h], i);
                    }
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        a[r][q][0] = codes2(v[0], 2 * q);
                        a[r][q][1] = codes2(v[1], 2 * q);
                        a[r][q][2] = codes2(v[0], 2 * q + 1);
                        a[r][q][3] = codes2(v[1], 2 * q + 1);
                    }
                }
                const int eight = FINE ? 4 * i + t : 4 * t + i;                   // this lane's eight channels of the chunk
#pragma unroll
                for (int j = 0; j < MT; ++j) {
                    const char* xr = xs + (j * 8 + g) * S::kRow;
                    uint4 b[3];
                    if (RES) {
#pragma unroll
                        for (int q = 0; q < kParts; ++q) b[q] = bs[(i * kParts + q) * 4 * m_here + b_lane[j]];
                    } else if (XF) pairs_f32(lds128(xr + x_piece<XF, FINE>(g, 2 * eight) * 16), lds128(xr + x_piece<XF, FINE>(g, 2 * eight + 1) * 16), b);
                    else b[0] = pairs_bf16(lds128(xr + x_piece<XF, FINE>(g, eight) * 16));
#pragma unroll
                    for (int q = kParts - 1; q >= 0; --q)                         // the smallest part first
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            mma_bf16(sum[r][j], a[r][0], b[q].x, b[q].y);
                            mma_bf16(sum[r][j], a[r][1], b[q].z, b[q].w);
                        }
                }
                if (FINE || i == 3)
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        const float lo = Scales<RT, FINE>::get(now, r, 0, i, lane), hi = Scales<RT, FINE>::get(now, r, 1, i, lane);
#pragma unroll
                        for (int j = 0; j < MT; ++j) {
                            acc[r][j][0] = fmaf(lo, sum[r][j][0], acc[r][j][0]);
                            acc[r][j][1] = fmaf(lo, sum[r][j][1], acc[r][j][1]);
                            acc[r][j][2] = fmaf(hi, sum[r][j][2], acc[r][j][2]);
                            acc[r][j][3] = fmaf(hi, sum[r][j][3], acc[r][j][3]);
                        }
                    }
            }
            slot = slot + 1 < p.stages ? slot + 1 : 0;
            __syncwarp();                                 // all lanes have read the stage that is filled next
        }
        // ---- sums of the warps that split K, added in their order
        float* set = part + turn * warps * kRows * kCols;
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    set[(first * kCols + j * 8 + 2 * t + (i & 1)) * channels + side * kRows + r * 16 + (i >> 1) * 8 + g] = acc[r][j][i];
        __syncthreads();
        for (int e = threadIdx.x; e < channels * m_here; e += blockDim.x) {
            if (n_out >= p.N) break;
            float v = 0.0f;
            for (int u = 0; u < step; ++u) v += set[u * channels * kCols + e];
            v = activate(fmaf(v, 1024.0f, bias), p.act);
            const int64_t at = (int64_t)(m0 + (e >> (p.side_log + (RT == 1 ? 4 : 5)))) * p.N + n_out;
            if (p.y_bf) reinterpret_cast<__nv_bfloat16*>(p.Y)[at] = __float2bfloat16_rn(v);
            else reinterpret_cast<float*>(p.Y)[at] = v;
        }
    }
}

// Many rows: a block of eight warps takes 128 RT output channels and 8 MT tokens. The activations of a chunk come into shared memory
// once for all its warps (fp32 ones are cut into their parts there, once); a word of codes is widened once for all its tokens. A cluster of
// blocks splits the chunks of a tile, and its blocks add up the sums of their share of the tokens, in the order of the chunks.
// What bounds it: with 64 rows some 660 instructions per 32 output channels and chunk from eight warps an SM, half of what mma.sync can
// do, on 128 of the SMs (a tile's clusters do not fill the rest); with 32 rows the widening, half of its instructions. 8192 > 16384 in
// groups of 128: 32 rows 46 us, 64 rows 70 to 75 (the kernel above, in passes of 16 rows: 62 and 115 to 125), 64 fp32 rows 173 (303).
// Twice the warps an SM with half the output channels each: 50 us for 32 rows, 72 for 64.
template <int RT, int MT, bool XF>
struct ManyStage {
    static constexpr int kCodes = RT * 8192, kRow = XF ? 512 : 256, kBytes = kCodes + MT * 8 * kRow, kStages = !XF || MT == 1 ? 4 : MT == 2 ? 3 : 2;
    static constexpr int kOps = XF ? MT * 8 * 768 : 0, kAll = kStages * kBytes + kOps, kSum = RT * 128 + 4;    // fp32 parts; floats a token
    static_assert(MT * 8 * kSum * 4 <= kAll, "the sums lie where the stages were");
};
__device__ __forceinline__ int raw_piece(int p) { return p ^ ((p >> 3) & 1); }

template <int RT, int MT, bool XF, bool FINE>
__global__ void __launch_bounds__(256, RT * MT > 8 ? 1 : RT * MT > 4 ? 2 : 3) linear_w4g_many_kernel(const W4Params p)
{
    using S = ManyStage<RT, MT, XF>;
    constexpr int kTokens = MT * 8, kRows = RT * 128, kParts = XF ? 3 : 1, kPieces = S::kRow / 16, kPer = XF ? 4 : 8, kSize = XF ? 4 : 2;
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g = lane >> 2, t = lane & 3;
    const cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), tile = (int)blockIdx.x / ranks;
    const int begin = p.chunks * rank / ranks, end = p.chunks * (rank + 1) / ranks;
    const int m0 = blockIdx.y * kTokens, m_here = min(p.M - m0, kTokens);
    char* ops = smem + S::kStages * S::kBytes;            // [part][token], as the activations of a stage lie
    // this thread's copies: piece threadIdx.x & 3 of every 64th row of codes, piece q of every (256 / kPieces)th row of activations
    const int piece = threadIdx.x & 3, q = threadIdx.x % kPieces, r0 = threadIdx.x / kPieces;
    const uint8_t* codes_at = p.Wp + (int64_t)tile * kRows * (p.K >> 1);
    uint32_t row_at[RT * 2];                              // rows behind the last output channel repeat it
#pragma unroll
    for (int i = 0; i < RT * 2; ++i) row_at[i] = (uint32_t)min(i * 64 + (int)(threadIdx.x >> 2), p.N - 1 - tile * kRows) * (uint32_t)(p.K >> 1) + piece * 16;
    const char* x_at = reinterpret_cast<const char*>(p.X) + (int64_t)m0 * p.ldx * kSize;
    auto copy = [&](int c) {
        if (c < end) {
            const uint32_t to = smem_u32(smem) + (uint32_t)((c - begin) % S::kStages * S::kBytes);
            const bool in = c * 128 + piece * 32 < p.K;   // else zeros; the address stays inside the row
#pragma unroll
            for (int i = 0; i < RT * 2; ++i) {
                const int row = i * 64 + (threadIdx.x >> 2);
                copy16(to + (uint32_t)(row * 64 + code_piece<FINE>(row, piece) * 16), codes_at + row_at[i] + (in ? c * 64 : -16 * piece), in);
            }
            const int k = c * 128 + q * kPer;
#pragma unroll
            for (int i = 0; i < kTokens * kPieces / 256; ++i) {
                const int row = i * (256 / kPieces) + r0, at = XF ? raw_piece(q) : x_piece<false, FINE>(row, q);
                const bool here = row < m_here && k < p.K;
                copy16(to + (uint32_t)(S::kCodes + row * S::kRow + at * 16), x_at + (here ? (int64_t)row * p.ldx + k : 0) * kSize, here);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i + 1 < S::kStages; ++i) copy(begin + i);
    Scales<RT, FINE> scales;                              // of this warp's rows, loaded two chunks ahead
    constexpr int kS = Scales<RT, FINE>::kN;
    scales.enter(p, tile, warp, begin, g, t);
    float s0[kS], s1[kS];
    scales.load(p, warp, begin, 1, g, t, s0);
    scales.load(p, warp, begin, 1, g, t, s1);
    float acc[RT][MT][4];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[r][j][e] = 0.0f;
#pragma unroll 1
    for (int c = begin; c < end; ++c) {
        asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 2) : "memory");
        __syncthreads();                                  // the chunk is here, and all have read the one before it
        copy(c + S::kStages - 1);
        const char* stage = smem + (c - begin) % S::kStages * S::kBytes;
        const char* xs = XF ? ops : stage + S::kCodes;
        if (XF) {
#pragma unroll
            for (int i = 0; i < (MT + 1) / 2; ++i) {
                if (MT == 1 && threadIdx.x >= 128) break;
                const int token = i * 16 + (int)(threadIdx.x >> 4), eight = threadIdx.x & 15;
                const char* raw = stage + S::kCodes + token * 512;
                uint4 b[3];
                pairs_f32(lds128(raw + raw_piece(2 * eight) * 16), lds128(raw + raw_piece(2 * eight + 1) * 16), b);
#pragma unroll
                for (int u = 0; u < 3; ++u) *reinterpret_cast<uint4*>(ops + (u * kTokens + token) * 256 + x_piece<false, FINE>(token, eight) * 16) = b[u];
            }
            __syncthreads();
        }
        float now[kS];
#pragma unroll
        for (int i = 0; i < kS; ++i) {
            now[i] = s0[i];
            s0[i] = s1[i];
        }
        scales.load(p, warp, begin, 1, g, t, s1);
        uint4 w[RT][2];
        if (!FINE)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h) w[r][h] = lds128(stage + ((warp * RT + r) * 16 + h * 8 + g) * 64 + t * 16);
        float sum[RT][MT][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {                     // 32 channels, as above
            uint32_t a[RT][2][4];
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int row = (warp * RT + r) * 16 + h * 8 + g;
                    const uint32_t v = FINE ? *reinterpret_cast<const uint32_t*>(stage + row * 64 + code_piece<FINE>(row, i) * 16 + t * 4) : word_of(w[r][h], i);
                    const uint32_t c0 = codes2(v, 0), c1 = codes2(v, 1), c2 = codes2(v, 2), c3 = codes2(v, 3);
                    // bf16 activations stay as they lie, in pairs of neighbours: here the codes change places
                    a[r][0][h] = XF ? c0 : __byte_perm(c0, c1, 0x5410);
                    a[r][0][h + 2] = XF ? c1 : __byte_perm(c2, c3, 0x5410);
                    a[r][1][h] = XF ? c2 : __byte_perm(c0, c1, 0x7632);
                    a[r][1][h + 2] = XF ? c3 : __byte_perm(c2, c3, 0x7632);
                }
            const int eight = FINE ? 4 * i + t : 4 * t + i;
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                uint4 b[kParts];
#pragma unroll
                for (int u = 0; u < kParts; ++u) b[u] = lds128(xs + (u * kTokens + j * 8 + g) * 256 + x_piece<false, FINE>(g, eight) * 16);
#pragma unroll
                for (int u = kParts - 1; u >= 0; --u)     // the smallest part first
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        if (u == kParts - 1 && (FINE || i == 0)) mma_bf16_first(sum[r][j], a[r][0], b[u].x, b[u].y);
                        else mma_bf16(sum[r][j], a[r][0], b[u].x, b[u].y);
                        mma_bf16(sum[r][j], a[r][1], b[u].z, b[u].w);
                    }
            }
            if (FINE || i == 3)
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const float lo = Scales<RT, FINE>::get(now, r, 0, i, lane), hi = Scales<RT, FINE>::get(now, r, 1, i, lane);
#pragma unroll
                    for (int j = 0; j < MT; ++j) {
                        acc[r][j][0] = fmaf(lo, sum[r][j][0], acc[r][j][0]);
                        acc[r][j][1] = fmaf(lo, sum[r][j][1], acc[r][j][1]);
                        acc[r][j][2] = fmaf(hi, sum[r][j][2], acc[r][j][2]);
                        acc[r][j][3] = fmaf(hi, sum[r][j][3], acc[r][j][3]);
                    }
                }
        }
    }
    __syncthreads();                                      // the stages are read
    float* sums = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sums[(j * 8 + 2 * t + (e & 1)) * S::kSum + (warp * RT + r) * 16 + (e >> 1) * 8 + g] = acc[r][j][e];
    cluster.sync();
    for (int token = warp * ranks + rank; token < m_here; token += 8 * ranks)
        for (int ch = lane * 4; ch < kRows; ch += 128) {
            const int n = tile * kRows + ch;
            if (n >= p.N) break;
            float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int u = 0; u < ranks; ++u) {
                const float4 x = *reinterpret_cast<const float4*>(cluster.map_shared_rank(sums, u) + token * S::kSum + ch);
                v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = activate(fmaf(v[e], 1024.0f, p.bias != nullptr && n + e < p.N ? __ldg(p.bias + n + e) : 0.0f), p.act);
            const int64_t at = (int64_t)(m0 + token) * p.N + n;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < p.N) {
                    if (p.y_bf) reinterpret_cast<__nv_bfloat16*>(p.Y)[at + e] = __float2bfloat16_rn(v[e]);
                    else reinterpret_cast<float*>(p.Y)[at + e] = v[e];
                }
        }
    cluster.sync();                                       // no block leaves while others read its sums
}

template <int RT, int MT, bool XF, bool FINE>
int launch_w4_many(stwq_ctx* ctx, W4Params& p, cudaStream_t st)
{
    using S = ManyStage<RT, MT, XF>;
    auto kern = linear_w4g_many_kernel<RT, MT, XF, FINE>;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(8);
    cfg.blockDim = dim3(256);
    cfg.dynamicSmemBytes = S::kAll;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    uint16_t* fit = ctx->w4g_clusters[(RT - 1) | (XF ? 2 : 0) | (FINE ? 4 : 0) | (MT == 1 ? 24 : MT == 2 ? 0 : MT == 4 ? 8 : 16)];
    if (!fit[0]) {
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kAll);
        for (int r = 1; r <= 8 && e == cudaSuccess; ++r) {
            int n = 0;
            at[0].val.clusterDim.x = cfg.gridDim.x = (unsigned)r;
            e = cudaOccupancyMaxActiveClusters(&n, kern, &cfg);
            fit[r] = (uint16_t)n;
        }
        if (e != cudaSuccess) return stwq_cuda_fail(ctx, e);
        fit[0] = 1;
    }
    p.side_log = 3;                                       // eight warps side by side
    p.tiles = (p.N + RT * 128 - 1) / (RT * 128);
    const int passes = (p.M + MT * 8 - 1) / (MT * 8);
    // Blocks of a cluster: a round costs its chunks and some six more for its start, its end and the exchange.
    int ranks = 1;
    int64_t best = INT64_MAX;
    for (int r = 1; r <= 8 && r <= p.chunks; ++r) {
        if (fit[r] == 0) continue;
        const int64_t cost = (((int64_t)p.tiles * passes + fit[r] - 1) / fit[r]) * ((p.chunks + r - 1) / r + 6);
        if (cost < best) {
            best = cost;
            ranks = r;
        }
    }
    at[0].val.clusterDim.x = (unsigned)ranks;
    cfg.gridDim = dim3((unsigned)(p.tiles * ranks), (unsigned)passes);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, p);
    ctx->launches += 1;
    return e == cudaSuccess ? STWQ_OK : stwq_cuda_fail(ctx, e);
}

template <int RT, int MT, bool XF, bool FINE, bool RES>
int launch_w4(stwq_ctx* ctx, W4Params& p, size_t resident, cudaStream_t st)
{
    constexpr int kCols = MT * 8, kRows = RT * 16, kStage = Stage<RT, MT, XF, RES>::kBytes, kSets = 2 * kRows * kCols * 4;
    // Two blocks of eight warps on an SM where there are tiles for them and rings of three stages and the activations fit twice, else one
    // of up to sixteen; four stages where there is room.
    constexpr size_t kHalf = 112 * 1024, kAll = 220 * 1024;
    const int strips = (p.N + kRows - 1) / kRows;         // of 16 RT output channels
    const bool two = strips > ctx->sm_count && 8 * (3 * kStage + kSets) + resident <= kHalf;
    int warps = 1;
    while (2 * warps <= (two ? 8 : kMaxWarps) && warps < p.chunks && (size_t)2 * warps * (3 * kStage + kSets) + resident <= (two ? kHalf : kAll)) warps *= 2;
    p.stages = (size_t)warps * (4 * kStage + kSets) + resident <= (two ? kHalf : kAll) ? 4 : 3;
    const size_t smem = (size_t)warps * (p.stages * kStage + kSets) + resident;
    auto kern = linear_w4g_kernel<RT, MT, XF, FINE, RES>;
    cudaError_t e = cudaSuccess;
    constexpr uint32_t kVariant = 1u << ((RT - 1) | (MT - 1) << 1 | (XF ? 4 : 0) | (FINE ? 8 : 0) | (RES ? 16 : 0));
    if (!(ctx->w4g_configured & kVariant)) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kAll);
        if (e != cudaSuccess) return stwq_cuda_fail(ctx, e);
        ctx->w4g_configured |= kVariant;
    }
    const int slots = (two ? 2 : 1) * ctx->sm_count;
    const int passes = (p.M + kCols - 1) / kCols, share = slots / passes > 0 ? slots / passes : 1;        // over the weights, side by side
    // A tile costs its chunks per warp and about one more for its end (sums, barrier, addresses): strips side by side have fewer ends,
    // strips one by one leave fewer blocks idle in the last round.
    int best = 0x7fffffff;
    for (int log = 0; (1 << log) <= warps; ++log) {
        const int tiles = (strips + (1 << log) - 1) >> log, step = warps >> log, cost = (tiles + share - 1) / share * ((p.chunks + step - 1) / step + 1);
        if (cost < best) {
            best = cost;
            p.side_log = log;
            p.tiles = tiles;
        }
    }
    const dim3 grid((unsigned)(p.tiles < share ? p.tiles : share), (unsigned)passes);
    kern<<<grid, 32 * warps, smem, st>>>(p);
    ctx->launches += 1;
    e = cudaGetLastError();
    return e == cudaSuccess ? STWQ_OK : stwq_cuda_fail(ctx, e);
}

template <bool FINE, bool XF>
int launch_w4_any(stwq_ctx* ctx, W4Params& p, cudaStream_t st)
{
    const int sm = ctx->sm_count;
    const size_t token = (size_t)p.chunks * 128 * (XF ? 6 : 2);            // bytes of a token's operands
    // The kernel for many rows, over N = 256 to 14000 and K = 1024 to 8192 (its time over that of this one in passes of 8 or 16 rows):
    // bf16, 64 rows 0.64 to 0.95 above N = 16 SMs, 48 rows 0.73 to 0.92 above 32 SMs, 1.0 to 1.3 between 16 and 32; 17 to 32 rows
    // 0.74 to 0.95 above 16 SMs, where tiles of 128 output channels win up to 48 SMs, of 256 beyond. fp32 the same with a pass for every
    // 32 rows (64 rows 0.48 to 0.97, 17 rows 0.7 to 0.97 above 24 SMs, 1.1 to 1.3 below). Fewer channels keep too few of its blocks busy: 1.1
    // to 2.7. 9 to 16 rows: fp32 0.67 to 0.95 (1.1 where it is worst), up to 16 SMs only while K is short (0.82 to 1.0, else 1.2); bf16 0.8 to 1.3: not taken.
    // 4 to 8 fp32 rows 0.68 to 1.0 up to 48 SMs, but 1.0 to 1.2 where its tiles are 8 to 16 and the other kernel's one for every SM; 1 to 3 rows 1.0 to 1.6.
    if (!XF && p.M > 32 && p.N > (p.M > 48 ? 16 : 32) * sm) return launch_w4_many<2, 8, false, FINE>(ctx, p, st);
    if (p.M > 16 && (XF || p.M <= 32)) {
        const int64_t work = (int64_t)p.N * ((p.M + 31) / 32);
        if (work > 48 * sm) return launch_w4_many<2, 4, XF, FINE>(ctx, p, st);
        if (work > (XF && p.M <= 24 ? 24 : 16) * sm) return launch_w4_many<1, 4, XF, FINE>(ctx, p, st);
    }
    if (XF && p.M > 8 && p.M <= 16 && (p.N > 16 * sm || token * p.M <= 144 * 1024)) return launch_w4_many<1, 2, true, FINE>(ctx, p, st);
    if (XF && p.M >= 4 && p.M <= 8 && p.N <= 48 * sm && (p.N <= 8 * sm || p.N > 16 * sm)) return launch_w4_many<1, 1, true, FINE>(ctx, p, st);
    // Tiles of 32 output channels share the operands of X, tiles of 16 spread further. Over K = 1024 to 8192 and 1 to 16 rows, 32 against
    // 16 took 1.22 times as long at N = 2048, 0.94 at 2560 to 4608, 0.92 to 1.0 above: 16 only while each has an SM of its own.
    const bool wide = p.N > 16 * sm;
    // the activations of up to 8 tokens as operands in shared memory, where that leaves room for the rings
    const size_t one = token * (p.M < 8 ? p.M : 8);
    if (one <= 96 * 1024 && (XF || p.M <= 8))
        return wide ? launch_w4<2, 1, XF, FINE, true>(ctx, p, one, st) : launch_w4<1, 1, XF, FINE, true>(ctx, p, one, st);
    if (XF || p.M <= 8) return wide ? launch_w4<2, 1, XF, FINE, false>(ctx, p, 0, st) : launch_w4<1, 1, XF, FINE, false>(ctx, p, 0, st);
    return wide ? launch_w4<2, 2, false, FINE, false>(ctx, p, 0, st) : launch_w4<1, 2, false, FINE, false>(ctx, p, 0, st);
}

int check_group(int N, int K, int group)
{
    if (N <= 0 || N > (1 << 30) || K <= 0 || K >= 131072 || group <= 0 || group > K) return STWQ_ERR_DIM;
    return (group & 31) != 0 || K % group != 0 ? STWQ_ERR_ALIGN : STWQ_OK;
}

}  // namespace

extern "C" {

int gps_fold_group4(stwq_ctx* ctx, const float* W, int N, int K, const float* s_ch, int group, uint8_t* Wp, void* s_g, int s_dtype,
                    void* stream)
{
    if (!ctx || !W || !Wp || !s_g) return STWQ_ERR_NULL;
    const int rc = check_group(N, K, group);
    if (rc != STWQ_OK) return rc;
    if (s_dtype != STWQ_OUT_F32 && s_dtype != STWQ_OUT_BF16) return STWQ_ERR_BITS;
    if (!stwq_aligned16(W) || !stwq_aligned16(Wp) || !stwq_aligned16(s_ch) || !stwq_aligned16(s_g)) return STWQ_ERR_ALIGN;
    const int64_t w_bytes = (int64_t)N * K * 4, es = s_dtype == STWQ_OUT_F32 ? 4 : 2;
    // warps read the operands while others already store
    const int64_t s_bytes = (int64_t)N * (K / group) * es, c_bytes = (int64_t)K * 4;
    if (stwq_overlap(Wp, w_bytes / 8, W, w_bytes) || stwq_overlap(Wp, w_bytes / 8, s_ch, c_bytes) || stwq_overlap(s_g, s_bytes, W, w_bytes) ||
        stwq_overlap(s_g, s_bytes, s_ch, c_bytes) || stwq_overlap(s_g, s_bytes, Wp, w_bytes / 8))
        return STWQ_ERR_ALIGN;
    StwqDevGuard dev(ctx->device);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t groups = (int64_t)N * (K / group), want = (groups + 7) / 8;
    const unsigned blocks = (unsigned)(want < 16 * ctx->sm_count ? want : 16 * ctx->sm_count);
    if (s_dtype == STWQ_OUT_F32) fold_group4_kernel<float><<<blocks, 256, 0, st>>>(W, groups, K, s_ch, group, Wp, static_cast<float*>(s_g));
    else fold_group4_kernel<__nv_bfloat16><<<blocks, 256, 0, st>>>(W, groups, K, s_ch, group, Wp, static_cast<__nv_bfloat16*>(s_g));
    ctx->launches += 1;
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? STWQ_OK : stwq_cuda_fail(ctx, e);
}

int linear_w4g(stwq_ctx* ctx, const void* X, int64_t ldx, int x_dtype, int64_t M, int K, int N, const uint8_t* Wp, const void* s_g,
               int s_dtype, int group, const float* bias, int act, int out_dtype, void* Y, void* stream)
{
    if (!ctx || !X || !Wp || !s_g || !Y) return STWQ_ERR_NULL;
    const int rc = check_group(N, K, group);
    if (rc == STWQ_ERR_DIM || M <= 0 || M > kMaxRows || ldx < K) return STWQ_ERR_DIM;
    auto real = [](int t) { return t == STWQ_OUT_F32 || t == STWQ_OUT_BF16; };
    if (!real(x_dtype) || !real(s_dtype) || !real(out_dtype) || act < STWQ_ACT_NONE || act > STWQ_ACT_GELU_FAST) return STWQ_ERR_BITS;
    const bool xf = x_dtype == STWQ_OUT_F32;
    if (rc != STWQ_OK || ldx % (xf ? 4 : 8) != 0 || !stwq_aligned16(X) || !stwq_aligned16(Wp)) return STWQ_ERR_ALIGN;
    auto aligned = [](const void* q, int bytes) { return (reinterpret_cast<uintptr_t>(q) & (uintptr_t)(bytes - 1)) == 0; };
    if (!aligned(s_g, s_dtype == STWQ_OUT_F32 ? 4 : 2) || !aligned(Y, out_dtype == STWQ_OUT_F32 ? 4 : 2) || !aligned(bias, 4)) return STWQ_ERR_ALIGN;
    // blocks read the operands while others already store
    const int64_t ex = xf ? 4 : 2, es = s_dtype == STWQ_OUT_F32 ? 4 : 2, y_bytes = M * N * (out_dtype == STWQ_OUT_F32 ? 4 : 2);
    if (stwq_overlap(Y, y_bytes, X, ((M - 1) * ldx + K) * ex) || stwq_overlap(Y, y_bytes, Wp, (int64_t)N * (K / 2)) ||
        stwq_overlap(Y, y_bytes, s_g, (int64_t)N * (K / group) * es) || stwq_overlap(Y, y_bytes, bias, (int64_t)N * 4))
        return STWQ_ERR_ALIGN;
    W4Params p;
    p.X = X; p.ldx = ldx; p.M = (int)M; p.K = K; p.N = N; p.per_row = K / group; p.chunks = (K + 127) / 128;
    p.Wp = Wp; p.s_g = s_g; p.s_bf = s_dtype == STWQ_OUT_BF16; p.bias = bias; p.act = act; p.y_bf = out_dtype == STWQ_OUT_BF16; p.Y = Y;
    p.group32 = (uint32_t)group / 32;
    p.magic = (uint32_t)(((1ull << 32) + p.group32 - 1) / p.group32);
    StwqDevGuard dev(ctx->device);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (group % 128 == 0) return xf ? launch_w4_any<false, true>(ctx, p, st) : launch_w4_any<false, false>(ctx, p, st);
    return xf ? launch_w4_any<true, true>(ctx, p, st) : launch_w4_any<true, false>(ctx, p, st);
}

}  // extern "C"
