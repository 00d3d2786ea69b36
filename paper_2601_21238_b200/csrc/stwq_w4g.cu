// Few-row products with 4-bit weights and a scale per group of input channels (linear_w4g), and the fold that makes
// the weights (gps_fold_group4).
//
//     Y[m,n] = act(sum_g s[n,g] sum_{k in g} X[m,k] c[n,k] + bias[n])
//
// Bound by HBM: N K / 2 bytes of codes, read once, straight into registers. The codes are the A operand (16 rows of n) of
// mma.sync m16n8k16, the activations the B operand (8 tokens): up to 8 rows of X cost what one costs. tcgen05 would need the
// codes widened into shared memory first; here a word of eight codes becomes four bf16 pairs in registers by masks and
// one subtraction each (0x3e00 | (nibble ^ 8) is 2^-3 + (code + 8) 2^-10 as bf16; less 2^-3 + 2^-7 it is code 2^-10, exactly).
// The 2^-10 keeps 128 codes times the largest activation inside fp32; it leaves the result at the end (bits below 2^-126 are lost).
// A lane loads 32 consecutive channels of a row (16 bytes), four lanes 128; the order in which channels meet in a product
// does not matter as long as both operands keep it, so word i of the four lanes gives the 32 channels of two products.
// Scales: where a group is a multiple of 128 channels, the products of one 128-channel chunk share it, and the chunk's fp32 sum
// is scaled once. Finer groups (a multiple of 32) differ between the four lanes; there the eight columns of B are 4 lanes x 2
// tokens, each column zero outside its lane's channels, so that every lane finds its own group's sums in its own accumulators.
// fp32 activations enter as three bf16 parts, cut off bit by bit (8 + 8 + 8 bits: exact), the smallest first.
// The warps of a block take different chunks of the same rows; their sums meet in shared memory and are added in warp order.
#include <cuda_bf16.h>

#include "stwq_internal.cuh"
#include "stwq_paged.cuh"
#include "stwq_ptx.cuh"

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
    int M, K, N, group, per_row, chunks;
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
// Nibbles q and q + 4 of a word as a pair of bf16: the codes times 2^-10.
__device__ __forceinline__ uint32_t codes2(uint32_t w, int q)
{
    const uint32_t t = ((w >> (4 * q)) & 0x000f000fu) ^ 0x3e083e08u;
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
__device__ __forceinline__ uint4 ld_weights(const uint8_t* p)
{
    uint4 v;
    asm("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// RT: tiles of 16 output channels per warp; MT: tiles of tokens (8, or 2 with FINE groups); XF: X is fp32.
template <int RT, int MT, bool XF, bool FINE>
__global__ void __launch_bounds__(32 * kMaxWarps, 1) linear_w4g_kernel(const W4Params p)
{
    constexpr int kTok = FINE ? 2 : 8;                    // tokens per tile
    constexpr int kCols = MT * kTok, kRows = RT * 16;
    extern __shared__ __align__(16) float part[];         // [warps][kRows][kCols]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * kRows, m0 = blockIdx.y * kCols;
    const int col = FINE ? (g & 1) : g;                   // the token of this lane's B fragments
    const bool holds = !FINE || (g >> 1) == t;

    float acc[RT][MT][4];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[r][j][i] = 0.0f;

    for (int c = warp; c < p.chunks; c += warps) {
        const int k = c * 128 + t * 32;
        const bool in = k < p.K;
        uint4 w[RT][2];
        float s[RT][2];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t n = min(n0 + r * 16 + h * 8 + g, p.N - 1);
                w[r][h] = in ? ld_weights(p.Wp + (n * p.K + k) / 2) : make_uint4(0u, 0u, 0u, 0u);
                const int64_t at = n * p.per_row + min(k, p.K - 1) / p.group;
                s[r][h] = p.s_bf ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p.s_g)[at]) : reinterpret_cast<const float*>(p.s_g)[at];
            }
        float sum[RT][MT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[r][j][i] = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {                     // word i: channels 8i .. 8i + 7 of the lane's 32
            uint32_t a[RT][2][4];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const uint32_t lo = i == 0 ? w[r][0].x : i == 1 ? w[r][0].y : i == 2 ? w[r][0].z : w[r][0].w;
                const uint32_t hi = i == 0 ? w[r][1].x : i == 1 ? w[r][1].y : i == 2 ? w[r][1].z : w[r][1].w;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    a[r][q][0] = codes2(lo, 2 * q);
                    a[r][q][1] = codes2(hi, 2 * q);
                    a[r][q][2] = codes2(lo, 2 * q + 1);
                    a[r][q][3] = codes2(hi, 2 * q + 1);
                }
            }
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const int m = m0 + j * kTok + col;
                const bool on = in && holds && m < p.M;
                if constexpr (!XF) {
                    uint4 x = make_uint4(0u, 0u, 0u, 0u);
                    if (on) x = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(p.X) + m * p.ldx + k + 8 * i));
                    const uint32_t b[4] = {__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632), __byte_perm(x.y, x.w, 0x5410),
                                           __byte_perm(x.y, x.w, 0x7632)};       // channels (0,4), (1,5), (2,6), (3,7)
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        mma_bf16(sum[r][j], a[r][0], b[0], b[1]);
                        mma_bf16(sum[r][j], a[r][1], b[2], b[3]);
                    }
                } else {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = 0.0f;
                    if (on) {
                        const float4* src = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.X) + m * p.ldx + k + 8 * i);
                        const float4 u = __ldg(src), v = __ldg(src + 1);
                        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
                        x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
                    }
                    uint32_t b[3][4];                     // the top, middle and bottom 8 bits of the significands
                    float rest[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        rest[e] = x[e] - __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u);
                        if (!(fabsf(x[e]) < INFINITY)) rest[e] = 0.0f;           // Inf and NaN stand in the first part alone
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) b[0][e] = __byte_perm(__float_as_uint(x[e]), __float_as_uint(x[e + 4]), 0x7632);
#pragma unroll
                    for (int e = 0; e < 4; ++e) b[1][e] = __byte_perm(__float_as_uint(rest[e]), __float_as_uint(rest[e + 4]), 0x7632);
#pragma unroll
                    for (int e = 0; e < 8; ++e) rest[e] -= __uint_as_float(__float_as_uint(rest[e]) & 0xffff0000u);
#pragma unroll
                    for (int e = 0; e < 4; ++e) b[2][e] = __byte_perm(__float_as_uint(rest[e]), __float_as_uint(rest[e + 4]), 0x7632);
#pragma unroll
                    for (int q = 2; q >= 0; --q)
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            mma_bf16(sum[r][j], a[r][0], b[q][0], b[q][1]);
                            mma_bf16(sum[r][j], a[r][1], b[q][2], b[q][3]);
                        }
                }
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[r][j][i] = fmaf(s[r][i >> 1], sum[r][j][i], acc[r][j][i]);
    }
    // ---- sums of the warps. A lane holds columns 2t, 2t + 1: two tokens, or (FINE) its own groups' part of tokens 0 and 1
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v = acc[r][j][i];
                if (FINE) {
                    v += __shfl_xor_sync(0xffffffffu, v, 1);
                    v += __shfl_xor_sync(0xffffffffu, v, 2);
                    if (t != 0) continue;
                }
                part[((warp * kCols) + j * kTok + (FINE ? 0 : 2 * t) + (i & 1)) * kRows + r * 16 + (i >> 1) * 8 + g] = v;
            }
    __syncthreads();
    for (int e = threadIdx.x; e < kRows * kCols; e += blockDim.x) {
        const int m = m0 + e / kRows, n = n0 + e % kRows;
        if (m >= p.M || n >= p.N) continue;
        float v = 0.0f;
        for (int u = 0; u < warps; ++u) v += part[u * kRows * kCols + e];
        v *= 1024.0f;
        if (p.bias != nullptr) v += p.bias[n];
        v = activate(v, p.act);
        const int64_t at = (int64_t)m * p.N + n;
        if (p.y_bf) reinterpret_cast<__nv_bfloat16*>(p.Y)[at] = __float2bfloat16_rn(v);
        else reinterpret_cast<float*>(p.Y)[at] = v;
    }
}

template <int RT, int MT, bool XF, bool FINE>
int launch_w4(stwq_ctx* ctx, const W4Params& p, cudaStream_t st)
{
    constexpr int kCols = MT * (FINE ? 2 : 8), kRows = RT * 16;
    int warps = 1;
    while (warps < kMaxWarps && warps < p.chunks) warps *= 2;
    const size_t smem = (size_t)warps * kRows * kCols * 4;
    const dim3 grid((unsigned)((p.N + kRows - 1) / kRows), (unsigned)((p.M + kCols - 1) / kCols));
    linear_w4g_kernel<RT, MT, XF, FINE><<<grid, 32 * warps, smem, st>>>(p);
    ctx->launches += 1;
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? STWQ_OK : stwq_cuda_fail(ctx, e);
}

template <int RT, int MT, bool FINE>
int launch_w4_any(stwq_ctx* ctx, const W4Params& p, bool xf, cudaStream_t st)
{
    return xf ? launch_w4<RT, MT, true, FINE>(ctx, p, st) : launch_w4<RT, MT, false, FINE>(ctx, p, st);
}

int check_group(int N, int K, int group)
{
    if (N <= 0 || K <= 0 || K >= 131072 || group <= 0 || group > K) return STWQ_ERR_DIM;
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
    W4Params p;
    p.X = X; p.ldx = ldx; p.M = (int)M; p.K = K; p.N = N; p.group = group; p.per_row = K / group; p.chunks = (K + 127) / 128;
    p.Wp = Wp; p.s_g = s_g; p.s_bf = s_dtype == STWQ_OUT_BF16; p.bias = bias; p.act = act; p.y_bf = out_dtype == STWQ_OUT_BF16; p.Y = Y;
    StwqDevGuard dev(ctx->device);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    // tokens per pass over the weights: 8 or 16; 2, 4 or 8 with groups that differ between the lanes
    if (group % 128 == 0) return M <= 8 ? launch_w4_any<1, 1, false>(ctx, p, xf, st) : launch_w4_any<1, 2, false>(ctx, p, xf, st);
    if (M <= 2) return launch_w4_any<1, 1, true>(ctx, p, xf, st);
    return M <= 4 ? launch_w4_any<1, 2, true>(ctx, p, xf, st) : launch_w4_any<1, 4, true>(ctx, p, xf, st);
}

}  // extern "C"
