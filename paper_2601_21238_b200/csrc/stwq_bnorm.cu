// The pass between two linears of a transformer block: residual sum, gate, norms, modulation, codes (block_norm).
//
// For a row of C channels, in fp32:
//     h' = h + r g (Npost(o) wp + bp),   y = (Npre(h') w + b) (1 + scale) + shift,
//     N: x / sqrt(mean(x^2) + eps), or (x - m) / sqrt(mean((x - m)^2) + eps) with m = mean(x), or x
//     out: y, y (1/s_ch), or the codes clamp(round((y rc) rt)), rc = 1/s_ch, rt = 1/s_tok[pos]
// Each row is read once and stays in registers: a mean and a sum of squares are one reduction each over the threads of the
// row, the squares are those of the centred values. Bound by HBM: |h| + |o| in, |h'| + |y| out; the vectors of C channels
// (weights, gate, scale, shift) come from L1 and L2, which is why a group of threads takes consecutive rows.
#include <cuda_bf16.h>

#include "stwq_internal.cuh"
#include "stwq_paged.cuh"

namespace {

constexpr int kMaxC = 16384;
constexpr int kMaxThreads = 512;           // of one row
constexpr int kWarpRows = 4;               // rows a block works on where a warp holds a row

struct BnParams {
    const void *H, *O, *gate, *scale, *shift;
    void *Ho, *Y;
    int64_t ldh, ldo, ldc, ldho, ldy, M;
    int C, G, P, h_bf, o_bf, c_bf, y_dtype, post, pre, qmin, qmax, rows;
    const int32_t *cond, *pos;
    const float *wp, *bp, *w, *b, *s_ch, *s_tok;
    float res_scale, eps, inv_C;
    uint32_t* status;
};

// Eight elements from `at` on. Rows are read with plain loads: the outputs may replace them.
__device__ __forceinline__ void load8(const void* base, int64_t at, int bf, float (&v)[8])
{
    if (bf) {
        const uint4 a = *reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(base) + at);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
        const float4* q = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + at);
        const float4 a = q[0], b = q[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
}
__device__ __forceinline__ void store8(void* base, int64_t at, int bf, const float (&v)[8])
{
    if (bf) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
        *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(base) + at) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        float4* q = reinterpret_cast<float4*>(reinterpret_cast<float*>(base) + at);
        q[0] = make_float4(v[0], v[1], v[2], v[3]);
        q[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// Sum over the threads of a row, the same value in all of them, added in a fixed order. `red` holds two sets of one value per
// warp, used in turn: no warp writes a set again before all have passed the barrier of the other one.
template <bool WARP>
__device__ __forceinline__ float row_sum(float v, float (*red)[kMaxThreads / 32], int& turn)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (WARP) return v;
    float* r = red[turn];
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) r[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.0f;
    for (int i = 0; i < (int)(blockDim.x >> 5); i += 4) {           // sets are padded with zeros
        const float4 q = *reinterpret_cast<const float4*>(r + i);
        s += (q.x + q.y) + (q.z + q.w);
    }
    return s;
}

// x <- N(x) w + b
template <int VPT, bool WARP>
__device__ __forceinline__ void normalise(float (&x)[VPT][8], int kind, const float* w, const float* b, const BnParams& p, int tid, int nt,
                                          float (*red)[kMaxThreads / 32], int& turn)
{
    float mean = 0.0f, r = 1.0f;
    if (kind == STWQ_NORM_LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < VPT; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += x[v][i];               // vectors beyond the row hold zeros
        mean = row_sum<WARP>(s, red, turn) * p.inv_C;
    }
    if (kind != STWQ_NORM_NONE) {
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < VPT; ++v)
            if ((v * nt + tid) * 8 < p.C)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float d = x[v][i] - mean;
                    s = fmaf(d, d, s);
                }
        r = rsqrtf(fmaf(row_sum<WARP>(s, red, turn), p.inv_C, p.eps));
    }
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int e0 = (v * nt + tid) * 8;
        if (e0 >= p.C) break;
        float a[8];
        if (kind != STWQ_NORM_NONE)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[v][i] = (x[v][i] - mean) * r;
        if (w != nullptr) {
            load8(w, e0, 0, a);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[v][i] *= a[i];
        }
        if (b != nullptr) {
            load8(b, e0, 0, a);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[v][i] += a[i];
        }
    }
}

// VPT vectors of eight channels per thread; WARP: a warp holds a row, else the block does.
template <int VPT, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kWarpRows : kMaxThreads) block_norm_kernel(const BnParams p)
{
    __shared__ __align__(16) float red[2][kMaxThreads / 32];
    const int tid = WARP ? threadIdx.x & 31 : threadIdx.x, nt = WARP ? 32 : blockDim.x;
    const int64_t group = WARP ? (int64_t)blockIdx.x * kWarpRows + (threadIdx.x >> 5) : blockIdx.x;
    int turn = 0;
    if (!WARP) {
        if (threadIdx.x < 2 * (kMaxThreads / 32)) (&red[0][0])[threadIdx.x] = 0.0f;
        __syncthreads();
    }
    const int64_t r1 = min(p.M, (group + 1) * p.rows);
    for (int64_t row = group * p.rows; row < r1; ++row) {
        const int pos = p.pos != nullptr ? p.pos[row] : 0;
        if (pos == -1) continue;                                    // a padding row
        int g = p.cond != nullptr ? p.cond[row] : 0;
        const bool bad_g = g < 0 || g >= p.G, bad_pos = p.y_dtype == STWQ_OUT_INT8 && (pos < 0 || pos >= p.P);
        if ((bad_g || bad_pos) && tid == 0) atomicOr(p.status, STWQ_DEV_POS_RANGE);
        if (bad_g) g = 0;
        const int64_t gc = g * p.ldc;

        float h[VPT][8];
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int e0 = (v * nt + tid) * 8;
            if (e0 < p.C) load8(p.H, row * p.ldh + e0, p.h_bf, h[v]);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) h[v][i] = 0.0f;
        }
        if (p.O != nullptr) {
            float o[VPT][8];
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                const int e0 = (v * nt + tid) * 8;
                if (e0 < p.C) load8(p.O, row * p.ldo + e0, p.o_bf, o[v]);
                else
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[v][i] = 0.0f;
            }
            normalise<VPT, WARP>(o, p.post, p.wp, p.bp, p, tid, nt, red, turn);
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                const int e0 = (v * nt + tid) * 8;
                if (e0 >= p.C) break;
                float a[8];
                if (p.gate != nullptr) load8(p.gate, gc + e0, p.c_bf, a);
                else
#pragma unroll
                    for (int i = 0; i < 8; ++i) a[i] = 1.0f;
                if (!bad_g)
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[v][i] = fmaf(p.res_scale * a[i], o[v][i], h[v][i]);
                if (p.Ho != nullptr) store8(p.Ho, row * p.ldho + e0, p.h_bf, h[v]);
            }
        }
        if (p.Y == nullptr) continue;
        normalise<VPT, WARP>(h, p.pre, p.w, p.b, p, tid, nt, red, turn);
        const float rt = p.y_dtype == STWQ_OUT_INT8 && !bad_pos ? __frcp_rn(p.s_tok[pos]) : 1.0f;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int e0 = (v * nt + tid) * 8;
            if (e0 >= p.C) break;
            float a[8];
            if (p.scale != nullptr) {
                load8(p.scale, gc + e0, p.c_bf, a);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[v][i] *= 1.0f + a[i];
            }
            if (p.shift != nullptr) {
                load8(p.shift, gc + e0, p.c_bf, a);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[v][i] += a[i];
            }
            if (p.s_ch != nullptr) {
                load8(p.s_ch, e0, 0, a);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[v][i] = __fmul_rn(h[v][i], __frcp_rn(a[i]));
            }
            if (bad_g || bad_pos)
#pragma unroll
                for (int i = 0; i < 8; ++i) h[v][i] = 0.0f;
            if (p.y_dtype == STWQ_OUT_INT8) {
                uint32_t w[2] = {0u, 0u};
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    w[i >> 2] |= (uint32_t)(stwq_code(__fmul_rn(h[v][i], rt), p.qmin, p.qmax) & 0xFF) << (8 * (i & 3));
                *reinterpret_cast<uint2*>(reinterpret_cast<int8_t*>(p.Y) + row * p.ldy + e0) = make_uint2(w[0], w[1]);
            } else store8(p.Y, row * p.ldy + e0, p.y_dtype == STWQ_OUT_BF16, h[v]);
        }
    }
}

template <int VPT, bool WARP>
int launch_bn(stwq_ctx* ctx, BnParams& p, int threads, cudaStream_t st)
{
    // consecutive rows per group while the groups still fill the GPU once
    const int64_t per_sm = WARP ? 2048 / 32 : 2048 / threads, slots = per_sm * ctx->sm_count;
    int64_t rows = (p.M + slots - 1) / slots;
    if (rows > 8) rows = 8;
    p.rows = (int)rows;
    const int64_t groups = (p.M + rows - 1) / rows, blocks = WARP ? (groups + kWarpRows - 1) / kWarpRows : groups;
    block_norm_kernel<VPT, WARP><<<(unsigned)blocks, WARP ? 32 * kWarpRows : threads, 0, st>>>(p);
    ctx->launches += 1;
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? STWQ_OK : stwq_cuda_fail(ctx, e);
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
    p.H = H; p.O = O; p.gate = gate; p.scale = scale; p.shift = shift; p.Ho = Hout; p.Y = Y;
    p.ldh = ldh; p.ldo = ldo; p.ldc = cond ? ldc : 0; p.ldho = ldho; p.ldy = ldy; p.M = M;
    p.C = C; p.G = cond ? G : 1; p.P = P;
    p.h_bf = h_dtype == STWQ_OUT_BF16; p.o_bf = o_dtype == STWQ_OUT_BF16; p.c_bf = c_dtype == STWQ_OUT_BF16; p.y_dtype = Y ? y_dtype : STWQ_OUT_F32;
    p.post = post_norm; p.pre = pre_norm;
    p.qmax = (1 << (bits == 6 ? 5 : 7)) - 1;
    p.qmin = -p.qmax - 1;
    p.cond = cond ? cond_ids : nullptr; p.pos = pos_ids;
    p.wp = w_post; p.bp = b_post; p.w = w_pre; p.b = b_pre; p.s_ch = s_ch; p.s_tok = s_tok;
    p.res_scale = res_scale; p.eps = eps; p.inv_C = 1.0f / (float)C;
    p.status = ctx->d_status;
    StwqDevGuard dev(ctx->device);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int vecs = C / 8;
    if (vecs <= 32) return launch_bn<1, true>(ctx, p, 32, st);
    if (vecs <= 64) return launch_bn<2, true>(ctx, p, 32, st);
    const int vpt = vecs <= kMaxThreads ? 1 : vecs <= 2 * kMaxThreads ? 2 : 4;
    const int threads = 32 * ((vecs + 32 * vpt - 1) / (32 * vpt));
    if (vpt == 1) return launch_bn<1, false>(ctx, p, threads, st);
    if (vpt == 2) return launch_bn<2, false>(ctx, p, threads, st);
    return launch_bn<4, false>(ctx, p, threads, st);
}
