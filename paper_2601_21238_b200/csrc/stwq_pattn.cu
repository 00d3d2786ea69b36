// Entry points of attention over the paged cache: argument checks, workspace, choice of kernel.
#include "stwq_paged.cuh"
#include "stwq_pattn.cuh"

namespace {

constexpr int kFewRows = 16;                 // rows per key head and request that the few-row kernel takes
constexpr int kMaxB = 4096;                  // requests per call (both kernels keep a prefix sum over them in shared memory)

int ensure(stwq_ctx* ctx, int B, int Hkv, int d, cudaStream_t st)
{
    const size_t few = stwq_pattn_few_part_bytes(ctx, B, Hkv, d), tiled = stwq_pattn_tiled_part_bytes(ctx, d);
    int rc = stwq_ensure_ws(ctx, &ctx->ws_pattn, &ctx->ws_pattn_bytes, tiled + few, st, 0);        // the two kernels may overlap
    if (rc != STWQ_OK) return rc;
    // arrival counters: zero when allocated, and every call leaves them at zero
    const size_t n = (size_t)ctx->sm_count + (size_t)B * (size_t)Hkv;
    return stwq_ensure_ws(ctx, &ctx->ws_pcnt, &ctx->ws_pcnt_bytes, n * 4, st, n * 4);
}

int check_sizes(int B, int Hq, int Hkv, int d)
{
    if (B <= 0 || B > kMaxB || Hq <= 0 || Hkv <= 0 || Hq > (1 << 16) || Hq % Hkv != 0 || d <= 0 || d > 128) return STWQ_ERR_DIM;
    return (d & 15) != 0 ? STWQ_ERR_ALIGN : STWQ_OK;
}

}  // namespace

extern "C" {

int stwq_reserve_paged_attention(stwq_ctx* ctx, int B, int Hq, int Hkv, int d)
{
    if (!ctx) return STWQ_ERR_NULL;
    const int rc = check_sizes(B, Hq, Hkv, d);
    if (rc != STWQ_OK) return rc;
    StwqDevGuard g(ctx->device);
    return ensure(ctx, B, Hkv, d, nullptr);
}

int paged_attention(stwq_ctx* ctx, const void* Q, int64_t q_ts, int64_t q_hs, const int32_t* cu_new, int64_t T, int max_new, int B,
                    int Hq, int Hkv, int d, const int32_t* block_table, int W, const int32_t* kv_lens, const void* Kp, const void* Vp,
                    int n_pages, int page_size, int kv_dtype, const float* s_k, int P, const float* s_v, float scale, int causal,
                    int out_dtype, void* O, int64_t o_ts, int64_t o_hs, void* stream)
{
    if (!ctx || !Q || !cu_new || !block_table || !kv_lens || !Kp || !Vp || !O) return STWQ_ERR_NULL;
    int rc = check_sizes(B, Hq, Hkv, d);
    if (rc != STWQ_OK) return rc;
    if (T <= 0 || T > 0x7fffffff || max_new <= 0 || W <= 0 || n_pages <= 0 || page_size <= 0 || (int64_t)W * page_size > 0x7ffffe00) return STWQ_ERR_DIM;
    if (kv_dtype != STWQ_KV_BF16 && kv_dtype != STWQ_KV_INT8) return STWQ_ERR_BITS;
    if (out_dtype != STWQ_OUT_F32 && out_dtype != STWQ_OUT_BF16) return STWQ_ERR_BITS;
    const bool i8 = kv_dtype == STWQ_KV_INT8;
    if (i8 && (!s_k || !s_v)) return STWQ_ERR_NULL;
    if (i8 && P <= 0) return STWQ_ERR_DIM;
    if (!(scale > 0.0f) || !(scale <= 3.0e38f)) return STWQ_ERR_DIM;
    const int e16 = out_dtype == STWQ_OUT_F32 ? 4 : 8;
    if ((page_size & 15) != 0 || !stwq_aligned16(Q) || !stwq_aligned16(Kp) || !stwq_aligned16(Vp) || !stwq_aligned16(O) || !stwq_aligned16(s_v))
        return STWQ_ERR_ALIGN;
    if (q_ts < 0 || q_hs < 0 || !stwq_disjoint(T, Hq, d, o_ts, o_hs)) return STWQ_ERR_DIM;
    if (q_ts % 8 != 0 || q_hs % 8 != 0 || o_ts % e16 != 0 || o_hs % e16 != 0) return STWQ_ERR_ALIGN;
    if ((int64_t)n_pages * Hkv * (page_size / 16) > 0x7fffffffll) return STWQ_ERR_DIM;    // 16-key blocks of a pool, counted in 32 bits
    const int g = Hq / Hkv;
    if (max_new > T) max_new = (int)T;
    if ((int64_t)max_new * g > 0x3fffff00) return STWQ_ERR_DIM;
    StwqDevGuard guard(ctx->device);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    rc = ensure(ctx, B, Hkv, d, st);
    if (rc != STWQ_OK) return rc;
    PaParams p = {};
    p.Q = Q; p.q_ts = q_ts; p.q_hs = q_hs;
    p.cu = cu_new; p.kv = kv_lens; p.table = block_table;
    p.T = T; p.B = B; p.W = W; p.Hq = Hq; p.Hkv = Hkv; p.g = g; p.d = d; p.S = page_size; p.n_pages = n_pages; p.P = P;
    p.causal = causal ? 1 : 0; p.out_bf16 = out_dtype == STWQ_OUT_BF16; p.max_new = max_new;
    p.Kp = Kp; p.Vp = Vp; p.s_k = i8 ? s_k : nullptr; p.s_v = i8 ? s_v : nullptr; p.scale = scale;
    p.O = O; p.o_ts = o_ts; p.o_hs = o_hs;
    p.part = static_cast<float*>(ctx->ws_pattn);
    p.counters = static_cast<uint32_t*>(ctx->ws_pcnt);
    p.status = ctx->d_status;
    p.wait_limit_ns = (unsigned long long)ctx->wait_limit_ms * 1000000ull;
    // Requests of up to 16 rows per key head (decoding ones) go to the kernel that streams the cache, the others to the
    // tiled one; a step that may hold both runs both, the second as a programmatic dependent of the first. Where all units of
    // the step together cannot outnumber the SMs, the tiled kernel cuts every unit's keys over the idle ones and takes the
    // decoding requests too (2 requests of up to 20 tokens: 15 against 23 us with both kernels; 4 of up to 8 tokens
    // behind up to 4000, 4 heads per key head: 29 against 56). With more units than SMs it does not cut keys, and a
    // long decoding request would wait for one CTA. Steps with more than 16 query heads per key head have no other kernel and do
    // wait: 200 requests of up to 512 keys, 32 heads over one of 128, take 29 us, and 407 us when one of them has 32768 keys (16
    // heads, in the few-row kernel: 41 and 68 us).
    const bool tiled = (int64_t)max_new * g > kFewRows;
    const bool alone = tiled && (g > kFewRows || (int64_t)Hkv * ((T * g + 127) / 128 + B) <= ctx->sm_count);
    p.few_max = alone ? 0 : kFewRows;
    if (tiled) {
        rc = stwq_launch_pattn_tiled(ctx, p, st);
        if (rc != STWQ_OK || alone) return rc;
    }
    p.part = reinterpret_cast<float*>(static_cast<char*>(ctx->ws_pattn) + stwq_pattn_tiled_part_bytes(ctx, d));
    p.counters += ctx->sm_count;
    return stwq_launch_pattn_few(ctx, p, tiled, st);
}

}  // extern "C"
