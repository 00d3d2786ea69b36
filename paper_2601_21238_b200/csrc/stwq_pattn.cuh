// Attention of new tokens over a paged KV cache: what the two kernels and the entry point share.
#pragma once

#include "stwq_internal.cuh"

struct PaParams {
    const void* Q;                 // bf16
    int64_t q_ts, q_hs;            // elements between tokens / heads
    const int32_t *cu, *kv, *table;
    int64_t T;
    int B, W, Hq, Hkv, g, d, S, n_pages, P, causal, out_bf16, max_new;
    const void *Kp, *Vp;
    const float *s_k, *s_v;
    float scale;
    void* O;
    int64_t o_ts, o_hs;
    float* part;                   // workspace: partial results of split units
    uint32_t* counters;            // workspace: arrivals per unit, zero between calls
    uint32_t* status;
    unsigned long long wait_limit_ns;
    int few_max;                   // the tiled kernel leaves requests with at most this many rows per key head to the other one
};

// Request b's rows and keys, clamped to what the caller's sizes allow (bad != 0: something was out of range).
struct PaReq {
    int t0, n, kv;
};
__device__ __forceinline__ PaReq pa_request(const PaParams& p, int b, bool& bad)
{
    const long long T = p.T;
    const long long c0 = p.cu[b], c1 = p.cu[b + 1];
    const long long a0 = min(max(c0, 0ll), T), a1 = min(max(c1, a0), T);
    long long n = a1 - a0;
    if (n > p.max_new) n = p.max_new;
    const long long cap = (long long)p.W * p.S;
    long long kv = p.kv[b];
    long long k = min(max(kv, 0ll), cap);
    if (p.s_k != nullptr) k = min(k, (long long)p.P);
    bad |= c0 != a0 || c1 - c0 != n || k != kv;
    return {(int)a0, (int)n, (int)k};
}

constexpr float kPaLog2e = 1.4426950408889634f;

// dependent: launched right behind the tiled kernel of the same call, which it may overlap
int stwq_launch_pattn_few(stwq_ctx* ctx, const PaParams& p, bool dependent, cudaStream_t st);
int stwq_launch_pattn_tiled(stwq_ctx* ctx, const PaParams& p, cudaStream_t st);
// bytes of partial results that the launch of a call of these sizes may need
size_t stwq_pattn_few_part_bytes(const stwq_ctx* ctx, int B, int Hkv, int d);
size_t stwq_pattn_tiled_part_bytes(const stwq_ctx* ctx, int d);
