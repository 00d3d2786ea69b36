"""The serving calls together, as a decoder's steps use them: page plan, quantized qkv linear, cache append, attention, head
linear, sampling; captured into a graph and replayed; on several streams; with pools beyond 32-bit offsets; and their refusals at
the C boundary."""
import numpy as np
import pytest

from test_gpu_paged_attention import call, check, make
from test_gpu_serving import check_close, head_ref, plan_ref, rope_cs, sample_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch

    import paper_2601_21238_b200 as pk
    from paper_2601_21238_b200 import build as pkbuild
    pkbuild.build()
    ctx = pk.Context(0)

    class G:
        pass
    g = G()
    g.torch, g.ctx, g.pk, g.dev = torch, ctx, pk, torch.device("cuda:0")
    g.T = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(g.dev)
    yield g
    ctx.close()


def linear(gpu, r, K, N):
    """A quantized layer: folded weights and unit-ish static scales."""
    torch = gpu.torch
    W = gpu.T((r.standard_normal((N, K)) * 0.05).astype(np.float32))
    Wq, s_w = torch.empty((N, K), dtype=torch.int8, device=gpu.dev), torch.empty(N, device=gpu.dev)
    gpu.ctx.gps_fold(W, None, 8, Wq, s_w)
    return Wq, s_w


@pytest.mark.parametrize("int8", [False, True])
def test_steps_of_a_batch_with_requests_joining(gpu, int8):
    torch, pk = gpu.torch, gpu.pk
    r = np.random.default_rng(17)
    K, Hq, Hkv, d, S, P, V, NP, W, cap = 256, 4, 2, 64, 16, 256, 500, 60, 8, 96
    Wqkv, sw1 = linear(gpu, r, K, (Hq + 2 * Hkv) * d)
    Whead, sw2 = linear(gpu, r, Hq * d, V)
    s_tok = gpu.T(r.uniform(0.02, 0.04, P).astype(np.float32))
    wq, wk = r.uniform(0.5, 1.5, d).astype(np.float32), r.uniform(0.5, 1.5, d).astype(np.float32)
    cs = rope_cs(r, P, d)
    Kp = torch.full((NP, Hkv, S, d), 7, dtype=torch.int8, device=gpu.dev) if int8 else torch.full((NP, Hkv, S, d), float("nan"), dtype=torch.bfloat16, device=gpu.dev)
    Vp = Kp.clone()
    s_k, s_v = r.uniform(0.02, 0.04, P).astype(np.float32), r.uniform(0.02, 0.04, (Hkv, d)).astype(np.float32)
    sk_d, sv_d = (gpu.T(s_k), gpu.T(s_v)) if int8 else (None, None)
    pool, table, cached = r.permutation(NP).astype(np.int32), np.full((4, W), -1, np.int32), np.zeros(4, np.int64)
    table_d = gpu.T(table)
    e = lambda *s: torch.full(s, -7, dtype=torch.int32, device=gpu.dev)  # noqa: E731
    for step, new in enumerate(([40, 5, 17, 0], [1, 1, 1, 0], [1, 1, 1, 33], [1, 0, 1, 1], [1, 1, 1, 1])):
        new = np.array(new)
        n = int(new.sum())
        cu, kv, slots, pos, used = e(5), e(4), e(cap), e(cap), e(1)
        gpu.ctx.page_plan(gpu.T(cached.astype(np.int32)), gpu.T(new.astype(np.int32)), gpu.T(pool), S, table_d, cu, kv, slots, pos, used)
        table, cu_h, kv_h, slots_h, pos_h, taken = plan_ref(cached, new, pool, S, table, cap)
        for a, b in zip((table_d, cu, kv, slots, pos), (table, cu_h, kv_h, slots_h, pos_h)):
            np.testing.assert_array_equal(a.cpu().numpy(), b)
        assert used.item() == taken
        pool = pool[taken:]
        # the step's rows are padded to the capacity, as the plan's lists are: positions of padding rows are 0 for the linear
        X = gpu.T(r.standard_normal((cap, K)).astype(np.float32))
        qkv = torch.empty((cap, (Hq + 2 * Hkv) * d), dtype=torch.bfloat16, device=gpu.dev)
        gpu.ctx.qlinear(X, pos.clamp(min=0), Wqkv, sw1, s_tok, None, None, 8, pk.ACT_NONE, pk.OUT_BF16, qkv)
        Q = torch.full((cap, Hq, d), 7.0, dtype=torch.bfloat16, device=gpu.dev)
        gpu.ctx.kv_append_paged(qkv, pos, slots, Hq, Hkv, gpu.T(wq), gpu.T(wk), pk.NORM_RMS, 1e-6, gpu.T(cs), pk.ROPE_HALF, sk_d, sv_d, 8, Q, Kp, Vp)
        x = qkv[:n].float().cpu().numpy().astype(np.float64).reshape(n, -1, d)
        qr, qm = head_ref(x[:, :Hq], wq, 1, 1e-6, cs[pos_h[:n]].astype(np.float64), d, 0)
        check_close(Q[:n].float().cpu().numpy(), qr, qm, True)
        assert (Q[n:] == 7.0).all()
        # attention of the step, against the cache as it now is
        s = dict(Q=Q, cu=cu_h, kv=kv_h, table=table, S=S, T=cap, new=new, d=d, Hq=Hq, Hkv=Hkv, scale=np.float32(1 / np.sqrt(d)), Kp=Kp, Vp=Vp,
                 s_k=s_k if int8 else None, s_v=s_v if int8 else None, K=Kp.float().cpu().numpy().astype(np.float64),
                 V=Vp.float().cpu().numpy().astype(np.float64))
        O = call(gpu, s, True, False)
        assert gpu.ctx.stwq_device_status() == 0
        check(gpu, s, True, False, O)
        # the last token of each request that had any gives a logits row
        last = torch.from_numpy(cu_h[1:][new > 0].astype(np.int64) - 1).to(gpu.dev)
        B = len(last)
        logits = torch.empty((B, V), device=gpu.dev)
        gpu.ctx.qlinear(O.reshape(cap, -1)[last].contiguous(), pos[last].contiguous(), Whead, sw2, s_tok, None, None, 8, pk.ACT_NONE, pk.OUT_F32, logits)
        u = r.uniform(0, 1, B).astype(np.float32)
        tok, pr, kept = e(B), torch.empty(B, device=gpu.dev), e(B)
        f = lambda v: torch.full((B,), v, device=gpu.dev)  # noqa: E731
        gpu.ctx.sample_tokens(logits, f(0.7), torch.full((B,), 40, dtype=torch.int32, device=gpu.dev), f(0.9), f(0.01), gpu.T(u), tok, pr, kept)
        for i in range(B):
            want = sample_ref(logits[i].cpu().numpy(), np.float32(0.7), 40, np.float32(0.9), np.float32(0.01), u[i])
            assert (tok[i].item(), kept[i].item()) == (want[0], want[2])
        assert gpu.ctx.stwq_device_status() == 0
        cached = cached + new


def test_normed_heads_feed_the_contiguous_quantized_cache(gpu):
    """qk_norm_rope in head-major fp32 is what kv_append and qattention take."""
    torch, pk = gpu.torch, gpu.pk
    r = np.random.default_rng(23)
    T, H, d, P = 40, 3, 64, 64
    X = gpu.T(r.standard_normal((T, 3 * H * d)).astype(np.float32))
    pos, cs = gpu.T(np.arange(T, dtype=np.int32)), gpu.T(rope_cs(r, P, d))
    Q, Kn = torch.empty((H, T, d), device=gpu.dev), torch.empty((H, T, d), device=gpu.dev)
    gpu.ctx.qk_norm_rope(X, pos, H, H, None, None, pk.NORM_RMS, 1e-6, cs, pk.ROPE_HALF, Q.transpose(0, 1), Kn.transpose(0, 1))
    Vn = X.view(T, 3 * H, d)[:, 2 * H:].transpose(0, 1).contiguous()
    s_q = torch.full((P,), 4.5 / 127, device=gpu.dev)
    s_v = torch.full((d,), 4.5 / 127, device=gpu.dev)
    Kc, Vt = torch.zeros((H, 48, d), dtype=torch.int8, device=gpu.dev), torch.zeros((H, d, 48), dtype=torch.int8, device=gpu.dev)
    gpu.ctx.kv_append(Kn, Vn, 0, s_q, s_v, 8, Kc, Vt)
    O = torch.empty((H, T, d), device=gpu.dev)
    gpu.ctx.qattention(Q, pos, T, Kc, Vt, s_q, s_q[:T].contiguous() / 8, s_v, 8, True, pk.OUT_F32, O)
    assert gpu.ctx.stwq_device_status() == 0
    q, k, v = Q.double(), Kn.double(), Vn.double()
    x = (q @ k.transpose(1, 2)) / 8 + torch.full((T, T), float("-inf"), device=gpu.dev, dtype=torch.float64).triu(1)
    want = torch.softmax(x, -1) @ v
    # 8-bit operands: queries and keys to a step of 4.5 / 127 each, probabilities to 1 / 255, values to 4.5 / 127
    assert (O.double() - want).abs().max() < 0.25 and ((O.double() - want).norm() / want.norm()) < 0.05


@pytest.mark.parametrize("max_new,int8", [(1, False), (1, True), (40, False), (40, True)])
def test_a_captured_step_follows_the_lengths_on_the_device(gpu, max_new, int8):
    torch, pk = gpu.torch, gpu.pk
    r = np.random.default_rng(3)
    B, Hq, Hkv, d, S, W, NP = 5, 8, 2, 64, 16, 40, 5 * 40 + 1
    T = B * max_new
    ctx = pk.Context(0)
    try:
        ctx.stwq_reserve_paged_attention(B, Hq, Hkv, d)
        i32 = lambda a: gpu.T(np.asarray(a, np.int32))  # noqa: E731
        cached, new, free = i32([0] * B), i32([1] * B), i32(np.arange(1, NP))
        table = torch.zeros((B, W), dtype=torch.int32, device=gpu.dev)
        mk = lambda n: torch.zeros(n, dtype=torch.int32, device=gpu.dev)  # noqa: E731
        cu, kv, slots, pos, used, tok = mk(B + 1), mk(B), mk(T), mk(T), mk(1), mk(T)
        X = torch.randn((T, (Hq + 2 * Hkv) * d), device=gpu.dev).to(torch.bfloat16)
        cs = gpu.T(rope_cs(r, W * S, d))
        kind = torch.int8 if int8 else torch.bfloat16
        Kp, Vp = torch.zeros((NP, Hkv, S, d), dtype=kind, device=gpu.dev), torch.zeros((NP, Hkv, S, d), dtype=kind, device=gpu.dev)
        sk, sv = (torch.full((W * S,), 0.03, device=gpu.dev), torch.full((Hkv, d), 0.03, device=gpu.dev)) if int8 else (None, None)
        Q, O = torch.zeros((T, Hq, d), dtype=torch.bfloat16, device=gpu.dev), torch.zeros((T, Hq, d), device=gpu.dev)
        u = torch.rand(T, device=gpu.dev)

        def step():
            ctx.page_plan(cached, new, free, S, table, cu, kv, slots, pos, used)
            ctx.kv_append_paged(X, pos, slots, Hq, Hkv, None, None, pk.NORM_RMS, 1e-6, cs, pk.ROPE_PAIRS, sk, sv, 8, Q, Kp, Vp)
            ctx.paged_attention(Q, cu, max_new, table, kv, Kp, Vp, sk, sv, 0.125, True, pk.OUT_F32, O)
            ctx.sample_tokens(O.view(T, Hq * d), None, None, None, None, u, tok)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
        for lens in ([600, 3, 17, 0, 31], [0, 0, 0, 0, 0], [39, 599, 1, 16, 15]):
            c = np.array(lens) * (1 if max_new == 1 else 0.9)
            cached.copy_(i32(c.astype(np.int32)))
            new.copy_(i32(r.integers(0, max_new + 1, B)))
            table.copy_(torch.arange(1, NP, device=gpu.dev, dtype=torch.int32).flip(0).view(B, W))
            O.fill_(5.0)
            g.replay()
            torch.cuda.synchronize()
            a = [t.clone() for t in (O, tok, table, cu, Kp)]
            O.fill_(5.0)
            step()
            torch.cuda.synchronize()
            for x, y in zip(a, (O, tok, table, cu, Kp)):
                assert torch.equal(x, y)
        assert ctx.stwq_device_status() == 0
    finally:
        ctx.close()


def test_two_contexts_on_two_streams_and_growth_is_refused_under_capture(gpu):
    torch, pk = gpu.torch, gpu.pk
    cases = [make(gpu, [1] * 9, list(range(0, 1800, 200)), 8, 2, 128, 16, False, 1), make(gpu, [300, 20], [700, 2000], 4, 4, 64, 32, True, 2)]
    alone = [call(gpu, s, True, True) for s in cases]
    ctxs, streams = [pk.Context(0), pk.Context(0)], [torch.cuda.Stream(), torch.cuda.Stream()]
    try:
        args = []
        for s, O in zip(cases, alone):
            t = lambda a: None if a is None else gpu.T(a)  # noqa: E731
            args.append([s["Q"], gpu.T(s["cu"]), int(s["new"].max()), gpu.T(s["table"]), gpu.T(s["kv"]), s["Kp"], s["Vp"], t(s["s_k"]), t(s["s_v"]),
                         float(s["scale"]), True, pk.OUT_BF16])
        outs = [[torch.zeros_like(O) for _ in range(20)] for O in alone]
        torch.cuda.synchronize()
        for k in range(20):
            for c, st, a, o in zip(ctxs, streams, args, outs):
                c.paged_attention(*a, o[k], stream=st)
        torch.cuda.synchronize()
        for O, o in zip(alone, outs):
            assert all(torch.equal(O, x) for x in o)
        fresh = pk.Context(0)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            with pytest.raises(pk.StwqError) as e:
                fresh.paged_attention(*args[0], outs[0][0])
        assert e.value.code == -11
        fresh.close()
    finally:
        for c in ctxs:
            c.close()


def test_pools_beyond_32_bit_offsets(gpu):
    """Pages on both sides of 2^31 and 2^32 elements, appended to and read by both kernels."""
    torch, pk = gpu.torch, gpu.pk
    Hkv, d, S = 8, 128, 64
    NP = (1 << 32) // (Hkv * S * d) + 3
    Kp, Vp = (torch.empty((NP, Hkv, S, d), dtype=torch.bfloat16, device=gpu.dev) for _ in range(2))
    small_K, small_V = (torch.zeros((4, Hkv, S, d), dtype=torch.bfloat16, device=gpu.dev) for _ in range(2))
    far = torch.tensor([NP - 1, NP // 2 + 1, 5, NP - 2], dtype=torch.int32, device=gpu.dev)
    near = torch.arange(4, dtype=torch.int32, device=gpu.dev)
    n = 200
    X = torch.randn((n, 3 * Hkv * d), device=gpu.dev).to(torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device=gpu.dev)
    slot = lambda pages: (pages.long()[pos.long() // S] * S + pos % S).to(torch.int32)  # noqa: E731
    outs = []
    for K, V, pages in ((Kp, Vp, far), (small_K, small_V, near)):
        Q = torch.empty((n, Hkv, d), dtype=torch.bfloat16, device=gpu.dev)
        gpu.ctx.kv_append_paged(X, pos, slot(pages), Hkv, Hkv, None, None, pk.NORM_RMS, 1e-6, None, pk.ROPE_HALF, None, None, 8, Q, K, V)
        kv = torch.tensor([n], dtype=torch.int32, device=gpu.dev)
        for q0 in (0, n - 3):                                    # 200 rows: tiled; 3 rows: few
            O = torch.empty((n - q0, Hkv, d), dtype=torch.bfloat16, device=gpu.dev)
            cu = torch.tensor([0, n - q0], dtype=torch.int32, device=gpu.dev)
            gpu.ctx.paged_attention(Q[q0:], cu, n - q0, pages[None].contiguous(), kv, K, V, None, None, 0.09, True, pk.OUT_BF16, O)
            outs.append(O)
    assert gpu.ctx.stwq_device_status() == 0
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3]) and torch.equal(small_K[:4, :, :8], Kp[far.long()][:, :, :8])
    del Kp, Vp
    torch.cuda.empty_cache()


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("n,L", [(5, 3), (40, 33), (300, 10), (2, 0), (150, 0)])
def test_more_new_tokens_than_keys_leaves_the_first_rows_without_any(gpu, n, L, int8):
    s = make(gpu, [n, 4], [0, 50], 2, 1, 64, 16, int8, 9)
    s["kv"] = np.array([L, 54], np.int32)                        # the request's cache holds fewer keys than it has new tokens
    for bf16 in (True, False):
        O = call(gpu, s, True, bf16)
        assert gpu.ctx.stwq_device_status() == 0
        check(gpu, s, True, bf16, O)
        assert (O[: max(0, n - L)] == 0).all()


def test_full_gpu_of_tiles_over_codes_against_fp64_on_samples(gpu):
    """Every SM several units deep (what a step of 32 images runs), sampled heads against fp64."""
    torch = gpu.torch
    s = make(gpu, [256] * 32, [424] * 32, 30, 30, 64, 32, True, 77)
    O = call(gpu, s, False, True)
    assert gpu.ctx.stwq_device_status() == 0
    for b in range(0, 32, 3):
        at = torch.from_numpy(s["table"][b].astype(np.int64)).to(gpu.dev)
        k = s["Kp"][at].transpose(1, 2).reshape(-1, 30, 64)[:680].double() * gpu.T(s["s_k"][:680])[:, None, None]
        v = s["Vp"][at].transpose(1, 2).reshape(-1, 30, 64)[:680].double() * gpu.T(s["s_v"])
        q = s["Q"][b * 256:(b + 1) * 256].double()
        p = torch.softmax(torch.einsum("nhd,lhd->hnl", q, k) / 8, -1)
        want = torch.einsum("hnl,lhd->nhd", p, v)
        mag = torch.einsum("hnl,lhd->nhd", p, v.abs())
        # fp16 probabilities 2^-11 of the sum of magnitudes, scores' and sums' roundings below that again; the store 2^-8
        assert ((O[b * 256:(b + 1) * 256].double() - want).abs() <= mag * 2.0 ** -10 + want.abs() * 2.0 ** -8 + 1e-6).all(), b


def test_bad_lengths_and_pages_are_reported(gpu):
    ERR = -12
    for new, cached in (([1, 1], [40, 7]), ([50, 3], [40, 7])):
        s = make(gpu, new, cached, 2, 1, 64, 16, False, 5)
        good = call(gpu, s, True, True)
        assert gpu.ctx.stwq_device_status() == 0
        NP = s["Kp"].shape[0]
        for bad in (NP, -3, 2 ** 31 - 1):                        # a needed page id outside the pool: page 0 is read instead
            t = dict(s, table=s["table"].copy())
            t["table"][1, 0] = bad
            O = call(gpu, t, True, True)
            assert gpu.ctx.stwq_device_status() == ERR and gpu.ctx.stwq_device_status() == 0
            assert gpu.torch.equal(O[: s["cu"][1]], good[: s["cu"][1]])
        for key, val in (("kv", [10 ** 6, 8]), ("kv", [-5, 8]), ("cu", [0, -3, 4]), ("cu", [0, 10 ** 8, 4])):
            call(gpu, dict(s, **{key: np.array(val, np.int32)}), True, True)
            assert gpu.ctx.stwq_device_status() == ERR


def test_the_c_boundary_refuses_bad_sizes_and_writes_nothing(gpu):
    import ctypes as C
    torch, pk = gpu.torch, gpu.pk
    L, h = gpu.ctx.lib, gpu.ctx.handle
    buf = torch.zeros(1 << 20, device=gpu.dev)
    out = torch.full((1 << 16,), 3.0, device=gpu.dev)
    p, o = buf.data_ptr(), out.data_ptr()
    st = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    DIM, ALIGN, BITS, NULL = -2, -3, -4, -1

    def bad(fn, names, base, changes):
        for ch, code in changes:
            a = dict(base, **ch)
            assert fn(h, *[a[n] for n in names], st) == code, ch
    names = "cached new B free F S table W cu kv slots pos T used".split()
    bad(L.page_plan, names, dict(cached=p, new=p, B=2, free=p, F=4, S=16, table=o, W=4, cu=o, kv=o, slots=o, pos=o, T=8, used=o),
        [({"cached": None}, NULL), ({"used": None}, NULL), ({"free": None}, NULL), ({"B": 0}, DIM), ({"B": 4097}, DIM), ({"F": -1}, DIM), ({"S": 0}, DIM), ({"W": 0}, DIM),
         ({"T": 0}, DIM), ({"W": 1 << 20, "S": 1 << 12}, DIM)])
    names = "X ld xt pos T Hq Hkv d wq nq wk nk norm eps cs rot rope P Q qt qh K kt kh od".split()
    base = dict(X=p, ld=4 * 64, xt=1, pos=p, T=4, Hq=2, Hkv=1, d=64, wq=p, nq=1, wk=p, nk=1, norm=1, eps=1e-6, cs=p, rot=64, rope=0, P=9, Q=o, qt=128, qh=64, K=o,
                kt=64, kh=64, od=1)
    common = [({"X": None}, NULL), ({"pos": None}, NULL), ({"Q": None}, NULL), ({"cs": None}, NULL), ({"wq": None}, NULL), ({"T": 0}, DIM), ({"Hq": 0}, DIM),
              ({"d": 0}, DIM), ({"d": 272}, DIM), ({"d": 40, "rot": 32}, ALIGN), ({"rot": 80}, DIM), ({"rot": 24}, ALIGN), ({"ld": 64}, DIM), ({"ld": 260}, ALIGN), ({"xt": 2}, BITS),
              ({"norm": 3}, BITS), ({"rope": 2}, BITS), ({"eps": -1.0}, DIM), ({"eps": float("nan")}, DIM), ({"nq": 3}, DIM), ({"P": 0}, DIM), ({"qt": 64}, DIM), ({"qh": 32}, DIM), ({"qt": 0}, DIM),
              ({"qt": 132}, ALIGN), ({"X": p + 2}, ALIGN), ({"cs": p + 4}, ALIGN), ({"wk": p + 4}, ALIGN)]
    bad(L.qk_norm_rope, names, base, common + [({"K": None}, NULL), ({"kt": 32}, DIM), ({"K": o + 8}, ALIGN), ({"od": 2}, BITS)])
    names = "X ld xt pos slots T Hq Hkv d wq nq wk nk norm eps cs rot rope P sk sv bits Q qt qh Kp Vp NP S kvt".split()
    base = dict(base, slots=p, sk=p, sv=p, bits=8, Kp=o, Vp=o, NP=2, S=16, kvt=1)
    bad(L.kv_append_paged, names, base, common + [({"slots": None}, NULL), ({"Kp": None}, NULL), ({"sk": None}, NULL), ({"sv": None}, NULL), ({"bits": 4}, BITS), ({"kvt": 2}, BITS),
                                                  ({"NP": 0}, DIM), ({"S": 0}, DIM), ({"Vp": o + 8}, ALIGN), ({"sv": p + 4}, ALIGN)])
    names = "Q qt qh cu T mn B Hq Hkv d tab W kv Kp Vp NP S kvt sk P sv scale causal od O ot oh".split()
    base = dict(Q=p, qt=128, qh=64, cu=p, T=4, mn=4, B=2, Hq=2, Hkv=1, d=64, tab=p, W=2, kv=p, Kp=p, Vp=p, NP=2, S=16, kvt=1, sk=p, P=32, sv=p, scale=0.1, causal=1, od=1, O=o,
                ot=128, oh=64)
    bad(L.paged_attention, names, base,
        [({"Q": None}, NULL), ({"O": None}, NULL), ({"sk": None}, NULL), ({"sv": None}, NULL), ({"B": 0}, DIM), ({"B": 4097}, DIM), ({"T": 0}, DIM), ({"mn": 0}, DIM), ({"Hq": 3, "Hkv": 2}, DIM),
         ({"d": 144}, DIM), ({"d": 40}, ALIGN), ({"S": 8}, ALIGN), ({"S": 0}, DIM), ({"W": 0}, DIM), ({"NP": 0}, DIM), ({"kvt": 5}, BITS), ({"od": 2}, BITS), ({"scale": 0.0}, DIM), ({"scale": -1.0}, DIM),
         ({"scale": float("nan")}, DIM), ({"scale": float("inf")}, DIM), ({"P": 0}, DIM), ({"ot": 64}, DIM), ({"ot": 132}, ALIGN), ({"qt": 4}, ALIGN), ({"qt": -128}, DIM), ({"Kp": p + 8}, ALIGN), ({"O": o + 8}, ALIGN),
         ({"W": 1 << 30}, DIM), ({"NP": 1 << 30, "S": 64}, DIM)])
    names = "X xt ld B V t k p m u tok pr kept".split()
    base = dict(X=p, xt=0, ld=100, B=2, V=100, t=p, k=p, p=p, m=p, u=p, tok=o, pr=o, kept=o)
    bad(L.sample_tokens, names, base, [({"X": None}, NULL), ({"u": None}, NULL), ({"tok": None}, NULL), ({"B": 0}, DIM), ({"V": 0}, DIM), ({"V": 360449, "ld": 400000}, DIM), ({"ld": 99}, DIM),
                                       ({"xt": 2}, BITS), ({"X": p + 2}, ALIGN)])
    assert L.stwq_reserve_paged_attention(h, 0, 2, 1, 64) == DIM and L.stwq_reserve_paged_attention(h, 2, 2, 1, 40) == ALIGN
    torch.cuda.synchronize()
    assert (out == 3.0).all() and gpu.ctx.stwq_device_status() == 0


def test_first_call_of_a_context_beside_a_busy_default_stream(gpu):
    """The workspace of a fresh context, reserved from the host and used on a stream that is not ordered behind the default
    one: its counters have to be zero by then, whatever the memory held and however busy the default stream is."""
    torch, pk = gpu.torch, gpu.pk
    s = make(gpu, [1] * 9, list(range(0, 1800, 200)), 8, 2, 128, 16, False, 3)
    want = call(gpu, s, True, True)
    args = [s["Q"], gpu.T(s["cu"]), 1, gpu.T(s["table"]), gpu.T(s["kv"]), s["Kp"], s["Vp"], None, None, float(s["scale"]), True, pk.OUT_BF16]
    side = torch.cuda.Stream()
    for reserve in (True, False):
        ctx = pk.Context(0)
        try:
            O = torch.zeros_like(want)
            dirty = [torch.full((1 << 18,), 3, dtype=torch.int32, device=gpu.dev) for _ in range(32)]
            torch.cuda.synchronize()
            del dirty
            torch.cuda.empty_cache()
            torch.cuda._sleep(50_000_000)                           # the default stream is busy for some 30 ms
            if reserve:
                ctx.stwq_reserve_paged_attention(9, 8, 2, 128)
            for _ in range(2):
                ctx.paged_attention(*args, O, stream=side)
                side.synchronize()
                assert torch.equal(O, want)
            torch.cuda.synchronize()
            assert ctx.stwq_device_status() == 0
        finally:
            ctx.close()


def test_a_plan_in_place_is_refused(gpu):
    torch, pk = gpu.torch, gpu.pk
    z = lambda *n: torch.zeros(n, dtype=torch.int32, device=gpu.dev)  # noqa: E731
    cached, new, pages = z(4), z(4) + 2, torch.arange(12, dtype=torch.int32, device=gpu.dev)
    outs = dict(block_table=z(4, 3), cu_new=z(5), kv_lens=z(4), slot_map=z(8), pos_ids=z(8), pages_used=z(1))
    for name, alias in (("kv_lens", cached), ("kv_lens", new), ("slot_map", pages[4:]), ("pages_used", new[3:]), ("block_table", pages.view(4, 3))):
        with pytest.raises(pk.StwqError) as e:
            gpu.ctx.page_plan(cached, new, pages, 16, **{**outs, name: alias})
        assert e.value.code == pk.binding.ERR_ALIGN, name
    # neighbours, and an empty list that begins inside an output, do not overlap
    both = z(8)
    gpu.ctx.page_plan(both[:4], new, pages, 16, **{**outs, "kv_lens": both[4:]})
    assert both.tolist() == [0] * 4 + [2] * 4 and outs["slot_map"].tolist() == [0, 1, 16, 17, 32, 33, 48, 49]
    gpu.ctx.page_plan(cached, z(4), outs["slot_map"][3:3], 16, **outs)
    assert outs["pages_used"].item() == 0 and outs["slot_map"].tolist() == [-1] * 8 and gpu.ctx.stwq_device_status() == 0
