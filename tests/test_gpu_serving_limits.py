"""The serving calls at the limits that their documentation names: lengths next to 2^31, the largest batches, values that are no
numbers."""
import subprocess
import sys

import numpy as np
import pytest

from conftest import ROOT
from test_gpu_paged_attention import call, check, make
from test_gpu_serving import rope_cs, run_plan, run_sample

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


ERR_PAGES, MAX = -12, 2 ** 31 - 1


@pytest.mark.parametrize("S,W,cached,new,table", [
    (715827882, 3, 2147483640, 100, [1, 0, 2]),                  # the row ends after 6 tokens, positions pass 2^31 after 8
    (16, 134217727, 2147483632 - 3, 40, None),                   # the same with a long row
    (MAX, 1, 2 ** 30 + 5, 3, [0]),                               # cached + page size - 1 is beyond 2^31
    (MAX, 1, MAX, 2, [0]), (2 ** 30, 1, 0, 7, [-9])])
def test_page_plan_next_to_2_31(gpu, S, W, cached, new, table):
    torch = gpu.torch
    if table is None:                                            # page 5 everywhere
        row = torch.full((1, W), 5, dtype=torch.int32, device=gpu.dev)
    else:
        row = gpu.T(np.array([table], np.int32))
    e = lambda n: torch.full((n,), -77, dtype=torch.int32, device=gpu.dev)  # noqa: E731
    i32 = lambda *a: gpu.T(np.array(a, np.int32))  # noqa: E731
    cu, kv, slots, pos, used = e(2), e(1), e(new + 2), e(new + 2), e(1)
    gpu.ctx.page_plan(i32(cached), i32(new), i32(1), S, row, cu, kv, slots, pos, used)
    fits = cached + new <= W * S
    assert gpu.ctx.stwq_device_status() == (0 if fits else ERR_PAGES)
    first_new = -(-cached // S)                                  # the first page that has to come from the free list, whose page is 1
    want = []
    for t in range(cached, cached + new):
        page = None if t >= W * S else 1 if t // S >= first_new else 5 if table is None else table[t // S]
        want.append(-1 if page is None or page * S + t % S > MAX else page * S + t % S)
    assert cu.tolist() == [0, new] and kv.item() == min(cached + new, W * S)
    assert slots.tolist() == want + [-1, -1]
    assert pos.tolist() == [min(t, MAX) for t in range(cached, cached + new)] + [-1, -1]
    assert used.item() == -(-min(cached + new, W * S) // S) - first_new
    if table is not None:
        table = [1 if first_new <= i < -(-min(cached + new, W * S) // S) else p for i, p in enumerate(table)]
        assert row.tolist() == [table]


@pytest.mark.parametrize("B", [4084, 4085, 4090, 4095])
def test_page_plan_of_large_batches_in_a_fresh_process(B):
    """The first plan of a process (a larger one before it could have raised the kernel's shared memory limit)."""
    code = f"""
import torch, paper_2601_21238_b200 as pk
z = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")
ctx = pk.Context(0)
slots = z({B})
ctx.page_plan(z({B}), z({B}) + 1, torch.arange({B}, dtype=torch.int32, device="cuda"), 16, z({B}, 1), z({B} + 1), z({B}), slots, z({B}), z(1))
assert ctx.stwq_device_status() == 0
assert torch.equal(slots, 16 * torch.arange({B}, dtype=torch.int32, device="cuda"))
ctx.close()
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 32), (128, 64), (80, 48), (256, 16), (48, 0), (64, 64)])
@pytest.mark.parametrize("pairs", [0, 1])
def test_infinities_beside_the_rotated_channels(gpu, d, rot, pairs, bf16):
    """Channels from rot on are not turned: an Inf or NaN there stays what it is, and changes no other channel."""
    torch, pk = gpu.torch, gpu.pk
    r = np.random.default_rng(d + rot)
    T, Hq, Hkv, P = 9, 5, 2, 20
    pos, cs = gpu.T(r.integers(0, P, T).astype(np.int32)), gpu.T(rope_cs(r, P, rot)) if rot else None
    x = r.standard_normal((T, Hq + 2 * Hkv, d)).astype(np.float32)
    odd = np.zeros(x.shape, bool)
    odd[:, :, rot:] = r.uniform(size=x[:, :, rot:].shape) < 0.2
    y = np.where(odd, r.choice(np.array([np.inf, -np.inf, np.nan], np.float32), x.shape), x)
    outs = []
    for a in (x, y):
        X = gpu.T(a.reshape(T, -1))
        X = X.to(torch.bfloat16) if bf16 else X
        Q, K = torch.full((T, Hq, d), 7.0, device=gpu.dev), torch.full((T, Hkv, d), 7.0, device=gpu.dev)
        gpu.ctx.qk_norm_rope(X, pos, Hq, Hkv, None, None, pk.NORM_NONE, 1e-6, cs, pairs, Q, K)
        outs.append(torch.cat([Q, K], 1).cpu().numpy())
    assert gpu.ctx.stwq_device_status() == 0
    o = odd[:, :Hq + Hkv]
    np.testing.assert_array_equal(outs[1][~o], outs[0][~o])
    np.testing.assert_array_equal(outs[1][o], y[:, :Hq + Hkv][o])


@pytest.mark.parametrize("norm,eps", [(1, 1e-6), (2, 1e-6), (2, 0.0), (2, 100.0)])
@pytest.mark.parametrize("d", [16, 80, 128, 256])
def test_norm_of_a_vector_with_a_nan_or_an_infinity(gpu, d, norm, eps):
    """As the formulas have it: a NaN makes every channel of its vector NaN; an Inf becomes NaN (Inf / Inf) beside zeros; the
    other vectors are what they are without it. A zero vector is 0, or 0 / 0 with eps = 0."""
    torch = gpu.torch
    r = np.random.default_rng(d)
    T, Hq, Hkv = 6, 3, 2
    x = r.standard_normal((T, Hq + 2 * Hkv, d)).astype(np.float32)
    y = x.copy()
    y[1, 0, d // 3], y[2, Hq, d - 1], y[3, 1, 5], y[4, Hq + 1, 0], y[5, 2] = np.nan, np.nan, np.inf, -np.inf, 0
    outs = []
    for a in (x, y):
        Q, K = torch.full((T, Hq, d), 7.0, device=gpu.dev), torch.full((T, Hkv, d), 7.0, device=gpu.dev)
        gpu.ctx.qk_norm_rope(gpu.T(a.reshape(T, -1)), gpu.T(np.arange(T, dtype=np.int32)), Hq, Hkv, None, None, norm, eps, None, 0, Q, K)
        outs.append(torch.cat([Q, K], 1).cpu().numpy())
    assert gpu.ctx.stwq_device_status() == 0
    want = outs[0].copy()
    want[1, 0], want[2, Hq] = np.nan, np.nan
    want[3, 1], want[4, Hq + 1] = 0, 0
    want[3, 1, 5], want[4, Hq + 1, 0] = np.nan, np.nan
    want[5, 2] = np.nan if eps == 0 else 0
    np.testing.assert_array_equal(outs[1], want)


@pytest.mark.parametrize("V", [37, 3000, 40000])
def test_sampling_at_the_ends_of_the_temperature(gpu, V):
    """From the smallest number to Inf, with finite rows and rows that hold +Inf: the limits of the weights."""
    r = np.random.default_rng(V)
    x = r.standard_normal((6, V)).astype(np.float32)
    x[1, [5, V - 2]] = np.inf
    x[2, V // 2:] = -np.inf
    x[3, 9] = np.inf
    x[3, 10:20] = -3.4e38
    x[4] = np.float32(-3.4028235e38)                             # every logit at the type's lowest value
    x[5, ::2] = np.nan
    X = gpu.T(x)
    live = x > -np.inf                                           # (NaN is not)
    m = np.where(live, x, -np.inf).max(1)
    top = live & (x == m[:, None])
    for temp, flat in ((1e-45, False), (1e-30, False), (1e35, True), (3.4e38, True), (np.inf, True)):
        for k, p, mp in ((0, 1.0, 0.0), (20, 1.0, 0.0), (0, 0.5, 0.0), (0, 1.0, 0.5)):
            for u in (0.0, 0.51, 1 - 2.0 ** -24):
                tok, prob, kept = run_sample(gpu, X, temp, k, p, mp, u)
                for i in range(6):
                    infinite = m[i] == np.inf
                    if flat and not infinite and i not in (4,):  # all weights 1 (1e35: 2^-42 off at most): the first live tokens, evenly
                        n = int(live[i].sum())
                        order = np.flatnonzero(live[i])[np.argsort(-x[i][live[i]], kind="stable")]
                        want = min(n, k) if k else n
                        want = -(-want // 2) if p < 1 else want
                        assert kept[i] == want and tok[i] in order[:want]
                        assert abs(prob[i] - 1 / want) <= 2.0 ** -22 / want
                    else:                                        # the largest share the mass
                        share = np.flatnonzero(top[i])
                        assert tok[i] in share
                        c = len(share)
                        c = min(c, k) if k else c
                        c = max(1, -(-c // 2)) if p < 1 else c
                        assert abs(prob[i] - 1 / c) <= 2.0 ** -22 / c


MIXED = ([1] * 30 + [120, 40, 1, 7], [20 * i for i in range(30)] + [60, 500, 2000, 3])


@pytest.mark.parametrize("int8", [False, True])
def test_a_captured_mixed_step_of_both_kernels(gpu, int8):
    """Decoding requests beside chunks, more units than SMs: the few-row kernel is launched behind the tiled one as its dependent.
    Captured, replayed on another stream with other inputs, a kernel that reads the output right behind it."""
    torch, pk = gpu.torch, gpu.pk
    s = make(gpu, *MIXED, 32, 8, 64, 16, int8, 31)
    ctx = pk.Context(0)
    try:
        ctx.stwq_reserve_paged_attention(len(s["new"]), 32, 8, 64)
        t = lambda a: None if a is None else gpu.T(a)  # noqa: E731
        O = torch.zeros((s["T"], 32, 64), dtype=torch.bfloat16, device=gpu.dev)
        copy = torch.zeros_like(O)
        args = [s["Q"], gpu.T(s["cu"]), 120, gpu.T(s["table"]), gpu.T(s["kv"]), s["Kp"], s["Vp"], t(s["s_k"]), t(s["s_v"]), float(s["scale"]), True, pk.OUT_BF16, O]
        side, other = torch.cuda.Stream(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        before = ctx.stwq_launch_count()
        with torch.cuda.stream(side):
            ctx.paged_attention(*args)
        torch.cuda.synchronize()
        assert ctx.stwq_launch_count() - before == 2             # both kernels
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            ctx.paged_attention(*args)
            copy.copy_(O)
            ctx.paged_attention(*args)
        for seed in range(3):
            s["Q"].copy_(torch.randn(s["Q"].shape, device=gpu.dev, generator=torch.Generator(device=gpu.dev).manual_seed(seed)).to(torch.bfloat16))
            O.fill_(9.0)
            torch.cuda.synchronize()
            with torch.cuda.stream(other):
                g.replay()
            torch.cuda.synchronize()
            assert torch.equal(O, copy) and ctx.stwq_device_status() == 0
            check(gpu, s, True, True, O)
            assert torch.equal(O, call(gpu, s, True, True))
    finally:
        ctx.close()


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("new,cached", [([1, 1, 2], [70, 500, 33]), ([90, 5], [40, 300]), MIXED])
def test_strided_queries_and_outputs(gpu, new, cached, int8):
    """Queries as a view of the rows of the qkv linear or head-major, outputs into a wider row or head-major: the same bits as
    dense ones, and nothing else written."""
    torch = gpu.torch
    s = make(gpu, new, cached, 8, 2, 64, 16, int8, 41, pad=2)
    for bf16 in (True, False):
        want = call(gpu, s, True, bf16)
        dt = want.dtype
        row = torch.randn((s["T"], 12 * 64 + 8), device=gpu.dev).to(torch.bfloat16)
        row[:, 8:8 + 8 * 64] = s["Q"].view(s["T"], -1)
        views = [row[:, 8:8 + 8 * 64].view(s["T"], 8, 64), s["Q"].transpose(0, 1).contiguous().transpose(0, 1)]
        wide, heads = torch.full((s["T"], 1000), 7.0, dtype=dt, device=gpu.dev), torch.full((8, s["T"], 64), 7.0, dtype=dt, device=gpu.dev)
        outs = [wide[:, 16:16 + 8 * 64].view(s["T"], 8, 64), heads.transpose(0, 1)]
        for q, o in zip(views, outs):
            call(gpu, dict(s, Q=q), True, bf16, O=o)
            assert gpu.ctx.stwq_device_status() == 0 and torch.equal(o, want)
        assert (wide[:, :16] == 7.0).all() and (wide[:, 16 + 8 * 64:] == 7.0).all()


def test_requests_that_share_pages(gpu):
    """Two requests with one prefix in common read the same pages."""
    for new in ([1, 1, 1], [60, 1, 30]):
        s = make(gpu, new, [320 - n for n in new], 4, 2, 128, 16, False, 51)
        s["table"][1, :16] = s["table"][0, :16]
        s["table"][2] = s["table"][0]
        O = call(gpu, s, True, True)
        assert gpu.ctx.stwq_device_status() == 0
        check(gpu, s, True, True, O)


@pytest.mark.parametrize("n,Hq", [(1, 16), (3, 2), (20, 1)])
def test_attention_of_the_largest_batch(gpu, n, Hq):
    r = np.random.default_rng(n)
    new = r.integers(0, n + 1, 4096)
    s = make(gpu, new, r.integers(0, 60, 4096), Hq, 1, 128, 16, False, 61)
    O = call(gpu, s, True, True)
    assert gpu.ctx.stwq_device_status() == 0
    check(gpu, s, True, True, O)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("B,n,Hq", [(64, 1, 8), (2, 24, 4)])
def test_a_million_keys_per_request(gpu, B, n, Hq, int8):
    """2^20 - 5 keys of one page over and over: 64-bit positions in the list of all blocks. Attention over repeated keys is attention
    over the page's keys, weighed by how often each is seen."""
    torch, S, d, Hkv, L = gpu.torch, 16, 64, 4, 2 ** 20 - 5
    r = np.random.default_rng(71)
    W = 2 ** 16
    table = np.ones((B, W), np.int32)
    Q = gpu.T(r.standard_normal((B * n, Hq, d)).astype(np.float32)).to(torch.bfloat16)
    if int8:
        Kp, Vp = (gpu.T(r.integers(-100, 101, (2, Hkv, S, d)).astype(np.int8)) for _ in range(2))
        s_k, s_v = np.full(L, 1 / 64, np.float32), np.full((Hkv, d), 1 / 64, np.float32)
    else:
        Kp, Vp = (gpu.T(r.standard_normal((2, Hkv, S, d)).astype(np.float32)).to(torch.bfloat16) for _ in range(2))
        s_k = s_v = None
    s = dict(Q=Q, cu=np.arange(B + 1, dtype=np.int32) * n, kv=np.full(B, L, np.int32), table=table, S=S, T=B * n, new=np.full(B, n), d=d, Hq=Hq, Hkv=Hkv,
             scale=0.125, Kp=Kp, Vp=Vp, s_k=s_k, s_v=s_v)
    O = call(gpu, s, True, True).float().cpu().numpy().reshape(B, n, Hkv, Hq // Hkv, d).astype(np.float64)
    assert gpu.ctx.stwq_device_status() == 0
    k, v = (a[1].float().cpu().numpy().astype(np.float64) * (1 / 64 if int8 else 1) for a in (Kp, Vp))
    q = Q.float().cpu().numpy().astype(np.float64).reshape(B, n, Hkv, Hq // Hkv, d)
    seen = L - n + np.arange(n) + 1
    times = (seen[:, None] - np.arange(S)[None] + S - 1) // S    # how often key j of the page is seen
    p = np.exp(np.einsum("bnhgd,hjd->bnhgj", q, k) * 0.125) * times[None, :, None, None]
    p /= p.sum(-1, keepdims=True)
    want, mag = np.einsum("bnhgj,hjd->bnhgd", p, v), np.einsum("bnhgj,hjd->bnhgd", p, np.abs(v))
    a = np.einsum("bnhgd,hjd->bnhgj", np.abs(q), np.abs(k)).max() * 0.125
    # P to 16 bits, scores and exponentials as in the other tests; a running sum of at most 2^20 / 16 terms of a thread or of the
    # tensor core (each at most 2^-23 of the sum so far, truncated), in numerator and denominator; the store
    tol = mag * (2.0 ** -8 + 2 * ((d + 8) * 2.0 ** -23 * a + 2.0 ** -20 + 7.5e-5) + 2 * 2.0 ** 16 * 2.0 ** -23)
    tol += 2.0 ** -8 * (np.abs(want) + tol)
    assert (np.abs(O - want) <= tol).all(), float((np.abs(O - want) / tol).max())
