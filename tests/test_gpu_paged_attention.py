"""paged_attention on the GPU against softmax attention in 64 bits, request by request: both kernels (few rows, tiled),
both cache types, shared key heads, odd sizes, empty requests, causal and full masks, work split over CTAs."""
import numpy as np
import pytest

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


def make(gpu, new, cached, Hq, Hkv, d, S, int8, seed, pad=0, magnitude=1.0):
    """A step: queries, a pool of scattered pages with NaN (code -128) in every slot that holds no visible token."""
    torch = gpu.torch
    r = np.random.default_rng(seed)
    new, cached = np.asarray(new), np.asarray(cached)
    kv = np.where(new > 0, cached + new, cached)
    B = len(new)
    need = -(-kv // S)
    W, NP = max(1, int(need.max())), int(need.sum()) + 2
    perm = r.permutation(NP)[: need.sum()].astype(np.int32)
    table = np.full((B, W), -1, np.int32)                       # entries that no token needs are not looked at
    table[np.arange(W)[None] < need[:, None]] = perm
    T = int(new.sum()) + pad
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    Q = gpu.T((r.standard_normal((max(T, 1), Hq, d)) * magnitude).astype(np.float32)).to(torch.bfloat16)
    s = dict(Q=Q, cu=cu, kv=kv.astype(np.int32), table=table, S=S, T=max(T, 1), new=new, d=d, Hq=Hq, Hkv=Hkv, scale=1 / np.sqrt(d))
    live = np.zeros((NP, S), bool)
    for b in range(B):
        j = np.arange(kv[b])
        live[table[b, j // S], j % S] = True
    if int8:
        code = lambda: r.integers(-128, 128, (NP, Hkv, S, d)).astype(np.int8)  # noqa: E731
        K, V = code(), code()
        K[~live[:, None].repeat(Hkv, 1)] = -128
        V[~live[:, None].repeat(Hkv, 1)] = -128
        s.update(Kp=gpu.T(K), Vp=gpu.T(V), s_k=(r.uniform(0.5, 1.5, W * S) / 64).astype(np.float32),
                 s_v=(r.uniform(0.5, 1.5, (Hkv, d)) / 64).astype(np.float32))
        s["K"], s["V"] = K.astype(np.float64), V.astype(np.float64)
    else:
        val = lambda: gpu.T(r.standard_normal((NP, Hkv, S, d)).astype(np.float32)).to(torch.bfloat16)  # noqa: E731
        K, V = val(), val()
        dead = gpu.T(~live)[:, None, :, None].expand(NP, Hkv, S, d)
        K[dead] = float("nan")
        V[dead] = float("nan")
        s.update(Kp=K, Vp=V, s_k=None, s_v=None, K=K.float().cpu().numpy().astype(np.float64), V=V.float().cpu().numpy().astype(np.float64))
    return s


def call(gpu, s, causal, bf16, max_new=None, O=None):
    torch = gpu.torch
    if O is None:
        O = torch.full((s["T"], s["Hq"], s["d"]), 7.0, dtype=torch.bfloat16 if bf16 else torch.float32, device=gpu.dev)
    t = lambda a: None if a is None else gpu.T(a)  # noqa: E731
    gpu.ctx.paged_attention(s["Q"], gpu.T(s["cu"]), max_new or max(1, int(s["new"].max())), gpu.T(s["table"]), gpu.T(s["kv"]), s["Kp"], s["Vp"],
                            t(s["s_k"]), t(s["s_v"]), float(s["scale"]), causal, 1 if bf16 else 0, O)
    return O


def check(gpu, s, causal, bf16, O):
    q64 = s["Q"].float().cpu().numpy().astype(np.float64)
    got = O.float().cpu().numpy().astype(np.float64)
    S, g, int8 = s["S"], s["Hq"] // s["Hkv"], s["s_k"] is not None
    for b in range(len(s["new"])):
        n, L, t0 = int(s["new"][b]), int(s["kv"][b]), int(s["cu"][b])
        if n == 0:
            continue
        j = np.arange(L)
        for h in range(s["Hkv"]):
            k, v = s["K"][s["table"][b, j // S], h, j % S], s["V"][s["table"][b, j // S], h, j % S]
            if int8:
                k, v = k * s["s_k"][:L, None], v * s["s_v"][h]
            q = q64[t0:t0 + n, h * g:(h + 1) * g]                                   # [n, g, d]
            x = np.einsum("ngd,ld->ngl", q, k) * s["scale"]
            a = np.einsum("ngd,ld->ngl", np.abs(q), np.abs(k)).max(initial=0.0) * s["scale"]
            seen = j[None] < (L - n + np.arange(n)[:, None] + 1 if causal else np.full((n, 1), L))
            x = np.where(seen[:, None], x, -np.inf)
            with np.errstate(invalid="ignore"):
                p = np.exp(x - np.where(seen.any(-1), 1, 0)[:, None, None] * x.max(-1, keepdims=True, initial=-1e300))
            p = np.where(seen[:, None], p, 0)
            den = p.sum(-1, keepdims=True)
            p = p / np.where(den > 0, den, 1)
            want = np.einsum("ngl,ld->ngd", p, v)
            mag = np.einsum("ngl,ld->ngd", p, np.abs(v))
            # roundings: P to 16 bits (bf16 2^-8; fp16 2^-11, and 2^-25 absolute against a reference at most 2^14 above or
            # 2^-4 below the largest weight); an exponent's absolute error (d + 8 roundings of the score's terms) twice, for
            # numerator and sum; exp2 and the final divide 2^-20; fp32 sums over L keys; the store
            tol = mag * ((2.0 ** -11 if int8 else 2.0 ** -8) + 2 * (d_units(s["d"]) * a + 2.0 ** -20) + L * 2.0 ** -23)
            if int8:
                tol += L * 2.0 ** -25 * np.abs(v).max(initial=0.0)
            tol += 2.0 ** -8 * (np.abs(want) + tol) if bf16 else 0
            err = np.abs(got[t0:t0 + n, h * g:(h + 1) * g] - want)
            assert np.isfinite(got[t0:t0 + n, h * g:(h + 1) * g]).all()
            assert (err <= tol + 1e-30).all(), (b, h, float((err / (tol + 1e-30)).max()))
    assert (got[int(s["cu"][-1]):] == 7.0).all()                                    # rows behind the last request


def d_units(d):
    return (d + 8) * 2.0 ** -23


FEW = [  # new, cached, Hq, Hkv, d, S
    ([1], [0], 1, 1, 64, 16), ([1], [16], 4, 4, 128, 16), ([1, 1, 1], [5, 700, 63], 8, 1, 128, 16), ([1] * 9, list(range(0, 900, 100)), 6, 2, 64, 32),
    ([1, 0, 1, 1], [33, 50, 0, 127], 4, 2, 80, 48), ([4, 1, 2], [100, 0, 3], 4, 1, 128, 16), ([16, 3], [40, 1], 2, 2, 48, 64),
    ([3, 8], [1000, 2], 2, 1, 16, 16), ([1] * 70, [37 * i % 400 for i in range(70)], 16, 16, 64, 16), ([2], [5000], 8, 1, 112, 128), ([1], [20000], 9, 1, 96, 16)]


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("case", range(len(FEW)))
def test_few_rows(gpu, case, int8):
    new, cached, Hq, Hkv, d, S = FEW[case]
    s = make(gpu, new, cached, Hq, Hkv, d, S, int8, 100 + case, pad=case % 3)
    for causal in (True, False):
        for bf16 in (True, False):
            O = call(gpu, s, causal, bf16)
            assert gpu.ctx.stwq_device_status() == 0
            check(gpu, s, causal, bf16, O)
            assert gpu.torch.equal(O, call(gpu, s, causal, bf16))                   # bit for bit the same again


TILED = [
    ([17], [0], 1, 1, 64, 16), ([128], [0], 1, 1, 128, 16), ([129], [5], 1, 1, 64, 32), ([256], [0], 1, 1, 128, 64), ([257], [300], 1, 1, 128, 16),
    ([64, 40], [100, 0], 4, 1, 128, 16), ([33, 1, 0, 5], [10, 300, 7, 1000], 8, 2, 64, 48), ([100, 2], [1, 77], 6, 3, 80, 16), ([300], [0], 2, 2, 112, 16),
    ([20], [3000], 2, 1, 128, 64), ([200] * 5, [11, 0, 400, 129, 64], 30, 30, 64, 16), ([3], [200], 20, 1, 48, 16), ([700, 650], [0, 50], 4, 4, 16, 16),
    ([1] * 40 + [100], list(range(0, 800, 20)) + [60], 8, 2, 128, 16), ([40], [9000], 8, 1, 64, 16)]


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("case", range(len(TILED)))
def test_many_rows(gpu, case, int8):
    new, cached, Hq, Hkv, d, S = TILED[case]
    s = make(gpu, new, cached, Hq, Hkv, d, S, int8, 200 + case, pad=case % 3)
    for causal, bf16 in ((True, True), (False, False)):
        O = call(gpu, s, causal, bf16)
        assert gpu.ctx.stwq_device_status() == 0
        check(gpu, s, causal, bf16, O)
        assert gpu.torch.equal(O, call(gpu, s, causal, bf16))


@pytest.mark.parametrize("seed", range(6))
def test_ranges_end_anywhere_in_a_unit(gpu, seed):
    """Lengths of every remainder, so that the ranges of blocks that the CTAs take end at, near and far from the units' ends;
    called twice, since the units' counters have to be back at zero."""
    r = np.random.default_rng(900 + seed)
    B = (3, 8, 8, 20, 40, 70)[seed]
    s = make(gpu, r.integers(1, 3, B), r.integers(0, (3000, 1024, 300, 700, 400, 200)[seed], B), 4, 4 if seed % 2 else 2, 64, 16, seed == 4, 70 + seed, pad=1)
    for _ in range(2):
        check(gpu, s, True, True, call(gpu, s, True, True))
