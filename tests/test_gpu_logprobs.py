"""token_logprobs on the GPU against 64 bits: ranks and ids are equal, floating outputs within a bound that counts the kernel's roundings."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
NAN, INF = float("nan"), float("inf")


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


def reference(x, t, temp, k):
    """One row in float64: log probability, rank, entropy, ids, their log probabilities; and bounds for the three floats."""
    V = x.size
    x = np.where(np.isnan(x), -INF, x) + 0.0
    order = np.lexsort((np.arange(V), -x))
    live = x > -INF
    n_live = int(live.sum())
    ids = np.full(k, -1)
    ids[:min(k, n_live)] = order[:min(k, n_live)]
    if n_live == 0:
        lp = np.full(V, -INF)
        ent, e_s, e_ent = 0.0, 0.0, 0.0
    elif not temp > 0:
        lp = np.where(np.arange(V) == order[0], 0.0, -INF)
        ent, e_s, e_ent = 0.0, 0.0, 0.0
    else:
        m, temp = x[order[0]], min(temp, 3.402823466e38)
        with np.errstate(invalid="ignore"):
            z = np.where(x == m, 0.0, (x - m) / temp)
        w = np.exp(z)
        S = w.sum()
        lp = z - np.log(S)
        p = w / S
        zz = np.where(w > 0, z, 0.0)
        ent = np.log(S) - (p * zz).sum()
        # a weight: the difference (U), the product with c (c itself off by U, the product by U: 3 U of the exponent |z|), ex2 2^-22; a
        # sum: one addition per two logits of a thread, 9 joins with a rescale each (ex2, product, and 3 U of the exponent)
        mean_z = (p * np.abs(zz)).sum()
        adds = V / 512 / 2 + 16 + 9
        e_s = 3 * U * mean_z + 2.0 ** -22 * 10 + (adds + 20) * U
        big = (p * zz * zz).sum()                              # what an error of the exponent does to sum p |z|
        e_ent = e_s + mean_z * (2 * (adds + 24) * U + 2.0 ** -22 * 10 + e_s) + 3 * U * (big + mean_z) + 4 * U * (ent + np.log(S))
    rank = int(np.where(order == t)[0][0]) if 0 <= t < V and live[t] else -1
    return lp, rank, ent, ids, e_s, e_ent


def run(gpu, X, tokens, temp, k, want=None):
    torch = gpu.torch
    B = X.shape[0]
    e = lambda *s: torch.full(s, 77.0, device=gpu.dev)  # noqa: E731
    i = lambda *s: torch.full(s, 77, device=gpu.dev, dtype=torch.int32)  # noqa: E731
    lp, rank, ent = e(B), i(B), e(B)
    ids, tlp = (i(B, k), e(B, k)) if k else (None, None)
    gpu.ctx.token_logprobs(X, temp, tokens, lp, rank, ent, ids, tlp)
    return lp, rank, ent, ids, tlp


def check(gpu, X, tokens, temp, k, status=0):
    lp, rank, ent, ids, tlp = run(gpu, X, tokens, temp, k)
    assert gpu.ctx.stwq_device_status() == status
    x = X.double().cpu().numpy()
    tk = tokens.cpu().numpy()
    T = np.ones(len(x)) if temp is None else temp.double().cpu().numpy()
    lp, rank, ent = lp.double().cpu().numpy(), rank.cpu().numpy(), ent.double().cpu().numpy()
    for b in range(len(x)):
        rlp, rrank, rent, rids, e_s, e_ent = reference(x[b], int(tk[b]), T[b], k)
        assert rank[b] == rrank, (b, rank[b], rrank)
        if tk[b] == -1:
            assert lp[b] == 0
        elif not 0 <= tk[b] < x.shape[1]:
            assert np.isnan(lp[b])
        else:
            close(lp[b], rlp[tk[b]], e_s)
        assert abs(ent[b] - rent) <= e_ent, (b, ent[b], rent, e_ent)
        if k:
            np.testing.assert_array_equal(ids[b].cpu().numpy(), rids)
            for j in range(k):
                close(float(tlp[b, j]), rlp[rids[j]] if rids[j] >= 0 else -INF, e_s)


def close(got, want, e_s):
    """(x - m) / t: two roundings; minus ln S (off by e_s, logf by 2 U relative, below 13): one more."""
    if abs(want) > 3.4028236e38:                              # beyond the largest fp32 plus half a step: the nearest fp32 is infinite
        assert got == np.sign(want) * INF
    else:
        assert abs(got - want) <= e_s + 4 * U * (abs(want) + 13), (got, want)


def logits(gpu, B, V, dt, seed, spread=2.5):
    g = gpu.torch.Generator(device=gpu.dev).manual_seed(seed)
    return gpu.torch.randn((B, V), device=gpu.dev, generator=g).mul_(spread).to(getattr(gpu.torch, dt)), g


@pytest.mark.parametrize("V", [1, 2, 7, 31, 100, 511, 2049, 16384, 50257, 128000, 360448])
@pytest.mark.parametrize("dt", ["bfloat16", "float32"])
@pytest.mark.parametrize("k", [0, 1, 20, 32])
def test_sizes(gpu, V, dt, k):
    torch = gpu.torch
    B = 3 if V > 20000 else 9
    X, g = logits(gpu, B, V, dt, V + k)
    t = torch.randint(0, V, (B,), device=gpu.dev, generator=g, dtype=torch.int32)
    temp = torch.rand((B,), device=gpu.dev, generator=g) + 0.4 if k % 2 == 0 else None
    check(gpu, X, t, temp, k)


@pytest.mark.parametrize("dt", ["bfloat16", "float32"])
@pytest.mark.parametrize("B,V,ld", [(40, 16384, 16384), (170, 1031, 1033), (600, 333, 340), (9, 70001, 70003), (1, 128000, 128000), (2, 99999, 100001)])
def test_rows_anywhere(gpu, dt, B, V, ld):
    """Rows at every alignment; what lies between them (NaN, and logits above all others) does not matter."""
    torch = gpu.torch
    wide, g = logits(gpu, B + 1, ld, dt, B)
    wide = wide.flatten()[3:3 + B * ld].view(B, ld)
    wide[:, V:] = 1e4
    X = wide[:, :V]
    t = torch.randint(0, V, (B,), device=gpu.dev, generator=g, dtype=torch.int32)
    t[0] = int(X[0].float().argmax())
    check(gpu, X, t, None, 20)


@pytest.mark.parametrize("dt", ["bfloat16", "float32"])
@pytest.mark.parametrize("V", [33, 4096, 100000])
def test_ties_go_to_the_lowest_index(gpu, dt, V):
    torch = gpu.torch
    X, g = logits(gpu, 7, V, dt, 3, spread=0.2)
    X[0] = X[0].float().mul(8).round().div(8).to(X.dtype)     # a handful of values
    X[1] = 0.5                                                # all equal
    X[2] = torch.arange(V, device=gpu.dev).to(X.dtype)        # ascending (in steps, where the type is short)
    X[3] = -torch.arange(V, device=gpu.dev).to(X.dtype)       # descending
    X[4] = 0.0
    X[4, ::2] = -0.0                                          # zeros of both signs are equal
    X[5, V // 2:] = 3.0                                       # a plateau of half the row
    t = torch.tensor([V // 2, V - 1, V // 3, V // 3, V // 2, V - 2, 0], device=gpu.dev, dtype=torch.int32)
    for k in (1, 5, 32):
        check(gpu, X, t, None, k)


@pytest.mark.parametrize("dt", ["bfloat16", "float32"])
def test_masked_nan_and_infinite_logits(gpu, dt):
    torch = gpu.torch
    V = 5000
    X, g = logits(gpu, 12, V, dt, 5)
    X[0] = -INF                                               # nothing to draw
    X[1] = NAN
    X[2] = -INF
    X[2, 77] = 1.0                                            # one token alone
    X[3, ::3] = NAN
    X[4, 1::2] = -INF
    X[5, 100] = INF
    X[6, [5, 4000, 17]] = INF                                 # three share everything
    X[7] = INF
    X[8] = torch.finfo(X.dtype).min                           # the lowest value is a logit like any other
    X[9] = torch.finfo(X.dtype).min
    X[9, 3] = 0.0
    X[10, 9] = torch.finfo(X.dtype).max
    X[11, :2500], X[11, 2500] = NAN, -INF
    t = torch.tensor([3, 4, 77, 1, 2, 100, 17, 4999, 8, 5, 9, 2500], device=gpu.dev, dtype=torch.int32)
    for k in (0, 6, 32):
        check(gpu, X, t, None, k)
        check(gpu, X, (t + 1) % V, None, k)
        check(gpu, X, t, torch.full((12,), 0.3, device=gpu.dev), k)


def test_temperatures(gpu):
    torch = gpu.torch
    temps = [1.0, 0.05, 30.0, 0.0, -1.0, NAN, INF, 1e-3, 1e-30, 3e38, 1e-42]
    X, g = logits(gpu, len(temps), 3000, "float32", 6)
    X[0:3] += 80                                              # large logits: the difference to the maximum is taken first
    t = X.argmax(-1).to(torch.int32)
    t[4] = 3
    temp = torch.tensor(temps, device=gpu.dev)
    check(gpu, X, t, temp, 4)
    X[3:7, 50] = INF
    X[5, 20] = INF
    check(gpu, X, t, temp, 4)


def test_tokens_outside_the_vocabulary(gpu):
    torch, ERR = gpu.torch, -13
    X, g = logits(gpu, 5, 1000, "float32", 7)
    t = torch.tensor([-1, 999, 0, -1, 5], device=gpu.dev, dtype=torch.int32)
    check(gpu, X, t, None, 3)
    t[1], t[2] = 1000, -2
    check(gpu, X, t, None, 3, status=ERR)
    assert gpu.ctx.stwq_device_status() == 0


def test_outputs_left_out(gpu):
    torch = gpu.torch
    X, g = logits(gpu, 6, 2000, "bfloat16", 8)
    t = torch.arange(6, device=gpu.dev, dtype=torch.int32)
    lp, rank, ent, ids, tlp = run(gpu, X, t, None, 4)
    a, b, c, d = (torch.empty_like(v) for v in (lp, ent, ids, tlp))
    gpu.ctx.token_logprobs(X, None, t, a)
    assert torch.equal(a, lp)
    gpu.ctx.token_logprobs(X, None, None, None, None, b)
    assert torch.equal(b, ent)
    gpu.ctx.token_logprobs(X, None, None, None, None, None, c, d)
    assert torch.equal(c, ids) and torch.equal(d, tlp)


def test_agrees_with_the_sampler(gpu):
    """The probability that sample_tokens returns without limits is exp of the log probability of its token."""
    torch = gpu.torch
    X, g = logits(gpu, 64, 16384, "bfloat16", 9)
    temp = torch.rand((64,), device=gpu.dev, generator=g) + 0.3
    u = torch.rand((64,), device=gpu.dev, generator=g)
    tok, prob = torch.empty((64,), device=gpu.dev, dtype=torch.int32), torch.empty((64,), device=gpu.dev)
    gpu.ctx.sample_tokens(X, temp, None, None, None, u, tok, prob)
    lp = run(gpu, X, tok, temp, 0)[0]
    assert ((lp.double().exp() / prob.double() - 1).abs() < 4e-6).all()


def test_rows_beyond_2_31_elements(gpu):
    torch = gpu.torch
    V, B = 200000, 11000
    X = torch.zeros((B, V), device=gpu.dev, dtype=torch.bfloat16)
    X[-1], _ = logits(gpu, 1, V, "bfloat16", 10)[0][0], None
    t = torch.full((B,), 5, device=gpu.dev, dtype=torch.int32)
    lp, rank, ent, ids, tlp = run(gpu, X, t, None, 0)
    # the row alone may be split among more blocks, whose sums are grouped differently: each result is held to its own bound
    rlp, rrank, rent, _, e_s, e_ent = reference(X[-1].double().cpu().numpy(), 5, 1.0, 0)
    one = run(gpu, X[-1:].clone(), t[-1:], None, 0)
    for got in ((lp[-1], rank[-1], ent[-1]), (one[0][0], one[1][0], one[2][0])):
        close(float(got[0]), rlp[5], e_s)
        assert got[1] == rrank and abs(float(got[2]) - rent) <= e_ent
    assert (rank[:-1] == 5).all() and ((lp[:-1] + np.log(V)).abs() < 2e-5).all()


def test_refusals(gpu):
    torch, pk = gpu.torch, gpu.pk
    X = torch.zeros((4, 100), device=gpu.dev)
    f, i = lambda *s: torch.zeros(s, device=gpu.dev), lambda *s: torch.zeros(s, device=gpu.dev, dtype=torch.int32)  # noqa: E731

    def refused(code, *a):
        with pytest.raises(pk.StwqError) as e:
            gpu.ctx.token_logprobs(*a)
        assert e.value.code == code
    refused(-1, X, None, None, None)                                        # nothing asked for
    refused(-1, X, None, i(4), None)
    refused(-1, X, None, None, f(4))
    refused(-1, X, None, None, None, i(4), f(4))
    refused(-1, X, None, i(4), f(4), None, None, i(4, 3))
    refused(-2, X, None, i(4), f(4), None, None, i(4, 33), f(4, 33))
    refused(-2, X, None, i(4), f(4), None, None, i(4, 3), f(4, 4))
    refused(-2, X, None, i(5), f(4))
    refused(-4, X.double(), None, i(4), f(4))
    refused(-4, X, None, f(4), f(4))
    refused(-3, X.t(), None, i(100), f(100))
    refused(-2, torch.zeros((1, 360449), device=gpu.dev), None, i(1), f(1))


@pytest.mark.parametrize("V", [33, 100, 313, 511, 787, 1575, 2047, 2619, 4768, 8191])
@pytest.mark.parametrize("k", [1, 16, 17, 32])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_the_likeliest_of_short_rows(gpu, V, k, x):
    """Exactly those of a sort: rows with ties (bf16), with most or all but one stretch masked, with few values, constant, in order."""
    torch = gpu.torch
    g = torch.Generator(device=gpu.dev).manual_seed(V * 37 + k)
    X = torch.randn((9, V), device=gpu.dev, generator=g) * 2
    ninf = float("-inf")
    X[1, torch.rand(V, device=gpu.dev, generator=g) < 0.5] = ninf
    X[2, torch.rand(V, device=gpu.dev, generator=g) < 0.95] = ninf
    X[3, :V // 3] = ninf
    X[3, V // 3 + V // 5 + 1:] = ninf
    X[4] = torch.randint(0, 4, (V,), device=gpu.dev, generator=g).float()
    X[5] = 1.5
    X[6] = torch.arange(V, device=gpu.dev) * 0.5
    X[7] = -torch.arange(V, device=gpu.dev) * 0.5
    X[8] = float("nan")
    X = X.to(torch.bfloat16 if x == "bf16" else torch.float32)
    ids, lps = torch.empty((9, k), device=gpu.dev, dtype=torch.int32), torch.empty((9, k), device=gpu.dev)
    gpu.ctx.token_logprobs(X, None, None, None, None, None, ids, lps)
    v = X.double().cpu().numpy()
    v[np.isnan(v)] = -np.inf
    for row in range(9):
        order = np.lexsort((np.arange(V), -v[row]))
        live = order[v[row][order] > -np.inf][:k]
        want = np.full(k, -1)
        want[:len(live)] = live
        assert (ids[row].cpu().numpy() == want).all(), row
        got = lps[row].double().cpu().numpy()
        assert (got[len(live):] == -np.inf).all()
        if len(live):
            z = v[row] - v[row].max()
            ref = z[live] - np.log(np.exp(z).sum())
            # x - max and the final difference round once each, ln S to a few units of its own size
            assert (np.abs(got[:len(live)] - ref) <= 2.0 ** -24 * (2 * np.abs(ref) + 16 + 4 * np.log(V))).all(), row
