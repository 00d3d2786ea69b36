"""The serving calls at the limits that their documentation names: lengths next to 2^31, the largest batches, values that are no
numbers."""
import subprocess
import sys

import numpy as np
import pytest

from conftest import ROOT
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
