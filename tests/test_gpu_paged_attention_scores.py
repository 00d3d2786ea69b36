"""paged_attention on scores that are far from flat: keys that exceed everything before them, by little and by much, so that
the running reference of the softmax has to move in every place where it can; against softmax attention in 64 bits."""
import numpy as np
import pytest

from test_gpu_paged_attention import call, d_units, make

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


def peaked(gpu, new, cached, Hq, Hkv, d, S, int8, seed, jumps, factors=(1.0, 1.0, 1.0, 0.5, 0.0, -1.0), pad=0):
    """The step of make() with channel 0 taken for the peaks: key j of every request scores jumps[j] (in nats, on top of the
    other channels' noise for a bf16 cache, alone for codes) times the row's factor, and every other key has a zero there."""
    torch = gpu.torch
    r = np.random.default_rng(seed + 1)
    s = make(gpu, new, cached, Hq, Hkv, d, S, int8, seed, pad=pad)
    s["Q"][:, :, 0] = gpu.T((8 * r.choice(factors, (s["T"], Hq))).astype(np.float32)).to(torch.bfloat16)
    for b in range(len(s["new"])):
        at = np.arange(s["kv"][b])
        page, off = gpu.T(s["table"][b, at // S].astype(np.int64)), gpu.T(at % S)
        s["Kp"][page, :, off, 0] = 0
        for j, nats in jumps.items():
            if j >= len(at):
                continue
            if int8:
                s["Kp"][page[j], :, off[j]] = 0
                s["Kp"][page[j], :, off[j], 0] = 127
                s["s_k"][j] = nats / (127 * 8 * s["scale"])
            else:
                s["Kp"][page[j], :, off[j], 0] = nats / (8 * s["scale"])
    s["K"] = s["Kp"].float().cpu().numpy().astype(np.float64)
    return s


def compare(gpu, s, causal, bf16, O):
    """Within the roundings of the kernels: P goes to 16 bits (bf16 2^-8; fp16 2^-11, and 2^-25 absolute beside a sum of 16 or
    more) and once more when a reference moves behind it; fp32 output keeps 22 bits of it. A score is off by d + 8 roundings of
    its terms' magnitude, which enters numerator and sum; an exponential by 2^-20, or 7.5e-5 where the cubic takes it (16-bit
    output). Sums over L keys and a rescale per move in fp32. The store."""
    q64 = s["Q"].float().cpu().numpy().astype(np.float64)
    got = O.float().cpu().numpy().astype(np.float64)
    S, g, int8 = s["S"], s["Hq"] // s["Hkv"], s["s_k"] is not None
    p_err = (2 * 2.0 ** -11 if int8 else 2 * 2.0 ** -8) + 2 * 7.5e-5 if bf16 else 2.0 ** -21
    for b in range(len(s["new"])):
        n, L, t0 = int(s["new"][b]), int(s["kv"][b]), int(s["cu"][b])
        j = np.arange(L)
        for h in range(s["Hkv"] if n else 0):
            k, v = s["K"][s["table"][b, j // S], h, j % S], s["V"][s["table"][b, j // S], h, j % S]
            if int8:
                v = v * s["s_v"][h].astype(np.float64)
            s_k = s["s_k"][:L].astype(np.float64) if int8 else 1.0
            q = q64[t0:t0 + n, h * g:(h + 1) * g]
            with np.errstate(invalid="ignore"):
                x = np.einsum("ngd,ld->ngl", q, k) * s_k * s["scale"]
            a = np.einsum("ngd,ld->ngl", np.abs(q), np.abs(k)) * np.abs(s_k)
            a = a[np.isfinite(a)].max(initial=0.0) * s["scale"]
            seen = j[None] < (L - n + np.arange(n)[:, None] + 1 if causal else np.full((n, 1), L))
            assert seen.any(-1).all()
            x = np.where(seen[:, None], x, -np.inf)
            with np.errstate(invalid="ignore"):
                p = np.exp(x - x.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            nan = np.isnan(p).any(-1)                            # a visible score is NaN or +Inf, or all of them are -Inf
            assert np.isnan(got[t0:t0 + n, h * g:(h + 1) * g][nan]).all(), (b, h)
            p[nan] = 0
            want, mag = np.einsum("ngl,ld->ngd", p, v), np.einsum("ngl,ld->ngd", p, np.abs(v))
            tol = mag * (p_err + np.expm1(2 * (d_units(s["d"]) * a + 2.0 ** -20)) + (L + 32) * 2.0 ** -23)
            if int8:
                tol += 2 * L * 2.0 ** -25 * np.abs(v).max()
            tol += (2.0 ** -8 if bf16 else 2.0 ** -24) * (np.abs(want) + tol)
            err = np.abs(got[t0:t0 + n, h * g:(h + 1) * g] - want)
            err[nan] = 0
            assert (err <= tol + 1e-30).all(), (b, h, float(np.nanmax(err / (tol + 1e-30))), np.argwhere(~(err <= tol + 1e-30))[:4].tolist())
    assert (got[int(s["cu"][-1]):] == 7.0).all()


# new, cached, Hq, Hkv, d, S: one unit whose keys are cut over many CTAs, units that fill the SMs (their keys are not cut), odd sizes
TILED = [([40], [390], 1, 1, 64, 16), ([24], [400], 80, 80, 64, 16), ([20, 33], [420, 387], 80, 40, 128, 64), ([150, 2], [300, 431], 6, 3, 80, 16),
         ([300], [140], 4, 4, 48, 32), ([3], [430], 20, 1, 128, 16), ([1] * 30 + [120], [400] * 30 + [330], 8, 2, 128, 16), ([2, 12], [420, 430], 4, 2, 64, 16)]
# the reference moves in the first keys' second half, in either half of later tiles, and twice within one; each by less than 80 nats
STEPS = {3: 5.0, 70: 18.0, 100: 36.0, 135: 70.0, 195: 130.0, 200: 150.0, 330: 215.0, 400: 223.0}


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("case", range(len(TILED)))
def test_reference_moves_in_the_tiles(gpu, case, int8):
    new, cached, Hq, Hkv, d, S = TILED[case]
    s = peaked(gpu, new, cached, Hq, Hkv, d, S, int8, 300 + case, STEPS, pad=case % 3)
    for causal, bf16 in ((True, True), (False, True), (True, False)):
        O = call(gpu, s, causal, bf16)
        assert gpu.ctx.stwq_device_status() == 0
        compare(gpu, s, causal, bf16, O)
        assert gpu.torch.equal(O, call(gpu, s, causal, bf16))


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("nats", [92.0, 140.0, 200.0, 280.0])
@pytest.mark.parametrize("shape", [([40], [390], 2, 2, 64, 16), ([20], [410], 80, 80, 64, 16), ([130], [300], 1, 1, 128, 32)])
def test_a_key_far_above_all_before_it(gpu, shape, nats, int8):
    """One key 133 to 404 octaves above the reference that the row's first keys set, in every column of eight."""
    new, cached, Hq, Hkv, d, S = shape
    for c in range(8):
        s = peaked(gpu, new, cached, Hq, Hkv, d, S, int8, 400 + c, {(72, 136, 200, 328)[(c + c // 4) % 4] + c: nats}, pad=1)
        O = call(gpu, s, True, True)
        assert gpu.ctx.stwq_device_status() == 0
        compare(gpu, s, True, True, O)


def nonfinite(gpu, shape, int8, kind, c, seed):
    """A step with NaN or Inf among its scores: in one key (column c of eight, so that rows before it do not see it), in one query,
    in all keys before a finite one, in all keys."""
    new, cached, Hq, Hkv, d, S = shape
    s = peaked(gpu, new, cached, Hq, Hkv, d, S, int8, seed, {3: 5.0, 300: 30.0}, factors=(1.0,), pad=1)
    nan, inf = float("nan"), float("inf")
    L = int(s["kv"].max())
    at = {"nan key": [L - 24 + c], "nan key early": [72 + c], "inf key": [L - 24 + c], "-inf keys": range(L - 10), "-inf everywhere": range(L)}.get(kind, [])
    value = nan if "nan" in kind else -inf if kind[0] == "-" else inf
    if kind == "nan query":
        s["Q"][s["T"] // 2, :, 1 + c] = nan
    for b in range(len(s["new"])):
        j = np.array([i for i in at if i < s["kv"][b]], np.int64)
        page, off = gpu.T(s["table"][b, j // S].astype(np.int64)), gpu.T(j % S)
        if int8:                                                 # Inf by way of the key's scale: every score of the key is that, or NaN
            s["s_k"][j] = abs(value)
            s["Kp"][page, :, off] = 0
            s["Kp"][page, :, off, 0] = -127 if value < 0 else 127
        else:
            s["Kp"][page, :, off, 0] = value
    s["K"] = s["Kp"].float().cpu().numpy().astype(np.float64)
    return s


KINDS = ["nan key", "nan key early", "nan query", "inf key", "-inf keys", "-inf everywhere"]


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", [([40], [390], 2, 2, 64, 16), ([20], [410], 80, 80, 64, 16), ([90, 33], [300, 350], 4, 2, 128, 32)])
def test_nan_and_infinite_scores_in_the_tiles(gpu, shape, kind, int8):
    for c in range(8):
        s = nonfinite(gpu, shape, int8, kind, c, 500 + c)
        for bf16 in (True, False):
            O = call(gpu, s, True, bf16)
            assert gpu.ctx.stwq_device_status() == 0
            compare(gpu, s, True, bf16, O)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_units_behind_one_that_ends_inside_a_block(gpu, d, int8):
    """Short requests of every remainder modulo 16, many to a CTA: the stage whose last value rows were cleared is refilled with
    the next unit's keys at once, and none of those may be lost. Large values make a lost row show."""
    r = np.random.default_rng(d)
    s = peaked(gpu, [1] * 600, r.integers(1, 150, 600), 16, 8, d, 16, int8, 700, {})
    s["Vp"] = s["Vp"] * 0 + 100 if int8 else s["Vp"] * 0 + 64        # (dead slots stay NaN)
    s["V"] = s["Vp"].float().cpu().numpy().astype(np.float64)
    for _ in range(4):
        O = call(gpu, s, True, True)
        assert gpu.ctx.stwq_device_status() == 0
        compare(gpu, s, True, True, O)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", [([1], [430], 1, 1, 64, 16), ([4, 1], [430, 409], 4, 1, 128, 16), ([1] * 40, [390 + i for i in range(40)], 16, 4, 64, 32)])
def test_nan_and_infinite_scores_of_few_rows(gpu, shape, kind, int8):
    for c in range(8):
        s = nonfinite(gpu, shape, int8, kind, c, 600 + c)
        for bf16 in (True, False):
            O = call(gpu, s, True, bf16)
            assert gpu.ctx.stwq_device_status() == 0
            compare(gpu, s, True, bf16, O)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("shape", [([1], [430], 1, 1, 64, 16), ([4, 1], [430, 99], 4, 1, 128, 16), ([1] * 40, [390 + i for i in range(40)], 16, 4, 64, 32),
                                   ([16], [420], 1, 1, 80, 16), ([3], [5000], 12, 4, 112, 64)])
def test_reference_moves_with_few_rows(gpu, shape, int8):
    """By little and by much: over keys of one warp, over warps, over the CTAs that share a unit."""
    new, cached, Hq, Hkv, d, S = shape
    for jumps in (STEPS, {72: 92.0}, {203: 280.0}, {5: 140.0, 333: 200.0}):
        s = peaked(gpu, new, cached, Hq, Hkv, d, S, int8, 800, jumps, pad=1)
        for causal, bf16 in ((True, True), (False, True), (True, False)):
            O = call(gpu, s, causal, bf16)
            assert gpu.ctx.stwq_device_status() == 0
            compare(gpu, s, causal, bf16, O)
            assert gpu.torch.equal(O, call(gpu, s, causal, bf16))
