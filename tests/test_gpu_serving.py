"""The serving calls (page_plan, qk_norm_rope, kv_append_paged, sample_tokens) on the GPU against plain
implementations in 64 bits. Integers (tables, slots, tokens, counts) are equal; floating outputs are held to a bound
that counts the roundings of the fp32 arithmetic and of the store."""
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


# ------------------------------------------------------------------------------------------------ page_plan
def plan_ref(cached, new, free, S, table, T):
    """The plan by a loop over requests and tokens (only for inputs that fit)."""
    table = table.copy()
    slots, pos, cu, taken = np.full(T, -1, np.int32), np.full(T, -1, np.int32), [0], 0
    for b in range(len(cached)):
        for i in range(-(-cached[b] // S), -(-(cached[b] + new[b]) // S)):
            table[b, i] = free[taken]
            taken += 1
        for i in range(new[b]):
            p = cached[b] + i
            slots[cu[-1] + i] = table[b, p // S] * S + p % S
            pos[cu[-1] + i] = p
        cu.append(cu[-1] + new[b])
    return table, np.array(cu, np.int32), (cached + new).astype(np.int32), slots, pos, taken


def run_plan(gpu, cached, new, free, S, table, T):
    torch = gpu.torch
    e = lambda n: torch.full((n,), -77, dtype=torch.int32, device=gpu.dev)  # noqa: E731
    B = len(cached)
    i32 = lambda a: gpu.T(np.asarray(a, np.int32))  # noqa: E731
    t = i32(table)
    out = [e(B + 1), e(B), e(T), e(T), e(1)]
    gpu.ctx.page_plan(i32(cached), i32(new), i32(free), S, t, *out)
    return [t.cpu().numpy()] + [o.cpu().numpy() for o in out]


@pytest.mark.parametrize("B,S,max_cached,max_new,pad", [(1, 16, 0, 1, 0), (1, 16, 40, 100, 3), (7, 16, 200, 1, 5), (64, 32, 500, 40, 100),
                                                        (513, 16, 300, 3, 0), (1000, 128, 3000, 60, 1), (4096, 16, 100, 2, 7), (5, 1, 9, 9, 2),
                                                        (33, 48, 1000, 0, 4)])
def test_page_plan_equals_the_loop(gpu, B, S, max_cached, max_new, pad):
    r = np.random.default_rng(B * 7 + S)
    cached = r.integers(0, max_cached + 1, B)
    new = r.integers(0, max_new + 1, B)                         # requests without a new token among them
    W = -(-(max_cached + max(max_new, 1)) // S) + 1
    have = -(-cached // S)
    pool = r.permutation(int((-(-(cached + new) // S)).sum()) + 5).astype(np.int32)
    table = np.full((B, W), -9, np.int32)
    table[np.arange(W)[None] < have[:, None]] = pool[: have.sum()]
    free = pool[have.sum():]
    T = max(1, int(new.sum()) + pad)
    want = plan_ref(cached, new, free, S, table, T)
    got = run_plan(gpu, cached, new, free, S, table, T)
    assert gpu.ctx.stwq_device_status() == 0
    for a, b in zip(got[:5], want[:5]):
        np.testing.assert_array_equal(a, b)
    assert got[5][0] == want[5]


def test_page_plan_reports_what_does_not_fit_and_stays_consistent(gpu):
    ERR_PAGES = -12
    # too few free pages: the second request gets one page of the two it needs
    t, cu, kv, slots, pos, used = run_plan(gpu, [16, 15], [16, 30], [5, 6], 16, np.array([[1, -9, -9], [2, -9, -9]]), 50)
    assert gpu.ctx.stwq_device_status() == ERR_PAGES and gpu.ctx.stwq_device_status() == 0
    assert t.tolist() == [[1, 5, -9], [2, 6, -1]] and used[0] == 2
    assert cu.tolist() == [0, 16, 46] and kv.tolist() == [32, 32]
    assert slots[:16].tolist() == list(range(80, 96)) and slots[16] == 47 and slots[17:33].tolist() == list(range(96, 112))
    assert (slots[33:] == -1).all() and (pos[46:] == -1).all()
    # a slot list that is too short: the tokens beyond it are dropped
    t, cu, kv, slots, pos, used = run_plan(gpu, [0, 0], [3, 3], [4, 5], 16, np.full((2, 2), -9), 4)
    assert gpu.ctx.stwq_device_status() == ERR_PAGES
    assert cu.tolist() == [0, 3, 4] and kv.tolist() == [3, 1] and slots.tolist() == [64, 65, 66, 80]
    # a negative length counts as 0, a row of the table that is too short holds what it can
    t, cu, kv, slots, pos, used = run_plan(gpu, [-3, 30], [-2, 10], [7, 8], 16, np.array([[-9, -9], [1, 2]]), 12)
    assert gpu.ctx.stwq_device_status() == ERR_PAGES
    assert cu.tolist() == [0, 0, 10] and kv.tolist() == [0, 32] and used[0] == 0
    assert slots.tolist() == [46, 47] + [-1] * 10
    # a needed entry that is no page
    *_, slots, pos, used = run_plan(gpu, [8], [1], [7], 16, np.array([[-1]]), 1)
    assert gpu.ctx.stwq_device_status() == ERR_PAGES and slots.tolist() == [-1] and pos.tolist() == [8]


# ------------------------------------------------------------------------------------------------ norms, rotation, append
def head_ref(x, w, norm, eps, cs, rot, pairs):
    """x [T, H, d] float64 -> value, and the magnitude its fp32 rounding errors scale with."""
    if norm == 1:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1 if w is None else w)
    elif norm == 2:
        x = x / np.maximum(np.sqrt((x * x).sum(-1, keepdims=True)), eps) * (1 if w is None else w)
    y, mag = x.copy(), np.abs(x)
    h = rot // 2
    for i in range(h):
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + h)
        c, s = cs[:, None, i], cs[:, None, h + i]
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        m = np.abs(x[..., a]) + np.abs(x[..., b])
        mag[..., a], mag[..., b] = m, m
    return y, mag


# fp32: sum of squares at most 8 + 5 roundings deep plus the mean, +eps, sqrt (halves what came before), reciprocal, two
# multiplies, the rotation's product, fma and subtraction: 7 + 1 + 1 + 1 + 2 + 3 = 15 units of 2^-24
F32_UNITS = 16 * 2.0 ** -24


def check_close(got, want, mag, bf16):
    tol = F32_UNITS * mag + (2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8) if bf16 else 0) + 1e-37
    err = np.abs(got.astype(np.float64) - want)
    assert (err <= tol).all(), float((err / np.maximum(tol, 1e-300)).max())


def make_qkv(gpu, r, T, Hq, Hkv, d, bf16, ld_extra=0):
    torch = gpu.torch
    x = (r.standard_normal((T, (Hq + 2 * Hkv) * d + ld_extra)) * np.exp(r.standard_normal((T, 1)) * 2)).astype(np.float32)
    X = gpu.T(x)
    if bf16:
        X = X.to(torch.bfloat16)
    X = X[:, : (Hq + 2 * Hkv) * d]
    return X, X.float().cpu().numpy().astype(np.float64).reshape(T, Hq + 2 * Hkv, d)


def rope_cs(r, P, rot):
    a = r.uniform(-50, 50, (P, rot // 2))
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


CASES = [  # T, Hq, Hkv, d, rot, norm, pairs, bf16, weights per head, extra columns
    (1, 1, 1, 16, 16, 1, 0, True, False, 0), (1, 3, 1, 64, 64, 2, 1, False, True, 8), (37, 5, 2, 80, 80, 1, 0, True, False, 16),
    (130, 8, 8, 128, 128, 1, 1, False, False, 0), (9, 2, 1, 128, 32, 2, 0, True, True, 0), (17, 3, 3, 48, 48, 0, 0, False, False, 4),
    (33, 4, 2, 256, 256, 1, 0, True, True, 0), (5, 7, 5, 144, 16, 1, 1, True, False, 0), (64, 30, 30, 64, 64, 2, 0, True, True, 0),
    (21, 6, 2, 64, 0, 1, 0, True, False, 0), (2, 1, 1, 240, 240, 2, 0, False, False, 0)]


@pytest.mark.parametrize("case", CASES)
def test_qk_norm_rope_and_the_paged_append(gpu, case):
    torch, pk = gpu.torch, gpu.pk
    T, Hq, Hkv, d, rot, norm, pairs, bf16, per_head, extra = case
    r = np.random.default_rng(T * 31 + d)
    P, eps = 50, 1e-6
    X, x = make_qkv(gpu, r, T, Hq, Hkv, d, bf16, extra)
    pos = r.integers(0, P, T).astype(np.int32)
    w = lambda H: None if norm == 0 else (r.uniform(0.5, 2, (H, d) if per_head else (d,)).astype(np.float32))  # noqa: E731
    wq, wk = w(Hq), w(Hkv)
    cs = rope_cs(r, P, rot) if rot else None
    at = None if cs is None else cs[pos].astype(np.float64)
    q, qm = head_ref(x[:, :Hq], wq, norm, eps, at, rot, pairs)
    k, km = head_ref(x[:, Hq:Hq + Hkv], wk, norm, eps, at, rot, pairs)
    v = x[:, Hq + Hkv:]
    t = lambda a: None if a is None else gpu.T(a)  # noqa: E731

    # dense, token-major in the other type than the input, and head-major in fp32 (what kv_append and qattention take)
    for out_bf16 in (True, False):
        dt = torch.bfloat16 if out_bf16 else torch.float32
        Qo, Ko = torch.full((T, Hq, d), 7.0, dtype=dt, device=gpu.dev), torch.full((T, Hkv, d), 7.0, dtype=dt, device=gpu.dev)
        gpu.ctx.qk_norm_rope(X, gpu.T(pos), Hq, Hkv, t(wq), t(wk), norm, eps, t(cs), pairs, Qo, Ko)
        check_close(Qo.float().cpu().numpy(), q, qm, out_bf16)
        check_close(Ko.float().cpu().numpy(), k, km, out_bf16)
    Qh, Kh = torch.empty((Hq, T, d), device=gpu.dev), torch.empty((Hkv, T, d), device=gpu.dev)
    gpu.ctx.qk_norm_rope(X, gpu.T(pos), Hq, Hkv, t(wq), t(wk), norm, eps, t(cs), pairs, Qh.transpose(0, 1), Kh.transpose(0, 1))
    assert torch.equal(Qh.transpose(0, 1), Qo) and torch.equal(Kh.transpose(0, 1), Ko)

    # paged, bf16 and codes; the last row has no slot, one row is padding
    S, NP = 16, -(-T // 16) + 2
    slots = r.permutation(NP * S)[:T].astype(np.int32)
    pad = T // 2 if T > 4 else -1
    if pad >= 0:
        pos[pad], slots[pad], slots[-1] = -1, -1, -1
    live = (slots >= 0)
    for int8 in (False, True):
        bits = 8 if T % 2 else 6
        lim = (-(1 << bits - 1), (1 << bits - 1) - 1)
        fill = 77 if int8 else 5.0
        Kp = torch.full((NP, Hkv, S, d), fill, dtype=torch.int8 if int8 else torch.bfloat16, device=gpu.dev)
        Vp = Kp.clone()
        Qo = torch.full((T, Hq, d), 7.0, dtype=torch.bfloat16, device=gpu.dev)
        s_k = r.uniform(0.01, 0.05, P if rot else P).astype(np.float32)
        s_v = r.uniform(0.01, 0.05, (Hkv, d)).astype(np.float32)
        gpu.ctx.kv_append_paged(X, gpu.T(pos), gpu.T(slots), Hq, Hkv, t(wq), t(wk), norm, eps, t(cs), pairs, t(s_k) if int8 else None,
                                t(s_v) if int8 else None, bits, Qo, Kp, Vp)
        assert gpu.ctx.stwq_device_status() == 0
        got = Qo.float().cpu().numpy()
        rows = np.arange(T) != pad
        check_close(got[rows], q[rows], qm[rows], True)
        assert pad < 0 or (got[pad] == 7.0).all()
        flat = lambda a: a.float().cpu().numpy().transpose(0, 2, 1, 3).reshape(NP * S, Hkv, d)  # noqa: E731
        gk, gv = flat(Kp), flat(Vp)
        untouched = np.setdiff1d(np.arange(NP * S), slots[live])
        assert (gk[untouched] == fill).all() and (gv[untouched] == fill).all()
        if int8:
            # value codes are those of the definition, the multiplies rounded to fp32 each; a key code may fall on the
            # other side of a tie that lies within the fp32 error of the value before rounding
            rv = (np.float32(1) / s_v).astype(np.float32)
            want = np.clip(np.rint(x[:, Hq + Hkv:].astype(np.float32) * rv[None]), *lim)
            np.testing.assert_array_equal(gv[slots[live]], want[live])
            u = k / s_k[pos][:, None, None].astype(np.float64)
            um = km / s_k[pos][:, None, None] * (F32_UNITS + 2 * 2.0 ** -24)
            lo, hi = np.clip(np.rint(u - um), *lim), np.clip(np.rint(u + um), *lim)
            g = gk[slots[live]]
            assert ((g >= lo[live]) & (g <= hi[live])).all()
        else:
            check_close(gk[slots[live]], k[live], km[live], True)
            np.testing.assert_array_equal(gv[slots[live]], gpu.T(v[live].astype(np.float32)).to(torch.bfloat16).float().cpu().numpy())


def test_bad_positions_and_slots_are_reported_and_write_nothing_wrong(gpu):
    torch = gpu.torch
    r = np.random.default_rng(5)
    T, H, d, P, S, NP = 6, 2, 64, 10, 16, 2
    X, x = make_qkv(gpu, r, T, H, H, d, True)
    cs = rope_cs(r, P, d)
    Kp = torch.full((NP, H, S, d), 5.0, dtype=torch.bfloat16, device=gpu.dev)
    Vp, Qo = Kp.clone(), torch.full((T, H, d), 7.0, dtype=torch.bfloat16, device=gpu.dev)
    call = lambda pos, slots: gpu.ctx.kv_append_paged(X, gpu.T(np.asarray(pos, np.int32)), gpu.T(np.asarray(slots, np.int32)), H, H,  # noqa: E731
                                                      None, None, 1, 1e-6, gpu.T(cs), 0, None, None, 8, Qo, Kp, Vp)
    call([0, 1, P, -2, 4, 5], [0, 1, 2, 3, -1, -1])
    assert gpu.ctx.stwq_device_status() == -8
    assert (Qo[2:4].float() == 0).all() and not (Qo[4:].float() == 0).all()
    k = Kp.permute(0, 2, 1, 3).reshape(NP * S, H, d).float()
    assert (k[2:] == 5).all() and not (k[:2] == 5).all()
    call([0, 1, 2, 3, 4, 5], [4, NP * S, -5, 2 ** 31 - 1, 5, -1])
    assert gpu.ctx.stwq_device_status() == -12
    k = Kp.permute(0, 2, 1, 3).reshape(NP * S, H, d).float()
    assert (k[6:] == 5).all() and not (k[4:6] == 5).all()


# ------------------------------------------------------------------------------------------------ sampling
def sample_ref(x, temp, k, p, mp, u):
    """One row by sorting, in 64 bits. Returns token, probability, kept."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    if not (x > -np.inf).any():
        return -1, 0.0, 0
    m = x.max()
    if not temp > 0:
        return int(np.argmax(x)), 1.0, 1
    order = np.lexsort((np.arange(x.size), -x))
    order = order[x[order] > -np.inf]
    if k > 0:
        order = order[:k]
    with np.errstate(invalid="ignore"):
        w = np.where(x[order] == m, 1.0, np.exp((x[order] - m) / np.float64(temp)))
    if p < 1:
        c = np.cumsum(w)
        order, w = order[: max(1, int((c - w < np.float64(p) * c[-1]).sum()))], w[: max(1, int((c - w < np.float64(p) * c[-1]).sum()))]
    keep = w >= min(max(np.float64(mp), 0), 1)
    order, w = order[keep], w[keep]
    by = np.argsort(order)
    c = np.cumsum(w[by])
    hit = np.flatnonzero(c > np.float64(u) * c[-1])
    i = hit[0] if hit.size else int(np.flatnonzero(w[by] > 0)[-1])
    return int(order[by][i]), w[by][i] / c[-1], order.size


def run_sample(gpu, X, temp, k, p, mp, u):
    torch = gpu.torch
    B = X.shape[0]
    f = lambda a: gpu.T(np.broadcast_to(np.asarray(a, np.float32), (B,)))  # noqa: E731
    tok, pr, kept = (torch.full((B,), -5, dtype=dt, device=gpu.dev) for dt in (torch.int32, torch.float32, torch.int32))
    gpu.ctx.sample_tokens(X, f(temp), gpu.T(np.broadcast_to(np.asarray(k, np.int32), (B,))), f(p), f(mp), f(u), tok, pr, kept)
    return tok.cpu().numpy(), pr.cpu().numpy(), kept.cpu().numpy()


def check_sample(gpu, X, temp, k, p, mp, u):
    B = X.shape[0]
    got = run_sample(gpu, X, temp, k, p, mp, u)
    x = X.float().cpu().numpy()
    b = lambda a, dt: np.broadcast_to(np.asarray(a, dt), (B,))  # noqa: E731
    temp, k, p, mp, u = b(temp, np.float32), b(k, np.int32), b(p, np.float32), b(mp, np.float32), b(u, np.float32)
    for r in range(B):
        want = sample_ref(x[r], temp[r], k[r], p[r], mp[r], u[r])
        assert (got[0][r], got[2][r]) == (want[0], want[2]), (r, got[0][r], got[2][r], want)
        assert abs(got[1][r] - want[1]) <= 2.0 ** -23 * want[1] + 2.0 ** -42


@pytest.mark.parametrize("B,V", [(1, 1), (3, 2), (5, 100), (40, 1000), (7, 4096), (300, 777), (2, 16384), (33, 16385), (4, 51200), (1, 51201),
                                 (3, 128001), (1, 360448)])
@pytest.mark.parametrize("bf16", [False, True])
def test_sampling_equals_the_sort(gpu, B, V, bf16):
    torch = gpu.torch
    r = np.random.default_rng(B * 1000 + V)
    X = gpu.T((r.standard_normal((B, V)) * 2.5).astype(np.float32))
    X = X.to(torch.bfloat16) if bf16 else X
    check_sample(gpu, X, r.uniform(0.3, 1.5, B), r.choice([0, 1, 2, 50, 900, V], B), r.choice([1.0, 0.99, 0.9, 0.3, 0.0], B),
                 r.choice([0.0, 0.01, 0.3, 1.0], B), r.uniform(0, 1, B).astype(np.float32))


def test_sampling_odd_rows_masks_ties_and_extremes(gpu):
    torch = gpu.torch
    V = 1003
    r = np.random.default_rng(3)
    rows = r.standard_normal((14, V)).astype(np.float32)
    rows[0] = -np.inf                                          # nothing to draw
    rows[1] = np.nan
    rows[2] = -np.inf
    rows[2, 517] = -3e38                                       # one token left, at the type's lowest end
    rows[3] = 1.25                                             # all equal: ties by index
    rows[4, ::2] = -np.inf
    rows[5, 100:900] = np.nan
    rows[6, 44] = np.inf                                       # an infinite logit takes everything
    rows[7, [3, 900]] = np.inf
    rows[8] = np.where(r.uniform(size=V) < 0.5, 0.0, -0.0)     # both zeros are one value
    rows[9] = np.round(rows[9])                                # few distinct values
    rows[10] *= 1e30                                           # differences far beyond any exponential
    rows[11] *= 1e-30
    rows[12, :] = np.finfo(np.float32).min
    rows[12, 7] = 0
    rows[13] = -rows[13] ** 2 * 40
    for ld in (V, V + 1, V + 5):                               # rows that start on any alignment
        for bf16 in (False, True):
            wide = torch.zeros((14, ld), device=gpu.dev)
            wide[:, :V] = gpu.T(rows)
            wide = wide.to(torch.bfloat16) if bf16 else wide
            X = wide[:, :V]
            for k, p, mp in ((0, 1.0, 0.0), (10, 1.0, 0.0), (501, 0.5, 0.0), (0, 0.5, 0.0), (0, 0.75, 0.5), (3, 0.999, 1.0)):
                for u in (0.0, 0.5, 1 - 2.0 ** -24, 2.0 ** -30):
                    check_sample(gpu, X, 1.0, k, p, mp, u)
            check_sample(gpu, X, 0.0, 0, 0.5, 0.0, 0.3)        # greedy


def test_sampling_limits_can_be_left_out_and_repeat_bit_for_bit(gpu):
    torch = gpu.torch
    r = np.random.default_rng(11)
    X = gpu.T((r.standard_normal((20, 30000)) * 2).astype(np.float32))
    u = gpu.T(r.uniform(0, 1, 20).astype(np.float32))
    tok = torch.empty(20, dtype=torch.int32, device=gpu.dev)
    gpu.ctx.sample_tokens(X, None, None, None, None, u, tok)
    want = [sample_ref(row, 1.0, 0, 1.0, 0.0, uu)[0] for row, uu in zip(X.cpu().numpy(), u.cpu().numpy())]
    assert tok.cpu().tolist() == want
    a = run_sample(gpu, X, 0.9, 0, 0.93, 0.0, 0.77)
    for _ in range(5):
        for x, y in zip(a, run_sample(gpu, X, 0.9, 0, 0.93, 0.0, 0.77)):
            np.testing.assert_array_equal(x, y)


@pytest.mark.parametrize("V", [16385, 17408, 45000, 128001, 360448])
def test_sampling_with_limits_that_keep_many(gpu, V):
    """top-k on both sides of what is compacted, nuclei of nearly everything, few distinct values and one value only."""
    torch = gpu.torch
    r = np.random.default_rng(V)
    rows = (r.standard_normal((4, V)) * 0.5).astype(np.float32)
    rows[1] = np.round(rows[1] * 4) / 4                        # a handful of values: borders inside long ties
    rows[2] = -1.5                                             # one value
    rows[3, : V // 2] = -np.inf
    X = gpu.T(rows)
    for k in (2047, 2048, 2049, 9000, V - 1, 0):
        for p, mp, u in ((1.0, 0.0, 0.999), (0.9995, 0.0, 0.4), (0.5, 0.02, 0.7)):
            check_sample(gpu, X, [1.0, 0.8, 0.5, 2.0], k, p, mp, u)
