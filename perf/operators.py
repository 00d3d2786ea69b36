"""The serving-side operators of the library as measured cases: page plan, head norms with rotation, attention of new
tokens over a paged cache, and token sampling.

`own` false: each operator in its plain form (elementary torch operations, fp32 or fp64). `own` true: the calls a
user's program makes of the library. Both work on what `prepare` returns. `exact` gives the floating outputs in 64
bits, written apart from the plain form.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
_ctx = None


def _context():
    """The library context a program keeps for its lifetime (workspaces live in it)."""
    global _ctx
    if _ctx is None:
        import paper_2601_21238_b200 as pk
        _ctx = pk.Context(torch.cuda.current_device())
    return _ctx


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # continuous batching, pure decode: 64 requests get one token each; some cross into a new page
        dict(name="plan decode 64", op="plan", B=64, max_new=1, max_cached=4096, page=16),
        # a scheduler step with chunked prefills: up to 256 new tokens for each of 300 requests, padded slot list
        dict(name="plan mixed 300", op="plan", B=300, max_new=256, max_cached=8192, page=64),
        # raster-order decode step of a batch of 256 images (2048-wide model, 16 heads of 128): one token each
        dict(name="qkv decode 256", op="qkv", form="paged", T=256, Hq=16, Hkv=16, d=128, x="bf16", norm="rms",
             rope="half", rot=128, page=64, P=256),
        # a scale of the VAR-d30 pyramid: 32 samples x 256 tokens, 30 heads of 64, unit-norm queries and keys
        dict(name="qkv scale 8192", op="qkv", form="paged", T=8192, Hq=30, Hkv=30, d=64, x="bf16", norm="l2",
             rope="pairs", rot=64, page=16, P=680),
        # MAR-Huge-shaped prefill: 256 tokens x 256 samples, 16 heads of 80, queries and keys only, fp32 out of the linear
        dict(name="qk prefill 65536", op="qkv", form="dense", T=65536, Hq=16, Hkv=16, d=80, x="f32", norm="rms",
             rope="half", rot=80, page=16, P=256),
        # decode of a small batch with shared key heads (4 query heads per key head), about a thousand keys each
        dict(name="decode 8 x 1k", op="attend", B=8, max_q=1, cached=1024, ragged=True, Hq=32, Hkv=8, d=128,
             cache="bf16", page=16, causal=True, out="bf16"),
        # raster-order decode of 256 images over the quantized cache (16 heads of 128, up to 255 earlier tokens)
        dict(name="decode 256 x 255 int8", op="attend", B=256, max_q=1, cached=255, ragged=False, Hq=16, Hkv=16, d=128,
             cache="int8", page=64, causal=True, out="bf16"),
        # long-context decode: 16 requests of up to 32k cached tokens
        dict(name="decode 16 x 32k", op="attend", B=16, max_q=1, cached=32767, ragged=True, Hq=32, Hkv=8, d=128,
             cache="bf16", page=64, causal=True, out="bf16"),
        # the last scale of a VAR-d30 pyramid: 256 new tokens see the 424 before them and each other, quantized cache
        dict(name="chunk 32 x 256 int8", op="attend", B=32, max_q=256, cached=424, ragged=False, Hq=30, Hkv=30, d=64,
             cache="int8", page=32, causal=False, out="bf16"),
        # chunked prefill: 2048 new tokens of each of 4 requests behind up to 6k cached ones
        dict(name="chunk 4 x 2048", op="attend", B=4, max_q=2048, cached=6144, ragged=True, Hq=32, Hkv=8, d=128,
             cache="bf16", page=64, causal=True, out="bf16"),
        # raster-order decode: one codebook token (16384 entries) for each of 256 images, top-k and top-p
        dict(name="sample 256 x 16384", op="sample", B=256, V=16384, x="bf16", top_k=2000, top_p=0.95, min_p=0.0),
        # text-sized vocabulary, nucleus and min-p only: no top-k bounds the candidates
        dict(name="sample 64 x 128000", op="sample", B=64, V=128000, x="f32", top_k=0, top_p=0.9, min_p=0.001),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["plan", "qkv", "attend", "attend", "sample"])
    if op == "plan":
        return dict(op="plan", B=_log_int(rng, 1, 512), max_new=_log_int(rng, 1, 256), max_cached=rng.randint(0, 8192),
                    page=rng.choice([16, 32, 64, 128]))
    if op == "qkv":
        d = rng.choice([64, 80, 128])
        Hkv = rng.choice([1, 2, 4, 8, 16])
        form = rng.choice(["paged", "paged", "dense"])
        return dict(op="qkv", form=form, T=_log_int(rng, 1, 20000), Hq=Hkv * rng.choice([1, 2, 3]), Hkv=Hkv, d=d,
                    x=rng.choice(["bf16", "f32"]), norm=rng.choice(["rms", "l2", "none"]),
                    rope=rng.choice(["half", "pairs"]), rot=rng.choice([16, 32, d]), page=rng.choice([16, 32, 64]),
                    P=rng.choice([256, 680, 2048]))
    if op == "attend":
        Hkv = rng.choice([1, 2, 4, 8])
        max_q = 1 if rng.random() < 0.5 else _log_int(rng, 2, 1024)
        B = _log_int(rng, 1, 128 if max_q == 1 else 6)
        return dict(op="attend", B=B, max_q=max_q, cached=_log_int(rng, 1, min(16384 if max_q == 1 else 4096, 262144 // B)),
                    ragged=rng.random() < 0.7, Hq=Hkv * rng.choice([1, 2, 4, 8] if Hkv <= 4 else [1, 4]), Hkv=Hkv,
                    d=rng.choice([64, 80, 128]), cache=rng.choice(["bf16", "int8"]), page=rng.choice([16, 32, 64, 128]),
                    causal=rng.random() < 0.7, out=rng.choice(["bf16", "bf16", "f32"]))
    V = _log_int(rng, 100, 150000)
    return dict(op="sample", B=_log_int(rng, 1, max(1, min(512, 8000000 // V))), V=V, x=rng.choice(["bf16", "f32"]),
                top_k=rng.choice([0, 1, 50, 900, 2000]), top_p=rng.choice([1.0, 0.95, 0.9, 0.5]),
                min_p=rng.choice([0.0, 0.0, 0.02, 0.1]))


# ---------------------------------------------------------------------------------------------- inputs
def _lens(case, seed):
    """Host-side lengths of the requests of an attention case: new tokens and cached tokens per request. The case fixes
    the set of lengths (a step's total stays the same), the seed their order."""
    r = np.random.RandomState(case["B"] * 131 + case["max_q"] * 7 + case["cached"])
    B = case["B"]
    if case["ragged"]:
        new = r.randint(max(1, case["max_q"] // 2), case["max_q"] + 1, B)
        cached = r.randint(case["cached"] // 4, case["cached"] + 1, B)
        new[0], cached[B // 2] = case["max_q"], case["cached"]
        r = np.random.RandomState(seed % (1 << 31))
        new, cached = r.permutation(new), r.permutation(cached)
    else:
        new, cached = np.full(B, case["max_q"]), np.full(B, case["cached"])
    return new.astype(np.int64), cached.astype(np.int64)


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), device=DEV).to(torch.int32)


def _pages(lens, page, seed):
    """A block table of scattered pages holding lens[b] tokens per request, and the number of pages in the pool."""
    need = -(-lens // page)
    W = max(1, int(need.max()))
    total = int(need.sum())
    NP = total + 3
    perm = np.random.RandomState((seed + 77) % (1 << 31)).permutation(NP)[:total]
    table = np.zeros((len(lens), W), np.int32)
    table[np.arange(W)[None, :] < need[:, None]] = perm
    return table, NP


def _rope_table(P, rot):
    f = 10000.0 ** (-torch.arange(0, rot // 2, device=DEV, dtype=torch.float64) / (rot // 2))
    a = torch.arange(P, device=DEV, dtype=torch.float64)[:, None] * f[None, :]
    return torch.cat([a.cos(), a.sin()], 1).float().contiguous()


def _prepare_plan(c, seed):
    r = np.random.RandomState(seed % (1 << 31))
    B, page = c["B"], c["page"]
    cached = r.randint(0, c["max_cached"] + 1, B)
    new = r.randint(1, c["max_new"] + 1, B)
    W = -(-(c["max_cached"] + c["max_new"]) // page)
    before, after = -(-cached // page), -(-(cached + new) // page)
    pool = r.permutation(int(after.sum()) + 8)
    table = np.full((B, W), -1, np.int32)
    table[np.arange(W)[None, :] < before[:, None]] = pool[: int(before.sum())]
    free = pool[int(before.sum()):]
    T = B * c["max_new"]                                     # capacity of the step: the rows behind the last token are padding
    e = lambda *s: torch.empty(s, dtype=torch.int32, device=DEV)  # noqa: E731
    return dict(cached=_i32(cached), new=_i32(new), free=_i32(free), page=page, table=_i32(table), T=T,
                cu=e(B + 1), kv=e(B), slots=e(T), pos=e(T), used=e(1))


def _prepare_qkv(c, seed):
    g = _gen(seed)
    T, Hq, Hkv, d, page = c["T"], c["Hq"], c["Hkv"], c["d"], c["page"]
    dt = torch.bfloat16 if c["x"] == "bf16" else torch.float32
    X = torch.randn((T, (Hq + 2 * Hkv) * d), device=DEV, generator=g).mul_(1.7).to(dt)
    s = dict(X=X, Hq=Hq, Hkv=Hkv, d=d, norm=c["norm"], rope=c["rope"], rot=c["rot"], eps=1e-6,
             pos=torch.randint(0, c["P"], (T,), device=DEV, generator=g, dtype=torch.int32), cs=_rope_table(c["P"], c["rot"]))
    if c["norm"] == "l2":                                    # a learned scale per head: the temperature of unit-norm attention
        s["wq"] = (torch.rand((Hq, 1), device=DEV, generator=g) * 3 + 1).expand(Hq, d).contiguous()
        s["wk"] = torch.ones((Hkv, d), device=DEV)
    elif c["norm"] == "rms":
        s["wq"] = torch.rand((d,), device=DEV, generator=g) + 0.5
        s["wk"] = torch.rand((d,), device=DEV, generator=g) + 0.5
    else:
        s["wq"] = s["wk"] = None
    if c["form"] == "dense":
        s.update(Qo=torch.empty((T, Hq, d), device=DEV, dtype=dt), Ko=torch.empty((T, Hkv, d), device=DEV, dtype=dt))
    else:
        NP = -(-T // page) + 2
        slots = torch.randperm(NP * page, device=DEV, generator=g)[:T].to(torch.int32)
        s.update(Qo=torch.empty((T, Hq, d), device=DEV, dtype=torch.bfloat16), slots=slots,
                 Kp=torch.randn((NP, Hkv, page, d), device=DEV, generator=g).to(torch.bfloat16),
                 Vp=torch.randn((NP, Hkv, page, d), device=DEV, generator=g).to(torch.bfloat16))
    return s


def _prepare_attend(c, seed):
    g = _gen(seed)
    new, cached = _lens(c, seed)
    B, Hq, Hkv, d, page = c["B"], c["Hq"], c["Hkv"], c["d"], c["page"]
    kv = new + cached
    table, NP = _pages(kv, page, seed)
    cu = np.concatenate([[0], np.cumsum(new)])
    T = int(cu[-1])
    s = dict(Q=torch.randn((T, Hq, d), device=DEV, generator=g).mul_(1.2).to(torch.bfloat16), cu=_i32(cu), max_q=int(new.max()),
             table=_i32(table), kv=_i32(kv), max_kv=int(kv.max()), scale=1.0 / math.sqrt(d), causal=c["causal"], g=Hq // Hkv, page=page)
    if c["cache"] == "bf16":
        s.update(Kp=torch.empty((NP, Hkv, page, d), device=DEV, dtype=torch.bfloat16).normal_(generator=g),
                 Vp=torch.empty((NP, Hkv, page, d), device=DEV, dtype=torch.bfloat16).normal_(generator=g), s_k=None, s_v=None)
    else:                                                    # codes of values of about unit size: a step is about 1/32
        code = lambda: torch.empty((NP, Hkv, page, d), device=DEV, dtype=torch.bfloat16).normal_(generator=g).mul_(32).round_().clamp_(-128, 127).to(torch.int8)  # noqa: E731
        s.update(Kp=code(), Vp=code(), s_k=(torch.rand((s["max_kv"],), device=DEV, generator=g) + 0.5) / 32,
                 s_v=(torch.rand((Hkv, d), device=DEV, generator=g) + 0.5) / 32)
    s["O"] = torch.empty((T, Hq, d), device=DEV, dtype=torch.bfloat16 if c["out"] == "bf16" else torch.float32)
    return s


def _prepare_sample(c, seed):
    g = _gen(seed)
    B, V = c["B"], c["V"]
    X = torch.randn((B, V), device=DEV, generator=g).mul_(2.5).to(torch.bfloat16 if c["x"] == "bf16" else torch.float32)
    f = lambda v: torch.full((B,), v, device=DEV, dtype=torch.float32)  # noqa: E731
    return dict(X=X, temp=torch.rand((B,), device=DEV, generator=g) * 0.7 + 0.5,
                top_k=torch.full((B,), c["top_k"], device=DEV, dtype=torch.int32), top_p=f(c["top_p"]), min_p=f(c["min_p"]),
                u=torch.rand((B,), device=DEV, generator=g), token=torch.empty((B,), device=DEV, dtype=torch.int32),
                prob=f(0.0), kept=torch.empty((B,), device=DEV, dtype=torch.int32))


_PREPARE = dict(plan=_prepare_plan, qkv=_prepare_qkv, attend=_prepare_attend, sample=_prepare_sample)


def prepare(case, seed):
    s = _PREPARE[case["op"]](case, int(seed))
    s["op"] = case["op"]
    return s


# ---------------------------------------------------------------------------------------------- the library's calls
def _own_plan(s):
    _context().page_plan(s["cached"], s["new"], s["free"], s["page"], s["table"], s["cu"], s["kv"], s["slots"], s["pos"], s["used"])
    return dict(table=s["table"], cu=s["cu"], kv=s["kv"], slots=s["slots"], pos=s["pos"], used=s["used"])


def _own_qkv(s):
    norm, rope = dict(none=0, rms=1, l2=2)[s["norm"]], dict(half=0, pairs=1)[s["rope"]]
    if "Kp" in s:
        _context().kv_append_paged(s["X"], s["pos"], s["slots"], s["Hq"], s["Hkv"], s["wq"], s["wk"], norm, s["eps"], s["cs"], rope,
                                   None, None, 8, s["Qo"], s["Kp"], s["Vp"])
        return dict(q=s["Qo"], k=s["Kp"], v=s["Vp"])
    _context().qk_norm_rope(s["X"], s["pos"], s["Hq"], s["Hkv"], s["wq"], s["wk"], norm, s["eps"], s["cs"], rope, s["Qo"], s["Ko"])
    return dict(q=s["Qo"], k=s["Ko"])


def _own_attend(s):
    _context().paged_attention(s["Q"], s["cu"], s["max_q"], s["table"], s["kv"], s["Kp"], s["Vp"], s["s_k"], s["s_v"], s["scale"],
                               s["causal"], 1 if s["O"].dtype == torch.bfloat16 else 0, s["O"])
    return dict(o=s["O"])


def _own_sample(s):
    _context().sample_tokens(s["X"], s["temp"], s["top_k"], s["top_p"], s["min_p"], s["u"], s["token"], s["prob"], s["kept"])
    return dict(token=s["token"], prob=s["prob"], kept=s["kept"])


# ---------------------------------------------------------------------------------------------- the plain forms
def _plain_plan(s):
    cached, new, page, table = s["cached"].long(), s["new"].long(), s["page"], s["table"]
    before, after = (cached + page - 1) // page, (cached + new + page - 1) // page
    need = after - before
    start = torch.cumsum(need, 0) - need
    col = torch.arange(table.shape[1], device=DEV)[None, :]
    fresh = (col >= before[:, None]) & (col < after[:, None])
    at = (start[:, None] + col - before[:, None]).clamp(0, s["free"].numel() - 1)
    full = torch.where(fresh, s["free"][at], table)
    cu = torch.cat([torch.zeros(1, device=DEV, dtype=torch.int64), torch.cumsum(new, 0)])
    t = torch.arange(s["T"], device=DEV)
    b = (torch.searchsorted(cu, t, right=True) - 1).clamp(max=new.numel() - 1)
    pos = cached[b] + t - cu[b]
    live = t < cu[-1]
    slot = full[b, (pos // page).clamp(max=table.shape[1] - 1)].long() * page + pos % page
    none = torch.full_like(t, -1)
    i32 = lambda v: v.to(torch.int32)  # noqa: E731
    return dict(table=full, cu=i32(cu), kv=i32(cached + new), slots=i32(torch.where(live, slot, none)),
                pos=i32(torch.where(live, pos, none)), used=i32(need.sum()[None]))


def _plain_head(x, w, cs, s):
    """x [T, H, d] fp32 -> normed, scaled and rotated."""
    if s["norm"] == "rms":
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * w
    elif s["norm"] == "l2":
        x = x / (x * x).sum(-1, keepdim=True).sqrt().clamp(min=s["eps"]) * w
    rot = s["rot"]
    h = rot // 2
    c, n = cs[:, None, :h], cs[:, None, h:]
    if s["rope"] == "half":
        a, b = x[..., :h], x[..., h:rot]
        return torch.cat([a * c - b * n, b * c + a * n, x[..., rot:]], -1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2), x[..., rot:]], -1)


def _plain_qkv(s):
    Hq, Hkv, d = s["Hq"], s["Hkv"], s["d"]
    x = s["X"].view(-1, Hq + 2 * Hkv, d)
    cs = s["cs"][s["pos"].long()]
    q = _plain_head(x[:, :Hq].float(), s["wq"], cs, s)
    k = _plain_head(x[:, Hq:Hq + Hkv].float(), s["wk"], cs, s)
    if "Kp" not in s:
        return dict(q=q.to(s["Qo"].dtype), k=k.to(s["Ko"].dtype))
    page = s["Kp"].shape[2]
    p, o = s["slots"].long() // page, s["slots"].long() % page
    s["Kp"][p, :, o] = k.to(torch.bfloat16)
    s["Vp"][p, :, o] = x[:, Hq + Hkv:].to(torch.bfloat16)
    return dict(q=q.to(torch.bfloat16), k=s["Kp"], v=s["Vp"])


def _plain_attend(s):
    T, Hq, d = s["Q"].shape
    Hkv, page, g = s["Kp"].shape[1], s["page"], s["g"]
    B, mq, mk = s["kv"].numel(), s["max_q"], s["max_kv"]
    cu, kv = s["cu"].long(), s["kv"].long()
    new = cu[1:] - cu[:-1]
    j = torch.arange(mk, device=DEV)
    pg = s["table"].long()[:, j // page]                     # [B, mk]
    k = s["Kp"][pg, :, j % page].float()                     # [B, mk, Hkv, d]
    v = s["Vp"][pg, :, j % page].float()
    if s["s_k"] is not None:
        k = k * s["s_k"][None, :mk, None, None]
        v = v * s["s_v"]
    i = torch.arange(mq, device=DEV)
    q = s["Q"][(cu[:-1, None] + i).clamp(max=T - 1)].float()  # [B, mq, Hq, d]
    q = q.view(B, mq, Hkv, g, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, g * mq, d)
    x = torch.matmul(q, k.permute(0, 2, 3, 1)) * s["scale"]
    seen = j[None, None, :] < kv[:, None, None]
    if s["causal"]:
        seen = seen & (j[None, None, :] <= (kv - new)[:, None, None] + i[None, :, None])
    x = x.view(B, Hkv, g, mq, mk).masked_fill(~seen[:, None, None], float("-inf"))
    m = x.amax(-1, keepdim=True).clamp(min=-3e38)
    x = torch.exp(x - m)
    o = torch.matmul(x.view(B, Hkv, g * mq, mk), v.permute(0, 2, 1, 3)).view(B, Hkv, g, mq, d)
    o = o / x.sum(-1, keepdim=True).clamp(min=1e-30)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, mq, Hq, d)
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(cu, t, right=True) - 1
    return dict(o=o[b, t - cu[b]].to(s["O"].dtype))


def _plain_sample(s):
    x = s["X"].double()
    B, V = x.shape
    live = x > float("-inf")
    x = torch.where(live, x, float("-inf"))                  # NaN counts as masked
    m = x.amax(-1, keepdim=True)
    w = torch.where(x == m, 1.0, torch.exp((x - m) / s["temp"].double()[:, None])) * live
    xs, order = torch.sort(x, dim=-1, descending=True, stable=True)
    ws = w.gather(1, order)
    rank = torch.arange(V, device=DEV)[None, :]
    k, p = s["top_k"].long()[:, None], s["top_p"].double()[:, None]
    keep = (xs > float("-inf")) & ((k <= 0) | (rank < k))
    ws = ws * keep
    cum = torch.cumsum(ws, -1)
    keep = keep & ((p >= 1) | (cum - ws < p * cum[:, -1:]))
    keep = keep & (ws >= s["min_p"].double()[:, None])
    kept = torch.zeros_like(live).scatter_(1, order, keep)
    w = w * kept
    c = torch.cumsum(w, -1)
    hit = c > s["u"].double()[:, None] * c[:, -1:]
    token = torch.where(hit.any(-1), hit.to(torch.int8).argmax(-1), V - 1 - kept.flip(-1).to(torch.int8).argmax(-1))
    prob = w.gather(1, token[:, None])[:, 0] / c[:, -1]
    return dict(token=token.to(torch.int32), prob=prob.float(), kept=kept.sum(-1).to(torch.int32))


_OWN = dict(plan=_own_plan, qkv=_own_qkv, attend=_own_attend, sample=_own_sample)
_PLAIN = dict(plan=_plain_plan, qkv=_plain_qkv, attend=_plain_attend, sample=_plain_sample)


def run(state):
    return (_OWN if own else _PLAIN)[state["op"]](state)


# ---------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    c = case
    if c["op"] == "plan":
        B, T = c["B"], c["B"] * c["max_new"]
        table = B * (-(-(c["max_cached"] / 2 + c["max_new"] / 2) // c["page"]))
        return dict(bytes=4.0 * (B * 4 + 2 * T + table), flops=0.0)
    if c["op"] == "qkv":
        e = 2 if c["x"] == "bf16" else 4
        n = c["T"] * c["d"]
        if c["form"] == "dense":
            return dict(bytes=float(n * (c["Hq"] + c["Hkv"]) * 2 * e + 4 * c["T"]), flops=6.0 * n * (c["Hq"] + c["Hkv"]))
        return dict(bytes=float(n * (c["Hq"] + 2 * c["Hkv"]) * (e + 2) + 8 * c["T"]), flops=6.0 * n * (c["Hq"] + c["Hkv"]))
    if c["op"] == "attend":
        # expected sums over the requests' lengths: new in [max_q/2, max_q], cached in [cached/4, cached] when ragged
        B = c["B"]
        new = 0.75 * c["max_q"] + 0.5 if c["ragged"] and c["max_q"] > 1 else c["max_q"]
        cached = 0.625 * c["cached"] if c["ragged"] else c["cached"]
        e = 2 if c["cache"] == "bf16" else 1
        seen = cached + (new / 2 if c["causal"] else new)
        return dict(bytes=float(B * (cached + new) * c["Hkv"] * c["d"] * 2 * e + B * new * c["Hq"] * c["d"] * (4 if c["out"] == "bf16" else 6)),
                    flops=4.0 * B * new * seen * c["Hq"] * c["d"])
    e = 2 if c["x"] == "bf16" else 4
    return dict(bytes=float(c["B"] * (c["V"] * e + 32)), flops=4.0 * c["B"] * c["V"])


# ---------------------------------------------------------------------------------------------- 64 bits
def _exact_qkv(c, s):
    Hq, Hkv, d, rot = c["Hq"], c["Hkv"], c["d"], c["rot"]
    x = s["X"].double().reshape(c["T"], Hq + 2 * Hkv, d)
    h = rot // 2
    ang = s["cs"].double()[s["pos"].long()]
    z = torch.complex(ang[:, :h], ang[:, h:])[:, None]       # the rotation as a product of complex numbers

    def head(y, w):
        if c["norm"] == "rms":
            y = y / torch.sqrt(torch.linalg.vector_norm(y, dim=-1, keepdim=True) ** 2 / d + s["eps"]) * w.double()
        elif c["norm"] == "l2":
            y = y / torch.linalg.vector_norm(y, dim=-1, keepdim=True).clamp(min=s["eps"]) * w.double()
        y = y.clone()
        i = torch.arange(h, device=DEV)
        a, b = (i, i + h) if c["rope"] == "half" else (2 * i, 2 * i + 1)
        r = torch.complex(y[..., a], y[..., b]) * z
        y[..., a], y[..., b] = r.real, r.imag
        return y

    q, k = head(x[:, :Hq], s["wq"]), head(x[:, Hq:Hq + Hkv], s["wk"])
    if c["form"] == "dense":
        return dict(q=q, k=k)
    page = c["page"]
    out = {}
    for name, val, pool in (("k", k, s["Kp"]), ("v", x[:, Hq + Hkv:], s["Vp"])):
        flat = pool.double().transpose(1, 2).reshape(-1, Hkv, d)     # [slot, head, d]
        flat.index_copy_(0, s["slots"].long(), val)
        out[name] = flat.view(-1, page, Hkv, d).transpose(1, 2).contiguous()
    return dict(q=q, **out)


def _exact_attend(c, s):
    new = (s["cu"][1:] - s["cu"][:-1]).tolist()
    kv = s["kv"].tolist()
    Hkv, d, page, g = c["Hkv"], c["d"], c["page"], s["g"]
    out = torch.zeros(s["Q"].shape, device=DEV, dtype=torch.float64)
    t0 = 0
    for b in range(c["B"]):
        n, L = new[b], kv[b]
        at = s["table"][b, : -(-L // page)].long()
        for h in range(Hkv):
            k = s["Kp"][at, h].reshape(-1, d)[:L].double()
            v = s["Vp"][at, h].reshape(-1, d)[:L].double()
            if s["s_k"] is not None:
                k, v = k * s["s_k"][:L, None].double(), v * s["s_v"][h].double()
            q = s["Q"][t0:t0 + n, h * g:(h + 1) * g].double().transpose(0, 1)      # [g, n, d]
            x = (q @ k.T) * s["scale"]
            if c["causal"]:
                x = x + torch.full((n, L), float("-inf"), device=DEV, dtype=torch.float64).triu(L - n + 1)
            out[t0:t0 + n, h * g:(h + 1) * g] = (torch.softmax(x, -1) @ v).transpose(0, 1)
        t0 += n
    return dict(o=out)


def _exact_sample(c, s):
    X, u = s["X"].double().cpu().numpy(), s["u"].double().cpu().numpy()
    T, P, M = (s[n].double().cpu().numpy() for n in ("temp", "top_p", "min_p"))
    prob = np.zeros(c["B"])
    for r in range(c["B"]):
        x = X[r]
        cand = np.lexsort((np.arange(x.size), -x))
        if c["top_k"] > 0:
            cand = cand[: c["top_k"]]
        w = np.exp((x[cand] - x[cand[0]]) / T[r])
        if P[r] < 1:
            n = int(np.searchsorted(np.cumsum(w), P[r] * w.sum())) + 1
            cand, w = cand[:n], w[:n]
        cand, w = cand[w >= M[r]], w[w >= M[r]]
        by = np.argsort(cand)
        c_ = np.cumsum(w[by])
        at = min(int(np.searchsorted(c_, u[r] * c_[-1], side="right")), c_.size - 1)
        prob[r] = w[by][at] / c_[-1]
    return dict(token=None, prob=torch.from_numpy(prob), kept=None)


def exact(case, seed):
    if case["op"] == "plan":
        return None
    s = prepare(case, seed)
    return dict(qkv=_exact_qkv, attend=_exact_attend, sample=_exact_sample)[case["op"]](case, s)
