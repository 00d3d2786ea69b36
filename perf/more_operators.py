"""The operators around the attention of a decoder's step as measured cases: the norms before and after a block with
its gate and residual, few-row products with 4-bit weights and group scales, and log probabilities of given tokens.

`own` false: each operator in its plain form (elementary torch operations, fp32). `own` true: the calls a user's
program makes of the library. Both work on what `prepare` returns. `exact` gives the floating outputs in 64 bits,
written apart from the plain form.
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
        # one decode step of a small batch in a text decoder with norms on both sides of the block: RMS, learned weights
        dict(name="norm 4 x 4096", op="norm", M=4, C=4096, h="bf16", o="bf16", y="bf16", post="rms", pre="rms", G=0, affine=True),
        # raster-order decode of 256 images (2048 wide), each with its own class vector: gate, scale and shift per row
        dict(name="norm 256 x 2048", op="norm", M=256, C=2048, h="f32", o="bf16", y="bf16", post="none", pre="layer", G=256, affine=False),
        # a scale of the VAR-d30 pyramid: 32 samples x 256 tokens, the norm emits the next linear's 8-bit codes
        dict(name="norm 8192 x 1920 codes", op="norm", M=8192, C=1920, h="bf16", o="bf16", y="codes", post="none", pre="layer", G=32, affine=False),
        # MAR-Huge prefill: 256 tokens of 256 samples, fp32 residual stream
        dict(name="norm 65536 x 1280", op="norm", M=65536, C=1280, h="f32", o="bf16", y="bf16", post="none", pre="layer", G=256, affine=False),
        # raster-order decode of one image: the MLP's first linear (2048 -> 8192, GELU)
        dict(name="w4 1 x 2048 > 8192", op="w4", M=1, K=2048, N=8192, group=128, x="bf16", s="f32", act="gelu", y="bf16"),
        # the second linear of the same MLP for eight images (8192 -> 2048), finer groups
        dict(name="w4 8 x 8192 > 2048", op="w4", M=8, K=8192, N=2048, group=64, x="bf16", s="f32", act="none", y="bf16"),
        # qkv of VAR-d30's width for the ragged rest of a batch, fp32 activations
        dict(name="w4 13 x 1920 > 5760", op="w4", M=13, K=1920, N=5760, group=32, x="f32", s="bf16", act="none", y="f32"),
        # head linear of a text-sized vocabulary, logits in fp32
        dict(name="w4 4 x 4096 > 128000", op="w4", M=4, K=4096, N=128000, group=128, x="bf16", s="bf16", act="none", y="f32"),
        # one image's codebook token: its log probability, entropy and the five likeliest
        dict(name="logprob 1 x 16384", op="logprob", B=1, V=16384, x="f32", k=5, temp=True, masked=0.0),
        # raster-order decode of 256 images over the codebook
        dict(name="logprob 256 x 16384", op="logprob", B=256, V=16384, x="bf16", k=5, temp=True, masked=0.0),
        # a served step of eight requests, constrained to part of a text-sized vocabulary, twenty alternatives
        dict(name="logprob 8 x 128000", op="logprob", B=8, V=128000, x="f32", k=20, temp=True, masked=0.3),
        # scoring prompts: log probability, rank and entropy of 4096 given tokens
        dict(name="logprob 4096 x 128000", op="logprob", B=4096, V=128000, x="bf16", k=0, temp=False, masked=0.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "w4", "logprob"])
    if op == "norm":
        C = 8 * _log_int(rng, 8, 1024)
        M = _log_int(rng, 1, min(32768, 60_000_000 // C))
        return dict(op="norm", M=M, C=C, h=rng.choice(["bf16", "f32"]), o=rng.choice(["bf16", "f32", "none"]), y=rng.choice(["bf16", "f32", "codes"]),
                    post=rng.choice(["none", "rms", "layer"]), pre=rng.choice(["rms", "layer"]), G=rng.choice([0, 1, 7, 64]), affine=rng.random() < 0.5)
    if op == "w4":
        group = rng.choice([32, 64, 96, 128, 256])
        K = group * _log_int(rng, 2, max(2, 8192 // group))
        return dict(op="w4", M=_log_int(rng, 1, 64), K=K, N=_log_int(rng, 64, 20000), group=group, x=rng.choice(["bf16", "bf16", "f32"]),
                    s=rng.choice(["f32", "bf16"]), act=rng.choice(["none", "gelu"]), y=rng.choice(["bf16", "f32"]))
    V = _log_int(rng, 100, 200000)
    return dict(op="logprob", B=_log_int(rng, 1, max(1, min(2048, 60_000_000 // V))), V=V, x=rng.choice(["bf16", "f32"]),
                k=rng.choice([0, 1, 5, 20, 32]), temp=rng.random() < 0.6, masked=rng.choice([0.0, 0.0, 0.5]))


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _prepare_norm(c, seed):
    g = _gen(seed)
    M, C, G = c["M"], c["C"], c["G"]
    n = lambda *s: torch.randn(s, device=DEV, generator=g)  # noqa: E731
    channel = torch.exp(n(C) * 0.7)                          # a residual stream has channels far above the others
    s = dict(H=(n(M, C) * channel + 0.3 * n(C)).to(_dt(c["h"])), O=None if c["o"] == "none" else n(M, C).to(_dt(c["o"])), y=c["y"],
             post=c["post"], pre=c["pre"], eps=1e-6, res_scale=1.0 if c["G"] else 0.5, cond=None, gate=None, scale=None, shift=None,
             wp=None, bp=None, w=None, b=None, pos=None, s_ch=None, s_tok=None)
    if G:                                                    # one row of a conditioning linear's output per sample: six vectors
        ada = (n(G, 6 * C) * 0.5).to(torch.bfloat16)
        s.update(gate=ada[:, :C], scale=ada[:, C:2 * C], shift=ada[:, 2 * C:3 * C])
        s["cond"] = (torch.arange(M, device=DEV) * G // M).to(torch.int32)      # a sample's rows stand together
    if c["affine"]:
        s.update(w=torch.rand((C,), device=DEV, generator=g) + 0.5, wp=torch.rand((C,), device=DEV, generator=g) + 0.5)
        if c["pre"] == "layer":
            s["b"] = n(C) * 0.1
        if c["post"] == "layer":
            s["bp"] = n(C) * 0.1
    s["Ho"] = None if s["O"] is None else torch.empty_like(s["H"])
    s["Y"] = torch.empty((M, C), device=DEV, dtype=torch.int8 if c["y"] == "codes" else _dt(c["y"]))
    if c["y"] == "codes":
        P = 680
        s.update(pos=torch.randint(0, P, (M,), device=DEV, generator=g, dtype=torch.int32), s_ch=torch.exp(n(C) * 0.3),
                 s_tok=(torch.rand((P,), device=DEV, generator=g) + 0.6) / 32, V=torch.empty((M, C), device=DEV, dtype=torch.bfloat16))
    return s


def _prepare_w4(c, seed):
    g = _gen(seed)
    M, K, N = c["M"], c["K"], c["N"]
    code = torch.empty((N, K), device=DEV, dtype=torch.bfloat16).normal_(generator=g).mul_(2.8).round_().clamp_(-8, 7).to(torch.int8)
    code = (code & 15).view(torch.uint8)
    s = dict(X=torch.randn((M, K), device=DEV, generator=g).mul_(1.5).to(_dt(c["x"])), Wp=(code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(),
             s_g=((torch.rand((N, K // c["group"]), device=DEV, generator=g) + 0.5) * 0.008).to(_dt(c["s"])),
             bias=torch.randn((N,), device=DEV, generator=g) * 0.02, act=c["act"], group=c["group"],
             Y=torch.empty((M, N), device=DEV, dtype=_dt(c["y"])))
    return s


def _prepare_logprob(c, seed):
    g = _gen(seed)
    B, V, k = c["B"], c["V"], c["k"]
    X = torch.randn((B, V), device=DEV, generator=g, dtype=torch.bfloat16 if c["x"] == "bf16" else torch.float32).mul_(2.5)
    if c["masked"] > 0:                                      # the tokens that a grammar forbids at this place
        X.masked_fill_(torch.rand((V,), device=DEV, generator=g) < c["masked"], float("-inf"))
    T = torch.rand((B,), device=DEV, generator=g) * 0.7 + 0.5 if c["temp"] else None
    if c["temp"]:                                            # tokens drawn from the distribution
        z = X.float() / T[:, None]
        noise = torch.empty_like(z).exponential_(generator=g).clamp_(min=1e-30)
        tokens = z.sub_(noise.log_()).argmax(-1)
    else:                                                    # tokens of a prompt; rows behind the last sequence have none
        tokens = torch.randint(0, V, (B,), device=DEV, generator=g)
        tokens[B - B // 32:] = -1
    s = dict(X=X, T=T, tokens=tokens.to(torch.int32), k=k, logprob=torch.empty((B,), device=DEV), rank=torch.empty((B,), device=DEV, dtype=torch.int32),
             entropy=torch.empty((B,), device=DEV), top=None, toplp=None)
    if k:
        s.update(top=torch.empty((B, k), device=DEV, dtype=torch.int32), toplp=torch.empty((B, k), device=DEV))
    return s


_PREPARE = dict(norm=_prepare_norm, w4=_prepare_w4, logprob=_prepare_logprob)


def prepare(case, seed):
    s = _PREPARE[case["op"]](case, int(seed))
    s["op"] = case["op"]
    return s


# ---------------------------------------------------------------------------------------------- the library's calls
_NORM = dict(none=0, rms=1, layer=3)


def _own_norm(s):
    _context().block_norm(s["H"], s["O"], s["cond"], s["gate"], s["scale"], s["shift"], _NORM[s["post"]], s["wp"], s["bp"], s["res_scale"],
                          _NORM[s["pre"]], s["w"], s["b"], s["eps"], s["Ho"], s["pos"], s["s_ch"], s["s_tok"], 8, s["Y"])
    if s["y"] != "codes":
        return dict(h=s["Ho"], y=s["Y"])
    torch.mul(s["Y"], s["s_tok"][s["pos"].long()][:, None], out=s["V"])      # the values that the codes stand for
    return dict(h=s["Ho"], y=s["V"])


def _own_w4(s):
    _context().linear_w4g(s["X"], s["Wp"], s["s_g"], s["bias"], 1 if s["act"] == "gelu" else 0, 1 if s["Y"].dtype == torch.bfloat16 else 0, s["Y"])
    return dict(y=s["Y"])


def _own_logprob(s):
    _context().token_logprobs(s["X"], s["T"], s["tokens"], s["logprob"], s["rank"], s["entropy"], s["top"], s["toplp"])
    return dict(logprob=s["logprob"], rank=s["rank"], entropy=s["entropy"], top=s["top"], toplp=s["toplp"])


# ---------------------------------------------------------------------------------------------- the plain forms
def _plain_norm_of(x, kind, w, b, eps):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    if kind != "none":
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
    if w is not None:
        x = x * w
    return x if b is None else x + b


def _plain_norm(s):
    h = s["H"].float()
    at = None if s["cond"] is None else s["cond"].long()
    if s["O"] is not None:
        o = _plain_norm_of(s["O"].float(), s["post"], s["wp"], s["bp"], s["eps"]) * s["res_scale"]
        h = h + (o if at is None else o * s["gate"].float()[at])
    y = _plain_norm_of(h, s["pre"], s["w"], s["b"], s["eps"])
    if at is not None:
        y = y * (1 + s["scale"].float()[at]) + s["shift"].float()[at]
    ho = None if s["O"] is None else h.to(s["H"].dtype)
    if s["y"] != "codes":
        return dict(h=ho, y=y.to(s["Y"].dtype))
    step = s["s_tok"][s["pos"].long()][:, None]
    code = torch.round((y * (1 / s["s_ch"])) * (1 / step)).clamp(-128, 127)
    return dict(h=ho, y=(code * step).to(torch.bfloat16))


def _plain_w4(s):
    p = s["Wp"]
    w = torch.stack([p & 15, p >> 4], -1).flatten(1).to(torch.float32)
    w = torch.where(w > 7, w - 16, w)
    w = (w.view(w.shape[0], -1, s["group"]) * s["s_g"].float()[:, :, None]).flatten(1)
    y = torch.matmul(s["X"].float(), w.T) + s["bias"]
    if s["act"] == "gelu":
        y = 0.5 * y * (1 + torch.erf(y * 0.7071067811865476))
    return dict(y=y.to(s["Y"].dtype))


def _plain_logprob(s):
    x = s["X"].float() + 0.0
    B, V = x.shape
    x = torch.where(x > float("-inf"), x, float("-inf"))     # NaN counts as masked
    t = s["tokens"].long()[:, None]
    given = t >= 0
    t = t.clamp(min=0)
    xt = x.gather(1, t)
    rank = (x > xt).sum(-1, keepdim=True) + ((x == xt) & (torch.arange(V, device=DEV) < t)).sum(-1, keepdim=True)
    rank = torch.where(given & (xt > float("-inf")), rank, -1)[:, 0].to(torch.int32)
    temp = torch.ones((B, 1), device=DEV) if s["T"] is None else s["T"][:, None]
    m = x.amax(-1, keepdim=True)
    top = toplp = None
    if s["k"]:
        xs, order = torch.sort(x, dim=-1, descending=True, stable=True)
        xs, order = xs[:, :s["k"]], order[:, :s["k"]]
        if s["k"] > V:
            pad = s["k"] - V
            xs, order = torch.cat([xs, xs.new_full((B, pad), float("-inf"))], 1), torch.cat([order, order.new_full((B, pad), -1)], 1)
        top = torch.where(xs > float("-inf"), order, -1).to(torch.int32)
    z = (x - m) / temp
    w = torch.exp(z)
    total = w.sum(-1, keepdim=True)
    log_total = torch.log(total)
    entropy = (log_total - (w * z.clamp(min=-1e30)).sum(-1, keepdim=True) / total)[:, 0]
    if s["k"]:
        toplp = (xs - m) / temp - log_total
    logprob = torch.where(given, (xt - m) / temp - log_total, 0.0)[:, 0]
    return dict(logprob=logprob, rank=rank, entropy=entropy, top=top, toplp=toplp)


_OWN = dict(norm=_own_norm, w4=_own_w4, logprob=_own_logprob)
_PLAIN = dict(norm=_plain_norm, w4=_plain_w4, logprob=_plain_logprob)


def run(state):
    return (_OWN if own else _PLAIN)[state["op"]](state)


# ---------------------------------------------------------------------------------------------- what a pass needs
_BYTES = dict(bf16=2, f32=4, codes=1, none=0)


def work(case):
    c = case
    if c["op"] == "norm":
        MC, C = c["M"] * c["C"], c["C"]
        per = _BYTES[c["h"]] * (2 if c["o"] != "none" else 1) + _BYTES[c["o"]] + _BYTES[c["y"]]
        side = (6 * c["G"] * C + 4 * c["M"] if c["G"] else 0) + (8 * C if c["affine"] else 0) + (8 * c["M"] + 4 * C if c["y"] == "codes" else 0)
        return dict(bytes=float(MC * per + side), flops=16.0 * MC)
    if c["op"] == "w4":
        M, K, N = c["M"], c["K"], c["N"]
        return dict(bytes=float(N * K / 2 + N * (K // c["group"]) * _BYTES[c["s"]] + M * K * _BYTES[c["x"]] + M * N * _BYTES[c["y"]] + 4 * N),
                    flops=2.0 * M * N * K)
    return dict(bytes=float(c["B"] * (c["V"] * _BYTES[c["x"]] + 20 + 8 * c["k"])), flops=6.0 * c["B"] * c["V"])


# ---------------------------------------------------------------------------------------------- 64 bits
def _exact_norm(c, s):
    def norm(x, kind, w, b):
        if kind == "rms":
            x = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / c["C"] + s["eps"])
        elif kind == "layer":
            var, mean = torch.var_mean(x, dim=-1, keepdim=True, correction=0)
            x = (x - mean) / torch.sqrt(var + s["eps"])
        return x * (1.0 if w is None else w.double()) + (0.0 if b is None else b.double())

    parts_h, parts_y = [], []
    for r0 in range(0, c["M"], 8192):                        # rows at a time: 64-bit copies of all would take many GB
        r = slice(r0, min(r0 + 8192, c["M"]))
        h = s["H"][r].double()
        ids = s["cond"][r].long() if c["G"] else None
        if s["O"] is not None:
            branch = norm(s["O"][r].double(), c["post"], s["wp"], s["bp"])
            h = torch.addcmul(h, branch, s["gate"].double()[ids], value=s["res_scale"]) if c["G"] else torch.add(h, branch, alpha=s["res_scale"])
        y = norm(h, c["pre"], s["w"], s["b"])
        if c["G"]:
            y = y + y * s["scale"].double()[ids] + s["shift"].double()[ids]
        if c["y"] == "codes":
            step = s["s_tok"].double()[s["pos"][r].long()].unsqueeze(1)
            y = torch.clamp(torch.round(y / (s["s_ch"].double() * step)), -128, 127) * step
        parts_h.append(h)
        parts_y.append(y)
    return dict(h=None if s["O"] is None else torch.cat(parts_h), y=torch.cat(parts_y))


def _exact_w4(c, s):
    table = torch.tensor([0, 1, 2, 3, 4, 5, 6, 7, -8, -7, -6, -5, -4, -3, -2, -1], device=DEV, dtype=torch.float64)
    X, out = s["X"].double(), []
    for n0 in range(0, c["N"], 16384):
        p = s["Wp"][n0:n0 + 16384].long()
        w = torch.empty((p.shape[0], c["K"]), device=DEV, dtype=torch.float64)
        w[:, 0::2], w[:, 1::2] = table[p % 16], table[torch.div(p, 16, rounding_mode="floor")]
        w *= s["s_g"][n0:n0 + 16384].double().repeat_interleave(c["group"], dim=1)
        out.append(X @ w.T + s["bias"][n0:n0 + 16384].double())
    y = torch.cat(out, 1)
    if c["act"] == "gelu":
        y = y * torch.special.ndtr(y)
    return dict(y=y)


def _exact_logprob(c, s):
    lp, ent, top = [], [], []
    for b0 in range(0, c["B"], 256):
        x = s["X"][b0:b0 + 256].double()
        x = x.masked_fill(torch.isnan(x), -math.inf)
        if s["T"] is not None:
            x = x / s["T"][b0:b0 + 256].double()[:, None]
        logp = x - torch.logsumexp(x, 1, keepdim=True)
        t = s["tokens"][b0:b0 + 256].long()
        lp.append(torch.where(t < 0, 0.0, logp.gather(1, t.clamp(min=0)[:, None])[:, 0]))
        ent.append(-torch.xlogy(logp.exp(), logp.exp()).sum(1))
        if c["k"]:
            v = torch.topk(logp, min(c["k"], c["V"]), dim=1).values
            top.append(torch.nn.functional.pad(v, (0, c["k"] - v.shape[1]), value=-math.inf))
    return dict(logprob=torch.cat(lp), rank=None, entropy=torch.cat(ent), top=None, toplp=torch.cat(top) if c["k"] else None)


def exact(case, seed):
    s = prepare(case, seed)
    return dict(norm=_exact_norm, w4=_exact_w4, logprob=_exact_logprob)[case["op"]](case, s)
