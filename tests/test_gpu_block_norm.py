"""block_norm on the GPU against its formula in 64 bits, with bounds that follow the fp32 roundings of the kernel."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24          # half a step of fp32, relative
# longest chain of additions in a sum over a row: 8 channels of 4 vectors in a thread, 5 steps in a warp, 16 warps in fours
DEPTH = 32 + 5 + 6


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
    yield g
    ctx.close()


def norm_ref(x, e, kind, w, b, eps):
    """N(x) w + b in float64 and a bound on the error of the fp32 kernel, given a bound e on the error of x."""
    C = x.shape[-1]
    if kind == 0:
        n, en = x, e
    else:
        mean = x.mean(-1, keepdims=True) if kind == 3 else 0.0 * x[:, :1]
        c = x - mean
        r = 1 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
        n = c * r
        # the mean: DEPTH additions, the product with 1 / C (itself rounded); the difference: half a step
        off = e + ((DEPTH + 2) * U * np.abs(x).mean(-1, keepdims=True) + e.mean(-1, keepdims=True) if kind == 3 else 0.0) + U * np.abs(c)
        # the squares' sum: DEPTH additions and a product each, 1 / C, eps, rsqrt (2 steps, i.e. 4 U); halved by the root, and what `off`
        # does to it: |d r / r| <= r sqrt(mean off^2)
        rel = (DEPTH + 4) / 2 * U + 4 * U + r * np.sqrt((off * off).mean(-1, keepdims=True))
        en = r * off + np.abs(n) * (rel + U)
    if w is not None:
        n = n * w
        en = en * np.abs(w) + U * np.abs(n)
    if b is not None:
        n = n + b
        en = en + U * np.abs(n)
    return n, en


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def reference(a):
    """Outputs of block_norm in float64 with their bounds, before the rounding of a store."""
    h = f64(a["H"])
    M, C = h.shape
    e = np.zeros_like(h)
    cond = np.zeros(M, np.int64) if a["cond_ids"] is None else a["cond_ids"].cpu().numpy().astype(np.int64)
    row = lambda t: None if t is None else f64(t)[cond]  # noqa: E731
    if a["O"] is not None:
        o, eo = norm_ref(f64(a["O"]), e, a["post_norm"], f64(a["w_post"]), f64(a["b_post"]), a["eps"])
        g = float(np.float32(a["res_scale"])) * (1.0 if a["gate"] is None else row(a["gate"]))
        h, e = h + g * o, np.abs(g) * eo + np.abs(g * o) * U + U * np.abs(h + g * o)
    y, ey = norm_ref(h, e, a["pre_norm"], f64(a["w_pre"]), f64(a["b_pre"]), a["eps"])
    if a["scale"] is not None:
        s = 1 + row(a["scale"])
        y, ey = y * s, ey * np.abs(s) + 2 * U * np.abs(y * s)
    if a["shift"] is not None:
        y = y + row(a["shift"])
        ey = ey + U * np.abs(y)
    if a["s_ch"] is not None:
        r = 1 / f64(a["s_ch"])
        y, ey = y * r, ey * r + 2 * U * np.abs(y * r)
    return h, e, y, ey


def check_store(got, want, bound, bf16):
    got = got.double().cpu().numpy()
    tol = bound + (2.0 ** -8 * (np.abs(want) + bound) if bf16 else 0.0)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), float(np.abs(got - want)[bad].max()), float(tol[bad].max()))


def make(gpu, M, C, h="f32", o="bf16", y="bf16", post=0, pre=3, G=0, w=True, cond="bf16", seed=0, s_ch=False):
    torch, dev = gpu.torch, gpu.dev
    g = torch.Generator(device=dev).manual_seed(seed * 1000 + M * 7 + C)
    n = lambda *s: torch.randn(s, device=dev, generator=g)  # noqa: E731
    dt = dict(f32=torch.float32, bf16=torch.bfloat16, i8=torch.int8)
    a = dict(H=(n(M, C) * torch.exp(n(C)) + 0.5).to(dt[h]), O=None if o is None else n(M, C).to(dt[o]), cond_ids=None, gate=None, scale=None, shift=None,
             post_norm=post, w_post=n(C) if w else None, b_post=n(C) * 0.1 if w else None, res_scale=0.7, pre_norm=pre, w_pre=n(C) if w else None,
             b_pre=n(C) * 0.1 if w else None, eps=1e-5, Hout=None, pos_ids=None, s_ch=None, s_tok=None, bits=8, Y=None)
    if G:
        ada = (n(G, 6 * C) * 0.6).to(dt[cond])
        a.update(gate=ada[:, 2 * C:3 * C], scale=ada[:, :C], shift=ada[:, 5 * C:])
        if G > 1 or seed % 2:
            a["cond_ids"] = torch.randint(0, G, (M,), device=dev, generator=g, dtype=torch.int32)
    if o is not None:
        a["Hout"] = torch.full((M, C), 7.0, device=dev).to(dt[h])
    if y is not None:
        a["Y"] = torch.full((M, C), 7.0, device=dev).to(dt[y])
    if s_ch or y == "i8":
        a["s_ch"] = torch.exp(n(C) * 0.3)
    if y == "i8":
        P = 37
        a.update(pos_ids=torch.randint(0, P, (M,), device=dev, generator=g, dtype=torch.int32), s_tok=(torch.rand((P,), device=dev, generator=g) + 0.5) / 30)
    return a


def run_and_check(gpu, a):
    keep = {k: v.clone() for k, v in a.items() if isinstance(v, gpu.torch.Tensor)}
    h, e, y, ey = reference(a)
    gpu.ctx.block_norm(**a)
    assert gpu.ctx.stwq_device_status() == 0
    bf = gpu.torch.bfloat16
    if a["Hout"] is not None:
        check_store(a["Hout"], h, e, a["H"].dtype == bf)
    if a["Y"] is not None and a["Y"].dtype != gpu.torch.int8:
        check_store(a["Y"], y, ey, a["Y"].dtype == bf)
    elif a["Y"] is not None:
        rt = 1 / f64(a["s_tok"])[a["pos_ids"].cpu().numpy()][:, None]
        top = 127 if a["bits"] == 8 else 31
        u, eu = y * rt, ey * rt + 2 * U * np.abs(y * rt)
        code = a["Y"].cpu().numpy().astype(np.float64)
        assert (np.abs(code - np.clip(u, -top - 1, top)) <= 0.5 + eu).all()
        assert (code == np.clip(np.rint(u), -top - 1, top)).mean() > 0.999
    return keep


@pytest.mark.parametrize("M,C", [(1, 8), (1, 1024), (3, 72), (5, 256), (4, 264), (2, 512), (7, 520), (130, 1280), (33, 1920), (300, 2048), (9, 4096), (6, 4104), (3, 8192),
                                 (2, 8200), (2, 16384), (2500, 64)])
@pytest.mark.parametrize("post,pre", [(0, 3), (1, 1), (3, 0)])
def test_sizes_and_norms(gpu, M, C, post, pre):
    run_and_check(gpu, make(gpu, M, C, post=post, pre=pre, G=3 if M > 1 else 1, seed=post + pre))


@pytest.mark.parametrize("h", ["f32", "bf16"])
@pytest.mark.parametrize("o", ["f32", "bf16", None])
@pytest.mark.parametrize("y", ["f32", "bf16", "i8", None])
@pytest.mark.parametrize("cond", ["f32", "bf16"])
def test_types(gpu, h, o, y, cond):
    if o is None and y is None:
        pytest.skip("nothing to compute")
    for C in (200, 1920):
        run_and_check(gpu, make(gpu, 21, C, h=h, o=o, y=y, G=5, cond=cond, seed=3, s_ch=True))


def test_vectors_left_out(gpu):
    for drop in (("gate",), ("scale",), ("shift",), ("gate", "scale", "shift"), ("w_post",), ("b_pre", "w_pre"), ("b_post", "gate")):
        a = make(gpu, 19, 640, post=3, G=4, seed=5)
        a.update({k: None for k in drop})
        if drop == ("gate", "scale", "shift"):
            a["cond_ids"] = None
        run_and_check(gpu, a)
    a = make(gpu, 19, 640, post=1, G=1, seed=2)              # one row of gates for all rows: a scale per channel
    assert a["cond_ids"] is None
    a["scale"] = a["shift"] = None
    run_and_check(gpu, a)


def test_six_bit_codes_and_the_linear_that_takes_them(gpu):
    a = make(gpu, 50, 1024, y="i8", G=2)
    a["bits"] = 6
    a["s_tok"] = a["s_tok"] * 4
    run_and_check(gpu, a)


def test_codes_are_those_of_the_quantizer(gpu):
    """The codes equal those that the library's quantizer gives on the floating output of the same call."""
    a = make(gpu, 300, 1920, y="i8", G=4, seed=4)
    gpu.ctx.block_norm(**a)
    b = dict(a, Y=gpu.torch.empty((300, 1920), device=gpu.dev), s_ch=None)
    gpu.ctx.block_norm(**b)
    want = gpu.torch.empty((300, 1920), device=gpu.dev, dtype=gpu.torch.int8)
    gpu.ctx.stwq_quantize(b["Y"], a["pos_ids"], a["s_ch"], a["s_tok"], 8, want)
    assert gpu.torch.equal(a["Y"], want)


def test_strided_rows_and_in_place(gpu):
    torch = gpu.torch
    for C in (96, 1280):
        a = make(gpu, 23, C, G=3, seed=7)
        wide = torch.full((23, 3 * C + 32), 9.0, device=gpu.dev)
        wide[:, C:2 * C] = a["H"]
        a["H"], a["Hout"] = wide[:, C:2 * C], wide[:, 2 * C:3 * C]                 # side by side in one buffer
        y = torch.full((23, 2 * C), 5.0, device=gpu.dev, dtype=torch.bfloat16)
        a["Y"] = y[:, C:]
        run_and_check(gpu, a)
        assert (wide[:, :C] == 9).all() and (wide[:, 3 * C:] == 9).all() and (y[:, :C] == 5).all()
        b = make(gpu, 23, C, h="bf16", G=3, seed=8)                               # the sum replaces H, the output replaces O
        first = {k: b[k].clone() for k in ("H", "O")}
        gpu.ctx.block_norm(**b)
        c = dict(b, H=first["H"].clone(), O=first["O"].clone())
        c["Hout"], c["Y"] = c["H"], c["O"]
        gpu.ctx.block_norm(**c)
        assert torch.equal(c["H"], b["Hout"]) and torch.equal(c["O"], b["Y"])
        d = dict(b, H=first["H"].clone(), O=None, Hout=None)
        d["Y"] = d["H"]
        e = dict(d, H=first["H"].clone(), Y=torch.empty_like(first["H"]))
        gpu.ctx.block_norm(**d)
        gpu.ctx.block_norm(**e)
        assert torch.equal(d["Y"], e["Y"])


def test_padding_rows_are_left_as_they_were(gpu):
    torch = gpu.torch
    for C, y in ((128, "bf16"), (1920, "i8"), (1920, "f32")):
        a = make(gpu, 40, C, y=y, G=3, seed=9)
        pos = torch.arange(40, device=gpu.dev, dtype=torch.int32) % 37
        pos[5], pos[17:20], pos[35:] = -1, -1, -1
        live = pos >= 0
        a["pos_ids"] = pos
        full = dict(a, pos_ids=pos.clamp(min=0), Hout=a["Hout"].clone(), Y=a["Y"].clone())
        a["H"][~live], a["O"][~live] = float("nan"), float("nan")
        a["cond_ids"][~live] = 99
        full["cond_ids"] = a["cond_ids"].clamp(max=2)
        gpu.ctx.block_norm(**a)
        assert gpu.ctx.stwq_device_status() == 0
        gpu.ctx.block_norm(**full)
        assert torch.equal(a["Hout"][live], full["Hout"][live]) and torch.equal(a["Y"][live], full["Y"][live])
        assert (a["Hout"][~live] == 7).all() and (a["Y"][~live] == 7).all()


def test_ids_out_of_range_are_reported(gpu):
    torch, ERR = gpu.torch, -8
    for C in (64, 1280):
        a = make(gpu, 12, C, y="i8", G=3, seed=11)
        a["cond_ids"][4], a["cond_ids"][9] = 3, -2
        a["pos_ids"][2] = 37
        b = dict(a, cond_ids=a["cond_ids"].clamp(0, 2), pos_ids=a["pos_ids"].clamp(max=36), Hout=a["Hout"].clone(), Y=a["Y"].clone())
        gpu.ctx.block_norm(**a)
        assert gpu.ctx.stwq_device_status() == ERR and gpu.ctx.stwq_device_status() == 0
        gpu.ctx.block_norm(**b)
        rows = torch.ones(12, dtype=torch.bool, device=gpu.dev)
        rows[[4, 9, 2]] = False
        assert torch.equal(a["Y"][rows], b["Y"][rows]) and (a["Y"][~rows] == 0).all()
        rows[2] = True
        assert torch.equal(a["Hout"][rows], b["Hout"][rows]) and torch.equal(a["Hout"][[4, 9]], a["H"][[4, 9]])


def test_nan_inf_and_constant_rows(gpu):
    torch, nan, inf = gpu.torch, float("nan"), float("inf")
    for C in (64, 1280):
        a = make(gpu, 6, C, y="f32", w=False, post=0, pre=3, seed=12)
        a["O"].zero_()
        a["H"][0], a["H"][1, 3], a["H"][2, 5], a["H"][3] = 4.0, nan, inf, 0.0
        gpu.ctx.block_norm(**a)
        y = a["Y"]
        assert (y[0] == 0).all() and (y[3] == 0).all()                      # nothing but the mean: 0 / sqrt(eps)
        assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all() and torch.isfinite(y[4:]).all()
        a["pre_norm"] = 1
        gpu.ctx.block_norm(**a)
        assert torch.isnan(y[1]).all() and torch.isnan(y[2, 5]) and (y[2, :5] == 0).all() and (y[3] == 0).all()
        a["pre_norm"] = 0
        gpu.ctx.block_norm(**a)
        assert torch.isnan(y[1, 3]) and y[2, 5] == inf and torch.isfinite(y[2, :5]).all()
        b = make(gpu, 2, C, y="i8", w=False, seed=13)
        b["H"][0, 1] = nan
        gpu.ctx.block_norm(**b)
        assert (b["Y"][0] == 0).all() and gpu.ctx.stwq_device_status() == 0


def test_refusals(gpu):
    torch, pk = gpu.torch, gpu.pk
    ok = make(gpu, 8, 64, G=2, seed=1)

    def refused(code, **k):
        a = dict(ok, **k)
        with pytest.raises(pk.StwqError) as e:
            gpu.ctx.block_norm(**a)
        assert e.value.code == code
    z = lambda *s, dt=torch.float32: torch.zeros(s, device=gpu.dev, dtype=dt)  # noqa: E731
    refused(-1, Hout=None, Y=None)
    refused(-1, O=None)                                                     # nothing to add, but a place for the sum
    refused(-4, pre_norm=pk.NORM_L2)
    refused(-4, post_norm=7)
    refused(-2, eps=-1.0)
    refused(-2, eps=float("nan"))
    refused(-1, Y=z(8, 64, dt=torch.int8))                                  # codes without scales
    refused(-4, Y=z(8, 64, dt=torch.int8), pos_ids=z(8, dt=torch.int32), s_tok=z(3) + 1, bits=4)
    buf = z(9, 64)
    refused(-3, H=buf[:8], Hout=buf[1:])                                    # one row further: another row's input
    refused(-3, Hout=ok["H"], Y=ok["H"])
    half = z(8, 64, dt=torch.bfloat16)
    refused(-3, O=half, Hout=None, Y=half.view(torch.int8)[:, :64], pos_ids=z(8, dt=torch.int32), s_tok=z(3) + 1)   # codes over the branch
    a = make(gpu, 8, 64, seed=1)
    big = z(8, 130)
    with pytest.raises(pk.StwqError) as e:                                  # rows that are not 16-byte aligned
        gpu.ctx.block_norm(**dict(a, H=big[:, :64]))
    assert e.value.code == -3
    with pytest.raises(pk.StwqError) as e:
        gpu.ctx.block_norm(**dict(a, H=z(8, 68)[:, 1:65]))
    assert e.value.code == -3
    with pytest.raises(pk.StwqError) as e:
        gpu.ctx.block_norm(**make(gpu, 2, 16392))
    assert e.value.code == -2
    b = make(gpu, 8, 64, seed=1)
    with pytest.raises(pk.StwqError) as e:                                  # 12 channels
        gpu.ctx.block_norm(**{k: (v[..., :12].contiguous() if isinstance(v, torch.Tensor) else v) for k, v in b.items()})
    assert e.value.code == -3
    assert gpu.ctx.stwq_device_status() == 0
