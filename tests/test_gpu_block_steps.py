"""block_norm, linear_w4g and token_logprobs as a decoder's step uses them, next to the calls they stand beside: a whole step, eager and
captured; on a stream beside a busy default stream; rows that share a conditioning vector; and the refusals of the C entry points."""
import ctypes as C

import numpy as np
import pytest

import test_gpu_block_norm as tn
import test_gpu_logprobs as tl
import test_gpu_w4g as tw

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


class Step:
    """One layer and the head of a decoder with class-conditioned norms, B requests of one new token each over a paged cache.
    norm -> codes -> quantized qkv -> cache append -> attention -> 4-bit projection -> gate, residual, norm -> 4-bit MLP -> gate,
    residual, norm -> 4-bit head -> sampling -> log probabilities."""

    def __init__(self, gpu, B, seed):
        self.gpu, torch, pk, ctx, dev = gpu, gpu.torch, gpu.pk, gpu.ctx, gpu.dev
        g = torch.Generator(device=dev).manual_seed(seed)
        self.B, self.D, self.H, self.V, self.P, self.k = B, 256, 4, 1000, 64, 4
        D, H, d, V, P, S, W = self.D, self.H, 64, self.V, self.P, 16, 4
        n = lambda *s: torch.randn(s, device=dev, generator=g)  # noqa: E731
        e = lambda *s, dt=torch.float32: torch.zeros(s, device=dev, dtype=dt)  # noqa: E731
        i32, bf = torch.int32, torch.bfloat16
        self.h = n(B, D)
        self.ada = (n(B, 6 * D) * 0.3).to(bf)
        self.cond = torch.randperm(B, device=dev, generator=g).to(i32)
        self.s_tok = torch.rand((P,), device=dev, generator=g) * 0.01 + 0.03
        self.Wq, self.s_w, self.s_ch = e(3 * H * d, D, dt=torch.int8), e(3 * H * d), torch.exp(n(D) * 0.2)
        ctx.gps_fold(n(3 * H * d, D) * 0.06, self.s_ch, 8, self.Wq, self.s_w)

        def w4(N, K, group, dt):
            Wp, s = e(N, K // 2, dt=torch.uint8), e(N, K // group, dt=dt)
            ctx.gps_fold_group4(n(N, K) * 0.06, None, Wp, s)
            return Wp, s
        self.proj, self.fc1, self.fc2, self.head = w4(D, H * d, 32, bf), w4(4 * D, D, 64, torch.float32), w4(D, 4 * D, 128, torch.float32), w4(V, D, 256, bf)
        self.bias = n(4 * D) * 0.1
        self.Kp, self.Vp = n(B * W + B, H, S, d).to(bf), n(B * W + B, H, S, d).to(bf)
        self.cached = torch.randint(0, S * W - 1, (B,), device=dev, generator=g, dtype=i32)
        self.new = torch.ones((B,), device=dev, dtype=i32)
        self.table = torch.randperm(B * W, device=dev, generator=g).to(i32).view(B, W)
        self.free = torch.arange(B * W, B * W + B, device=dev, dtype=i32)       # a request at the end of a page takes one
        self.cu, self.kv, self.slots, self.pos, self.used = e(B + 1, dt=i32), e(B, dt=i32), e(B, dt=i32), e(B, dt=i32), e(1, dt=i32)
        self.codes, self.qkv, self.Q, self.O = e(B, D, dt=torch.int8), e(B, 3 * H * d, dt=bf), e(B, H, d, dt=bf), e(B, H, d, dt=bf)
        self.y1, self.h1, self.x2, self.a, self.y2, self.h2, self.x3 = e(B, D, dt=bf), e(B, D), e(B, D, dt=bf), e(B, 4 * D, dt=bf), e(B, D, dt=bf), e(B, D), e(B, D, dt=bf)
        self.logits, self.temp = e(B, V), torch.rand((B,), device=dev, generator=g) + 0.5
        self.u, self.tok = torch.rand((B,), device=dev, generator=g), e(B, dt=i32)
        self.lp, self.rank, self.ent, self.ids, self.tlp = e(B), e(B, dt=i32), e(B), e(B, self.k, dt=i32), e(B, self.k)
        self.cs = torch.cat([torch.cos(n(P, 32)), torch.sin(n(P, 32))], 1).contiguous()

    def norm(self, which):
        """Arguments of the three block_norm calls."""
        D, ada, pk = self.D, self.ada, self.gpu.pk
        part = lambda i: ada[:, i * D:(i + 1) * D]  # noqa: E731
        a = dict(cond_ids=self.cond, post_norm=pk.NORM_NONE, w_post=None, b_post=None, res_scale=1.0, pre_norm=pk.NORM_LAYER, w_pre=None, b_pre=None, eps=1e-6,
                 s_ch=None, s_tok=None, bits=8)
        if which == 0:
            return dict(a, H=self.h, O=None, gate=None, scale=part(0), shift=part(1), Hout=None, pos_ids=self.pos, s_ch=self.s_ch, s_tok=self.s_tok, Y=self.codes)
        if which == 1:
            return dict(a, H=self.h, O=self.y1, gate=part(2), scale=part(3), shift=part(4), Hout=self.h1, pos_ids=None, Y=self.x2)
        return dict(a, H=self.h1, O=self.y2, gate=part(5), scale=None, shift=None, pre_norm=pk.NORM_RMS, Hout=self.h2, pos_ids=self.pos, Y=self.x3)

    def run(self):
        ctx, pk, B = self.gpu.ctx, self.gpu.pk, self.B
        ctx.page_plan(self.cached, self.new, self.free, 16, self.table, self.cu, self.kv, self.slots, self.pos, self.used)
        ctx.block_norm(**self.norm(0))
        ctx.qlinear_q(self.codes, self.pos, self.Wq, self.s_w, self.s_tok, None, pk.ACT_NONE, pk.OUT_BF16, self.qkv)
        ctx.kv_append_paged(self.qkv, self.pos, self.slots, self.H, self.H, None, None, pk.NORM_L2, 1e-6, self.cs, pk.ROPE_PAIRS, None, None, 8, self.Q, self.Kp, self.Vp)
        ctx.paged_attention(self.Q, self.cu, 1, self.table, self.kv, self.Kp, self.Vp, None, None, 8.0, True, pk.OUT_BF16, self.O)
        ctx.linear_w4g(self.O.view(B, -1), *self.proj, None, pk.ACT_NONE, pk.OUT_BF16, self.y1)
        ctx.block_norm(**self.norm(1))
        ctx.linear_w4g(self.x2, *self.fc1, self.bias, pk.ACT_GELU_ERF, pk.OUT_BF16, self.a)
        ctx.linear_w4g(self.a, *self.fc2, None, pk.ACT_NONE, pk.OUT_BF16, self.y2)
        ctx.block_norm(**self.norm(2))
        ctx.linear_w4g(self.x3, *self.head, None, pk.ACT_NONE, pk.OUT_F32, self.logits)
        ctx.sample_tokens(self.logits, self.temp, None, None, None, self.u, self.tok)
        ctx.token_logprobs(self.logits, self.temp, self.tok, self.lp, self.rank, self.ent, self.ids, self.tlp)

    def outputs(self):
        return [t.clone() for t in (self.codes, self.y1, self.h1, self.x2, self.a, self.y2, self.h2, self.x3, self.logits, self.tok, self.lp, self.rank, self.ent,
                                    self.ids, self.tlp)]

    def check(self):
        """Each call against its formula, on the operands that it had."""
        gpu, torch = self.gpu, self.gpu.torch
        for i in range(3):
            a = self.norm(i)
            h, e, y, ey = tn.reference(a)
            if i == 0:
                rt = 1 / tn.f64(self.s_tok)[self.pos.cpu().numpy()][:, None]
                u, eu = y * rt, ey * rt + 2 * tn.U * np.abs(y * rt)
                assert (np.abs(self.codes.cpu().numpy() - np.clip(u, -128, 127)) <= 0.5 + eu).all()
            else:
                tn.check_store(a["Hout"], h, e, False)
                tn.check_store(a["Y"], y, ey, True)
        tw.check(gpu, self.O.view(self.B, -1), *self.proj, None, 0, self.y1, False)
        tw.check(gpu, self.x2, *self.fc1, self.bias, 1, self.a, False)
        tw.check(gpu, self.a, *self.fc2, None, 0, self.y2, False)
        tw.check(gpu, self.x3, *self.head, None, 0, self.logits, False)
        x, tok, T = self.logits.double().cpu().numpy(), self.tok.cpu().numpy(), self.temp.double().cpu().numpy()
        assert (tok >= 0).all()
        for b in range(self.B):
            lp, rank, ent, ids, e_s, e_ent = tl.reference(x[b], int(tok[b]), T[b], self.k)
            assert self.rank[b] == rank and abs(float(self.ent[b]) - ent) <= e_ent
            tl.close(float(self.lp[b]), lp[tok[b]], e_s)
            np.testing.assert_array_equal(self.ids[b].cpu().numpy(), ids)


@pytest.mark.parametrize("B", [1, 7, 40])
def test_a_whole_step_eager_and_captured(gpu, B):
    torch = gpu.torch
    s = Step(gpu, B, 3 + B)
    gpu.ctx.stwq_reserve_layer(64, 1024, 3 * 256, 64)
    gpu.ctx.stwq_reserve_paged_attention(64, 4, 4, 64)
    s.run()
    assert gpu.ctx.stwq_device_status() == 0
    s.check()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        s.run()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            s.run()
    before = gpu.ctx.stwq_launch_count()
    for _ in range(2):                                        # other inputs and lengths in the same buffers
        s.h.normal_()
        s.cached.random_(0, 62)
        s.u.uniform_()
        graph.replay()
        torch.cuda.synchronize()
        assert gpu.ctx.stwq_device_status() == 0
        s.check()
        replayed = s.outputs()
        s.run()
        for a, b in zip(replayed, s.outputs()):
            assert torch.equal(a, b)
    assert gpu.ctx.stwq_launch_count() > before


def test_on_a_stream_beside_a_busy_default_stream(gpu):
    torch = gpu.torch
    s = Step(gpu, 7, 99)
    want = Step(gpu, 7, 99)
    want.run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy = torch.randn((6000, 6000), device=gpu.dev)
    torch.cuda.synchronize()
    for _ in range(10):
        busy = (busy @ busy).clamp(-1, 1)                     # the default stream is far behind
    with torch.cuda.stream(side):
        s.run()
        got = s.outputs()
    side.synchronize()
    for a, b in zip(got, want.outputs()):
        assert torch.equal(a, b)
    torch.cuda.synchronize()


def test_group_folded_weights_and_their_norm(gpu):
    """A channel scale folded into 4-bit weights is divided out by the norm before them: Y = N(h) W^T within the weights' quantization."""
    torch, ctx, pk = gpu.torch, gpu.ctx, gpu.pk
    g = torch.Generator(device=gpu.dev).manual_seed(1)
    h, W, s_ch = torch.randn((9, 512), device=gpu.dev, generator=g), torch.randn((200, 512), device=gpu.dev, generator=g) * 0.05, torch.exp(torch.randn(512, device=gpu.dev, generator=g))
    Wp, s = torch.empty((200, 256), dtype=torch.uint8, device=gpu.dev), torch.empty((200, 16), device=gpu.dev)
    ctx.gps_fold_group4(W, s_ch, Wp, s)
    x, Y = torch.empty((9, 512), device=gpu.dev), torch.empty((9, 200), device=gpu.dev)
    ctx.block_norm(h, None, None, None, None, None, 0, None, None, 1.0, pk.NORM_RMS, None, None, 1e-6, None, None, s_ch, None, 8, x)
    ctx.linear_w4g(x, Wp, s, None, 0, pk.OUT_F32, Y)
    n = h.double() / (h.double().pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()
    # a code is at most half a step from its weight (the largest of a group: 7.5 steps, clamped to 7, half a step too); half steps of all channels
    # at once would add up to this; fp32 rounding is far below
    bound = (n.abs() / s_ch.double()) @ (0.5 * s.double().repeat_interleave(32, 1)).T * (1 + 1e-5) + 1e-4
    assert ((Y.double() - n @ W.double().T).abs() <= bound).all()


def test_one_conditioning_row_for_many_and_one_for_each(gpu):
    """The same rows with one vector per sample, in any order of the samples, and with the vectors written out per row."""
    torch, ctx = gpu.torch, gpu.ctx
    for M, Cn in ((700, 1920), (9000, 320)):
        a = tn.make(gpu, M, Cn, h="bf16", G=6, w=False, seed=M)
        a["cond_ids"] = (torch.arange(M, device=gpu.dev) * 6 // M).to(torch.int32)
        ctx.block_norm(**a)
        rows = a["cond_ids"].long()
        wide = torch.cat([a[k][rows] for k in ("gate", "scale", "shift")], 1)
        b = dict(a, gate=wide[:, :Cn], scale=wide[:, Cn:2 * Cn], shift=wide[:, 2 * Cn:], cond_ids=torch.arange(M, device=gpu.dev, dtype=torch.int32),
                 Hout=torch.empty_like(a["Hout"]), Y=torch.empty_like(a["Y"]))
        ctx.block_norm(**b)
        assert torch.equal(a["Hout"], b["Hout"]) and torch.equal(a["Y"], b["Y"])


def test_rows_beyond_2_31_elements(gpu):
    torch, ctx = gpu.torch, gpu.ctx
    M, Cn = 270000, 8192
    H = torch.zeros((M, Cn), device=gpu.dev, dtype=torch.bfloat16)
    H[-3:].normal_()
    Y = torch.empty_like(H)
    none = (None, None, None, None)
    ctx.block_norm(H, None, *none, 0, None, None, 1.0, 1, None, None, 1e-6, None, None, None, None, 8, Y)
    small = torch.empty((3, Cn), device=gpu.dev, dtype=torch.bfloat16)
    want = H[-3:].double()
    want = want / (want.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()
    assert (Y[:-3] == 0).all()
    e = np.abs(tn.f64(want)) * (tn.DEPTH + 20) * tn.U
    tn.check_store(Y[-3:], tn.f64(want), e, True)
    ctx.block_norm(H[-3:], None, *none, 0, None, None, 1.0, 1, None, None, 1e-6, None, None, None, None, 8, small)
    tn.check_store(small, tn.f64(want), e, True)


def test_the_c_entry_points_refuse_and_write_nothing(gpu):
    torch, lib, h = gpu.torch, gpu.ctx.lib, gpu.ctx.handle
    NULL, DIM, ALIGN, BITS = -1, -2, -3, -4
    buf = torch.full((1 << 20,), 7.0, device=gpu.dev)
    at = lambda off=0: C.c_void_p(buf.data_ptr() + off)  # noqa: E731
    st = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    p = [at(i * 65536) for i in range(16)]

    def bn(**k):
        a = dict(H=p[0], ldh=64, hd=0, O=p[1], ldo=64, od=0, M=4, C=64, cond=None, G=1, gate=p[2], scale=p[3], shift=p[4], ldc=64, cd=0, post=0, wp=None, bp=None, rs=1.0,
                 pre=1, w=p[5], b=None, eps=1e-6, Ho=p[6], ldho=64, pos=p[7], sch=None, stok=p[8], P=4, bits=8, Y=p[9], ldy=64, yd=0)
        a.update(k)
        return lib.block_norm(h, *a.values(), st)
    for code, k in ((NULL, dict(H=None)), (DIM, dict(M=0)), (DIM, dict(M=1 << 31)), (DIM, dict(C=0)), (DIM, dict(C=16392, ldh=16392)), (ALIGN, dict(C=60)), (DIM, dict(ldh=56)), (DIM, dict(ldy=60)),
                    (ALIGN, dict(ldh=66)), (ALIGN, dict(H=at(4))), (ALIGN, dict(gate=at(8))), (ALIGN, dict(w=at(12))), (BITS, dict(hd=2)), (BITS, dict(od=3)), (BITS, dict(cd=2)), (BITS, dict(yd=2)),
                    (BITS, dict(pre=2)), (BITS, dict(post=-1)), (DIM, dict(eps=-1.0)), (DIM, dict(G=0)), (DIM, dict(G=2, ldc=32)), (NULL, dict(yd=3, stok=None)), (BITS, dict(yd=3, bits=7)), (DIM, dict(yd=3, P=0)),
                    (ALIGN, dict(Ho=p[1])), (ALIGN, dict(Y=at(16)))):
        assert bn(**k) == code, k

    def w4(**k):
        a = dict(X=p[0], ldx=128, xd=0, M=2, K=128, N=16, W=p[1], s=p[2], sd=0, group=32, bias=p[3], act=0, od=0, Y=p[4])
        a.update(k)
        return lib.linear_w4g(h, *a.values(), st)
    for code, k in ((NULL, dict(X=None)), (NULL, dict(Y=None)), (DIM, dict(M=0)), (DIM, dict(M=65)), (DIM, dict(K=0)), (DIM, dict(K=131072, ldx=131072)), (DIM, dict(N=0)), (DIM, dict(ldx=120)),
                    (DIM, dict(group=0)), (DIM, dict(group=256)), (ALIGN, dict(group=48)), (ALIGN, dict(group=96)), (ALIGN, dict(ldx=130)), (ALIGN, dict(X=at(4))), (ALIGN, dict(W=at(8))), (ALIGN, dict(s=at(2))),
                    (ALIGN, dict(Y=at(2))), (ALIGN, dict(bias=at(1))), (DIM, dict(N=(1 << 30) + 1)), (ALIGN, dict(Y=p[0])), (ALIGN, dict(Y=at(65536 + 64))), (ALIGN, dict(Y=at(2 * 65536 - 8))),
                    (ALIGN, dict(Y=p[3])), (BITS, dict(xd=2)), (BITS, dict(sd=-1)), (BITS, dict(od=3)), (BITS, dict(act=4))):
        assert w4(**k) == code, k
    assert lib.gps_fold_group4(h, p[0], 4, 128, None, 24, p[1], p[2], 0, st) == ALIGN and lib.gps_fold_group4(h, p[0], 4, 128, None, 32, p[1], p[2], 2, st) == BITS
    assert lib.gps_fold_group4(h, p[0], 0, 128, None, 32, p[1], p[2], 0, st) == DIM and lib.gps_fold_group4(h, at(4), 4, 128, None, 32, p[1], p[2], 0, st) == ALIGN
    assert lib.gps_fold_group4(h, p[0], 4, 128, None, 32, at(1024), p[2], 0, st) == ALIGN

    def lp(**k):
        a = dict(X=p[0], xd=0, ld=100, B=4, V=100, T=None, tok=p[1], lp=p[2], rk=p[3], en=p[4], k=3, ids=p[5], tl=p[6])
        a.update(k)
        return lib.token_logprobs(h, *a.values(), st)
    for code, k in ((NULL, dict(X=None)), (NULL, dict(tok=None)), (NULL, dict(lp=None)), (NULL, dict(ids=None)), (NULL, dict(k=0)), (NULL, dict(tok=None, lp=None)), (DIM, dict(B=0)), (DIM, dict(V=0)),
                    (DIM, dict(V=360449, ld=360449)), (DIM, dict(ld=99)), (DIM, dict(k=-1)), (DIM, dict(k=33)), (BITS, dict(xd=2)), (ALIGN, dict(X=at(2))), (ALIGN, dict(lp=at(400))), (ALIGN, dict(tl=p[0])), (ALIGN, dict(en=at(1596)))):
        assert lp(**k) == code, k
    torch.cuda.synchronize()
    assert (buf == 7).all() and gpu.ctx.stwq_device_status() == 0
