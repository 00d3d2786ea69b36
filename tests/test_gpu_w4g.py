"""gps_fold_group4 and linear_w4g on the GPU: the fold against its formula in the same roundings, the products against 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


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


def weights(gpu, N, K, group, s_bf16=False, seed=0):
    """Random nibbles (every code from -8 to 7) and scales; and the codes."""
    torch = gpu.torch
    g = torch.Generator(device=gpu.dev).manual_seed(seed * 77 + N * 3 + K + group)
    Wp = torch.randint(0, 256, (N, K // 2), device=gpu.dev, generator=g, dtype=torch.int32).to(torch.uint8)
    s = ((torch.rand((N, K // group), device=gpu.dev, generator=g) + 0.3) * 0.02).to(torch.bfloat16 if s_bf16 else torch.float32)
    return Wp, s, g


def codes(Wp):
    p = Wp.cpu().numpy().astype(np.int64)
    c = np.stack([p & 15, p >> 4], -1).reshape(p.shape[0], -1)
    return np.where(c > 7, c - 16, c)


def gelu(z, form):
    if form == 0:
        return z
    if form == 1:
        return z * 0.5 * (1 + np.vectorize(math.erf)(z / math.sqrt(2)))
    return 0.5 * z * (1 + np.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))


def check(gpu, X, Wp, s, bias, act, Y, fp32_in):
    K = X.shape[1]
    w = codes(Wp) * np.repeat(s.double().cpu().numpy(), K // s.shape[1], 1)
    x = X.double().cpu().numpy()
    z = x @ w.T + (0 if bias is None else bias.double().cpu().numpy())
    mag = np.abs(x) @ np.abs(w).T + (0 if bias is None else np.abs(bias.double().cpu().numpy()))
    # a chunk of 128 channels is 8 products (24 with fp32 activations, whose parts add up to at most 1 + 2^-7 of them), each taken
    # to lose at most a unit of 2^-22 of the chunk's magnitude; then the scale, an addition per chunk, the warps' sums, the bias
    per_chunk = 25 if fp32_in else 8
    e = mag * (per_chunk * 2.0 ** -22 + (math.ceil(K / 128) + 16 + 3) * U)
    want = gelu(z, act)
    # |gelu'| < 1.13; the erf form is off by 1.5e-7 |z| and a product, the tanh form by 2^-20, the short one by 6e-4 |z|
    e = e * (1.13 if act else 1) + np.abs(z) * (0, 1.5e-7 + 2 * U, 2.0 ** -20, 6e-4)[act]
    if Y.dtype == gpu.torch.bfloat16:
        e = e + 2.0 ** -8 * (np.abs(want) + e)
    err = np.abs(Y.double().cpu().numpy() - want)
    assert (err <= e).all(), (float((err / e).max()), int((err > e).sum()))


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 8, 9, 16, 17, 40, 64])
@pytest.mark.parametrize("group", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_rows_and_groups(gpu, M, group, x):
    torch = gpu.torch
    K, N = group * (9 if group < 128 else 5), 83
    Wp, s, g = weights(gpu, N, K, group, s_bf16=M % 2 == 0, seed=M)
    X = torch.randn((M, K), device=gpu.dev, generator=g).to(torch.bfloat16 if x == "bf16" else torch.float32)
    bias = torch.randn((N,), device=gpu.dev, generator=g)
    for out, dt in ((gpu.pk.OUT_F32, torch.float32), (gpu.pk.OUT_BF16, torch.bfloat16)):
        Y = torch.full((M, N), 7.0, device=gpu.dev, dtype=dt)
        gpu.ctx.linear_w4g(X, Wp, s, bias, 0, out, Y)
        check(gpu, X, Wp, s, bias, 0, Y, x == "f32")


@pytest.mark.parametrize("N,K,group", [(1, 32, 32), (16, 128, 128), (17, 64, 64), (15, 160, 32), (1000, 2048, 128), (2048, 8192, 64), (640, 1920, 32), (33, 65536, 128),
                                       (5000, 96, 96), (4096, 512, 512), (129, 131040, 32)])
@pytest.mark.parametrize("M", [1, 7, 13])
def test_sizes(gpu, N, K, group, M):
    torch = gpu.torch
    Wp, s, g = weights(gpu, N, K, group, seed=M)
    X = torch.randn((M, K), device=gpu.dev, generator=g).to(torch.bfloat16)
    Y = torch.full((M, N), 7.0, device=gpu.dev)
    gpu.ctx.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, Y)
    check(gpu, X, Wp, s, None, 0, Y, False)


@pytest.mark.parametrize("act", [0, 1, 2, 3])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_activations(gpu, act, out):
    torch = gpu.torch
    Wp, s, g = weights(gpu, 300, 256, 64, seed=act)
    X = torch.randn((6, 256), device=gpu.dev, generator=g)
    bias = torch.randn((300,), device=gpu.dev, generator=g)
    Y = torch.empty((6, 300), device=gpu.dev, dtype=torch.float32 if out == "f32" else torch.bfloat16)
    gpu.ctx.linear_w4g(X, Wp, s, bias, act, gpu.pk.OUT_F32 if out == "f32" else gpu.pk.OUT_BF16, Y)
    check(gpu, X, Wp, s, bias, act, Y, True)


def test_strided_rows_and_what_lies_beside_them(gpu):
    torch = gpu.torch
    for x, M in ((torch.bfloat16, 5), (torch.float32, 11)):
        Wp, s, g = weights(gpu, 70, 320, 32)
        wide = torch.full((M + 2, 400), float("nan"), device=gpu.dev, dtype=x)
        X = wide[1:M + 1, 40:360]
        X.copy_(torch.randn((M, 320), device=gpu.dev, generator=g))
        Y = torch.full((M + 1, 70), 7.0, device=gpu.dev)
        gpu.ctx.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, Y[:M])
        check(gpu, X, Wp, s, None, 0, Y[:M], x == torch.float32)
        assert (Y[M] == 7).all()


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("group", [32, 128])
def test_nan_and_inf_stay_in_their_row(gpu, x, group):
    torch, nan, inf = gpu.torch, float("nan"), float("inf")
    dt = torch.bfloat16 if x == "bf16" else torch.float32
    Wp, s, g = weights(gpu, 64, 256, group)
    Wp[:, 20] = 0x77                                          # channels 40, 41: code 7 in every row
    X = torch.randn((5, 256), device=gpu.dev, generator=g).to(dt)
    X[1, 40], X[2, 41], X[3, 40] = nan, inf, -inf
    clean = X.clone()
    clean[1:4] = 0
    Y, Z = torch.empty((5, 64), device=gpu.dev), torch.empty((5, 64), device=gpu.dev)
    gpu.ctx.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, Y)
    gpu.ctx.linear_w4g(clean, Wp, s, None, 0, gpu.pk.OUT_F32, Z)
    assert torch.isnan(Y[1]).all() and (Y[2] == inf).all() and (Y[3] == -inf).all()
    assert torch.equal(Y[[0, 4]], Z[[0, 4]])
    for act in (1, 2, 3):
        gpu.ctx.linear_w4g(X, Wp, s, None, act, gpu.pk.OUT_F32, Y)
        assert (Y[2] == inf).all() and torch.isnan(Y[1]).all() and torch.isnan(Y[3]).all()


def test_large_and_small_activations(gpu):
    """fp32 activations over the whole range of exponents: the three parts cover all bits, the largest values do not overflow a part."""
    torch = gpu.torch
    Wp, s, g = weights(gpu, 48, 128, 128)
    for top in (3.4e38, 1e30, 1.0, 1e-25):
        X = (torch.rand((3, 128), device=gpu.dev, generator=g) * 2 - 1) * torch.exp2(-40 * torch.rand((3, 128), device=gpu.dev, generator=g))
        X = (X * top).contiguous()
        if top > 1e38:
            X[0].zero_()
            X[0, 3] = 3.4028234e38
            small = s * 0.01                                  # keeps the products finite
        else:
            small = s
        Y = torch.empty((3, 48), device=gpu.dev)
        gpu.ctx.linear_w4g(X, Wp, small, None, 0, gpu.pk.OUT_F32, Y)
        if top > 1e38:
            X, Y = X[:1], Y[:1]
        check(gpu, X, Wp, small, None, 0, Y, True)


def test_same_bits_every_time_and_in_any_batch(gpu):
    torch = gpu.torch
    Wp, s, g = weights(gpu, 2048, 4096, 128)
    X = torch.randn((8, 4096), device=gpu.dev, generator=g).to(torch.bfloat16)
    Y = [torch.empty((8, 2048), device=gpu.dev) for _ in range(2)]
    for y in Y:
        gpu.ctx.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, y)
    assert torch.equal(*Y)


@pytest.mark.parametrize("N,K,group", [(1, 32, 32), (37, 256, 64), (64, 96, 96), (5, 1920, 128), (3, 4096, 4096)])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("scaled", [False, True])
def test_fold(gpu, N, K, group, bf16, scaled):
    torch = gpu.torch
    r = np.random.default_rng(N + K)
    W = (r.standard_normal((N, K)) * 0.02).astype(np.float32)
    W[0, :group] = 0                                          # a group of zeros: scale 1
    s_ch = np.exp(0.4 * r.standard_normal(K)).astype(np.float32) if scaled else None
    T = lambda a: None if a is None else torch.from_numpy(a).to(gpu.dev)  # noqa: E731
    Wp = torch.full((N, K // 2), 0xEE, device=gpu.dev, dtype=torch.uint8)
    s = torch.zeros((N, K // group), device=gpu.dev, dtype=torch.bfloat16 if bf16 else torch.float32)
    gpu.ctx.gps_fold_group4(T(W), T(s_ch), Wp, s)
    v = W if s_ch is None else W * s_ch                       # fp32 product
    a = np.abs(v.reshape(N, -1, group)).max(-1)
    want = np.where(a > 0, (a + a) / np.float32(15), np.float32(1)).astype(np.float32)
    want = torch.from_numpy(want).to(s.dtype)
    assert torch.equal(s.cpu(), want)
    d = np.repeat(want.float().numpy(), group, 1)
    np.testing.assert_array_equal(codes(Wp), np.clip(np.rint(v / d), -8, 7).astype(np.int64))


def test_one_group_per_row_is_the_per_channel_fold(gpu):
    """With group = K the codes and scales are those of gps_fold_packed4, and its weights are taken as they are."""
    torch = gpu.torch
    g = torch.Generator(device=gpu.dev).manual_seed(5)
    W = torch.randn((96, 384), device=gpu.dev, generator=g)
    Wp, Wp2 = (torch.empty((96, 192), device=gpu.dev, dtype=torch.uint8) for _ in range(2))
    s, s_w = torch.empty((96, 1), device=gpu.dev), torch.empty((96,), device=gpu.dev)
    gpu.ctx.gps_fold_group4(W, None, Wp, s)
    gpu.ctx.gps_fold_packed4(W, None, Wp2, s_w)
    assert torch.equal(Wp, Wp2) and torch.equal(s[:, 0], s_w)
    X = torch.randn((4, 384), device=gpu.dev, generator=g)
    Y = torch.empty((4, 96), device=gpu.dev)
    gpu.ctx.linear_w4g(X, Wp2, s_w.view(96, 1), None, 0, gpu.pk.OUT_F32, Y)
    check(gpu, X, Wp2, s_w.view(96, 1), None, 0, Y, True)


@pytest.mark.parametrize("N,K,group,M,x", [(40000, 4096, 128, 4, "bf16"), (33001, 2048, 64, 1, "f32"), (40000, 4096, 128, 13, "bf16"), (24000, 8192, 32, 8, "bf16"),
                                           (128000, 1024, 1024, 2, "bf16")])
def test_blocks_with_several_tiles(gpu, N, K, group, M, x):
    """Many tiles for each block, twice in a row and on two streams at once."""
    torch = gpu.torch
    Wp, s, g = weights(gpu, N, K, group, seed=M)
    X = torch.randn((M, K), device=gpu.dev, generator=g).to(torch.bfloat16 if x == "bf16" else torch.float32)
    p = Wp.long()
    c = torch.stack([p & 15, p >> 4], -1).flatten(1).double()
    del p
    c = torch.where(c > 7, c - 16, c) * s.double().repeat_interleave(group, 1)
    want, mag = X.double() @ c.T, X.double().abs() @ c.abs().T
    e = mag * ((25 if x == "f32" else 8) * 2.0 ** -22 + (math.ceil(K / 128) + 16 + 3) * U)
    other, ctx2 = torch.cuda.Stream(), gpu.pk.Context(0)
    Y = [torch.full((M, N), 7.0, device=gpu.dev) for _ in range(3)]
    torch.cuda.synchronize()
    gpu.ctx.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, Y[0])
    ctx2.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, Y[1], stream=other)
    gpu.ctx.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, Y[2])
    torch.cuda.synchronize()
    assert gpu.ctx.stwq_device_status() == 0 and ctx2.stwq_device_status() == 0
    assert ((Y[0].double() - want).abs() <= e).all()
    assert torch.equal(Y[0], Y[1]) and torch.equal(Y[0], Y[2])
    ctx2.close()


def test_weights_beyond_2_31_elements(gpu):
    """Row offsets in the packed weights pass 32 bits: the last rows agree with a call on them alone."""
    torch = gpu.torch
    N, K = 70000, 65536
    Wp = torch.empty((N, K // 2), device=gpu.dev, dtype=torch.uint8)
    g = torch.Generator(device=gpu.dev).manual_seed(9)
    Wp[:64] = torch.randint(0, 256, (64, K // 2), device=gpu.dev, generator=g, dtype=torch.int32).to(torch.uint8)
    Wp[-64:] = torch.randint(0, 256, (64, K // 2), device=gpu.dev, generator=g, dtype=torch.int32).to(torch.uint8)
    Wp[64:-64] = 0
    s = torch.full((N, K // 64), 0.01, device=gpu.dev)
    X = torch.randn((1, K), device=gpu.dev, generator=g)
    Y, Z = torch.empty((1, N), device=gpu.dev), torch.empty((1, 64), device=gpu.dev)
    gpu.ctx.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, Y)
    assert (Y[0, 64:-64] == 0).all()
    for rows in (slice(0, 64), slice(N - 64, N)):
        gpu.ctx.linear_w4g(X, Wp[rows], s[rows], None, 0, gpu.pk.OUT_F32, Z)
        check(gpu, X, Wp[rows], s[rows], None, 0, Y[:, rows], True)
        check(gpu, X, Wp[rows], s[rows], None, 0, Z, True)


def test_refusals(gpu):
    torch, pk = gpu.torch, gpu.pk
    Wp, s, g = weights(gpu, 32, 128, 32)
    X, Y = torch.zeros((4, 128), device=gpu.dev), torch.zeros((4, 32), device=gpu.dev)

    def refused(code, X=X, Wp=Wp, s=s, bias=None, act=0, out=pk.OUT_F32, Y=Y):
        with pytest.raises(pk.StwqError) as e:
            gpu.ctx.linear_w4g(X, Wp, s, bias, act, out, Y)
        assert e.value.code == code
    z = lambda *n, dt=torch.float32: torch.zeros(n, device=gpu.dev, dtype=dt)  # noqa: E731
    refused(-2, X=z(65, 128), Y=z(65, 32))                                  # more rows than a few
    refused(-2, s=z(32, 3))                                                 # groups that do not divide K
    refused(-3, s=z(32, 8))                                                 # 16 channels per group
    refused(-2, Wp=z(32, 63, dt=torch.uint8))
    refused(-4, act=9)
    refused(-4, out=pk.OUT_INT32)
    refused(-4, s=z(32, 4, dt=torch.float16))
    refused(-3, X=z(4, 130)[:, :128])                                       # rows 520 bytes apart
    refused(-3, X=z(4, 132)[:, 1:129])
    refused(-2, X=z(4, 128).as_strided((4, 128), (64, 1)))                  # rows that overlap
    refused(-2, bias=z(31))
    refused(-1, Y=None)
    with pytest.raises(pk.StwqError) as e:
        gpu.ctx.gps_fold_group4(z(4, 128), None, z(4, 64, dt=torch.uint8), z(4, 8))
    assert e.value.code == -3
    with pytest.raises(pk.StwqError) as e:
        gpu.ctx.gps_fold_group4(z(4, 128), None, z(4, 64, dt=torch.uint8), z(4, 5))
    assert e.value.code == -2


# many rows: output channels enough for it on 148 SMs, each form of the kernel, ragged in every direction
MANY = [("bf16", 17, 2500, 640, 64), ("bf16", 25, 3001, 1152, 128), ("bf16", 32, 5000, 32, 32), ("bf16", 32, 7333, 416, 32), ("bf16", 20, 7500, 1280, 256),
        ("bf16", 64, 2405, 544, 32), ("bf16", 49, 4099, 768, 96), ("bf16", 40, 4801, 1024, 128), ("bf16", 33, 9000, 160, 160), ("bf16", 64, 2370, 8192, 64),
        ("f32", 9, 2401, 320, 32), ("f32", 16, 130, 512, 128), ("f32", 13, 5760, 1920, 32), ("f32", 16, 2370, 4096, 256), ("f32", 64, 1300, 512, 128),
        ("f32", 20, 4000, 96, 96), ("f32", 31, 3000, 1056, 32), ("f32", 33, 7200, 352, 32), ("f32", 64, 3700, 1024, 128), ("f32", 63, 8191, 64, 64), ("f32", 4, 2370, 1056, 32),
        ("f32", 7, 7001, 640, 128), ("f32", 8, 5760, 1920, 96), ("f32", 5, 1184, 4096, 64), ("f32", 6, 3001, 32, 32)]


@pytest.mark.parametrize("x,M,N,K,group", MANY)
def test_many_rows(gpu, x, M, N, K, group):
    torch = gpu.torch
    Wp, s, g = weights(gpu, N, K, group, s_bf16=M % 2 == 0, seed=M)
    dt = torch.bfloat16 if x == "bf16" else torch.float32
    wide = torch.full((M + 2, K + 48), float("nan"), device=gpu.dev, dtype=dt)
    X = wide[1:M + 1, 16:K + 16]
    X.copy_(torch.randn((M, K), device=gpu.dev, generator=g))
    bias = torch.randn((N,), device=gpu.dev, generator=g) if N % 2 else None
    for out, ydt, act in ((gpu.pk.OUT_F32, torch.float32, 0), (gpu.pk.OUT_BF16, torch.bfloat16, 2)):
        Y = torch.full((M + 1, N), 7.0, device=gpu.dev, dtype=ydt)
        gpu.ctx.linear_w4g(X, Wp, s, bias, act, out, Y[:M])
        check(gpu, X, Wp, s, bias, act, Y[:M], x == "f32")
        assert (Y[M] == 7).all()
        again = torch.empty((M, N), device=gpu.dev, dtype=ydt)
        gpu.ctx.linear_w4g(X, Wp, s, bias, act, out, again)
        assert torch.equal(again, Y[:M])


@pytest.mark.parametrize("x,M,N", [("bf16", 30, 2500), ("bf16", 64, 2500), ("f32", 12, 2500), ("f32", 64, 2500), ("f32", 40, 7200)])
@pytest.mark.parametrize("group", [32, 128])
def test_many_rows_nan_and_inf_stay_in_their_row(gpu, x, M, N, group):
    torch, nan, inf = gpu.torch, float("nan"), float("inf")
    Wp, s, g = weights(gpu, N, 256, group)
    Wp[:, 20] = 0x77                                          # channels 40, 41: code 7 in every row
    X = torch.randn((M, 256), device=gpu.dev, generator=g).to(torch.bfloat16 if x == "bf16" else torch.float32)
    X[1, 40], X[M - 2, 41], X[9, 40] = nan, inf, -inf
    clean = X.clone()
    clean[[1, 9, M - 2]] = 0
    Y, Z = torch.empty((M, N), device=gpu.dev), torch.empty((M, N), device=gpu.dev)
    gpu.ctx.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, Y)
    gpu.ctx.linear_w4g(clean, Wp, s, None, 0, gpu.pk.OUT_F32, Z)
    assert torch.isnan(Y[1]).all() and (Y[M - 2] == inf).all() and (Y[9] == -inf).all()
    rest = [m for m in range(M) if m not in (1, 9, M - 2)]
    assert torch.equal(Y[rest], Z[rest])


@pytest.mark.parametrize("x,M,N,K", [("bf16", 24, 3000, 1024), ("bf16", 64, 3000, 1024), ("f32", 64, 3000, 1024), ("f32", 13, 3000, 2048), ("f32", 8, 3000, 2048)])
def test_many_rows_captured_as_a_contexts_first_call(gpu, x, M, N, K):
    torch = gpu.torch
    Wp, s, g = weights(gpu, N, K, 64)
    X = torch.randn((M, K), device=gpu.dev, generator=g).to(torch.bfloat16 if x == "bf16" else torch.float32)
    Y, Z = torch.zeros((M, N), device=gpu.dev), torch.empty((M, N), device=gpu.dev)
    fresh = gpu.pk.Context(0)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        fresh.linear_w4g(X, Wp, s, None, 1, gpu.pk.OUT_F32, Y)
    X.copy_(torch.randn((M, K), device=gpu.dev, generator=g))
    graph.replay()
    gpu.ctx.linear_w4g(X, Wp, s, None, 1, gpu.pk.OUT_F32, Z)
    torch.cuda.synchronize()
    assert torch.equal(Y, Z)
    check(gpu, X, Wp, s, None, 1, Y, x == "f32")
    fresh.close()


@pytest.mark.parametrize("x,M", [("bf16", 64), ("bf16", 20), ("f32", 33), ("f32", 12)])
def test_many_rows_offsets_beyond_2_31(gpu, x, M):
    """Offsets in the packed weights, and then in Y, pass 32 bits: the first and the last rows against 64 bits, zeros between."""
    torch = gpu.torch
    g = torch.Generator(device=gpu.dev).manual_seed(M)
    dt = torch.bfloat16 if x == "bf16" else torch.float32
    for N, K in ((70000, 65536), (2 ** 31 // M + 300, 32)):
        Wp = torch.zeros((N, K // 2), device=gpu.dev, dtype=torch.uint8)
        for rows in (slice(0, 64), slice(N - 64, N)):
            Wp[rows] = torch.randint(0, 256, (64, K // 2), device=gpu.dev, generator=g, dtype=torch.int32).to(torch.uint8)
        s = torch.full((N, K // 32), 0.01, device=gpu.dev, dtype=torch.bfloat16)
        X = torch.randn((M, K), device=gpu.dev, generator=g).to(dt)
        Y = torch.empty((M, N), device=gpu.dev)
        gpu.ctx.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, Y)
        assert all(not Y[m, 64:-64].any() for m in range(M))
        for rows in (slice(0, 64), slice(N - 64, N)):
            check(gpu, X, Wp[rows], s[rows], None, 0, Y[:, rows], x == "f32")
        del Wp, s, X, Y
        torch.cuda.empty_cache()


@pytest.mark.parametrize("M,N", [(8, 3000), (12, 3000), (40, 3000), (64, 4000)])
@pytest.mark.parametrize("group", [32, 128])
def test_many_rows_large_and_small_activations(gpu, M, N, group):
    """fp32 activations over 40 octaves and up to the largest: the parts cover all bits."""
    torch = gpu.torch
    Wp, s, g = weights(gpu, N, 256, group)
    for top in (1e30, 1.0, 1e-25):
        X = (torch.rand((M, 256), device=gpu.dev, generator=g) * 2 - 1) * torch.exp2(-40 * torch.rand((M, 256), device=gpu.dev, generator=g)) * top
        Y = torch.empty((M, N), device=gpu.dev)
        gpu.ctx.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, Y)
        check(gpu, X, Wp, s, None, 0, Y, True)
    X = torch.zeros((M, 256), device=gpu.dev)
    X[:, 3] = 3.4028234e38
    small = s * 0.01                                          # keeps the products finite
    Y = torch.empty((M, N), device=gpu.dev)
    gpu.ctx.linear_w4g(X, Wp, small, None, 0, gpu.pk.OUT_F32, Y)
    check(gpu, X, Wp, small, None, 0, Y, True)


def test_many_rows_beside_each_other(gpu):
    """Clusters of several calls on two streams share the SMs: each call's bits stay what they are alone."""
    torch = gpu.torch
    jobs = []
    for i, (M, N, K, dt) in enumerate([(64, 9000, 2048, torch.bfloat16), (24, 3000, 4096, torch.bfloat16), (64, 3000, 1024, torch.float32), (8, 3000, 2048, torch.float32)]):
        Wp, s, g = weights(gpu, N, K, 64, seed=i)
        X = torch.randn((M, K), device=gpu.dev, generator=g).to(dt)
        alone, Y, Z = (torch.empty((M, N), device=gpu.dev) for _ in range(3))
        gpu.ctx.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, alone)
        jobs.append((X, Wp, s, alone, (Y, Z)))
    other, streams = gpu.pk.Context(0), [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for turn in range(12):
        for j in range(len(jobs)):
            for k, ctx in enumerate((gpu.ctx, other)):
                X, Wp, s, _, Y = jobs[(j + 2 * k + turn * k) % len(jobs)]
                ctx.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, Y[k], stream=streams[k])
    torch.cuda.synchronize()
    for _, _, _, alone, Y in jobs:
        assert torch.equal(alone, Y[0]) and torch.equal(alone, Y[1])
    other.close()
