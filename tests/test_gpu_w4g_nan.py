"""linear_w4g on NaN of every payload, in each of its forms."""
import pytest

import test_gpu_w4g as tw
from test_gpu_w4g import gpu  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

# rows, K, N on 148 SMs: operands resident, in two widths of tiles; coming with the codes; the kernel for many rows with 8, 16 and 32 tokens
FORMS = [(3, 256, 300), (3, 256, 2500), (2, 256, 8000), (3, 8192, 300), (3, 8192, 2500), (8, 4096, 7200), (5, 1024, 300), (12, 1024, 300), (24, 512, 4000),
         (40, 512, 9000)]


@pytest.mark.parametrize("M,K,N", FORMS)
@pytest.mark.parametrize("group", [64, 128])
def test_every_nan_is_one(gpu, M, K, N, group):  # noqa: F811
    """All bits that make the value a NaN may lie in the lower half of the word, whose upper half alone is that of an infinity."""
    torch, pk = gpu.torch, gpu.pk
    Wp, s, g = tw.weights(gpu, N, K, group)
    Wp[:, 20] = 0x77                                          # channels 40, 41: code 7 in every row
    Wp[: N // 2, 20] = 0x70                                   # and 0 at channel 40 in half of them: NaN times 0
    X = torch.randn((M, K), device=gpu.dev, generator=g)
    clean, inf = X.clone(), float("inf")
    clean[0] = 0
    Y, Z = torch.empty((M, N), device=gpu.dev), torch.empty((M, N), device=gpu.dev)
    gpu.ctx.linear_w4g(clean, Wp, s, None, 0, pk.OUT_F32, Z)
    for word in (0x7F800001, -0x7FFFFF, 0x7F808000, 0x7F80FFFF, 0x7FC00000, 0x7FFFFFFF, -1):      # -0x7fffff: 0xff800001
        X.view(torch.int32)[0, 40] = word
        assert torch.isnan(X[0, 40])
        for act in (0, 1):
            gpu.ctx.linear_w4g(X, Wp, s, None, act, pk.OUT_F32, Y)
            assert torch.isnan(Y[0]).all(), hex(word)
            if act == 0:
                assert torch.equal(Y[1:], Z[1:])
    X[0, 40], X[0, 41] = 1.0, -inf                            # an infinity stays one
    gpu.ctx.linear_w4g(X, Wp, s, None, 0, pk.OUT_F32, Y)
    assert (Y[0] == -inf).all()


@pytest.mark.parametrize("M,K,N", [(3, 256, 300), (13, 256, 300), (40, 512, 9000)])
def test_every_nan_of_bf16(gpu, M, K, N):  # noqa: F811
    torch = gpu.torch
    Wp, s, g = tw.weights(gpu, N, K, 64)
    X = torch.randn((M, K), device=gpu.dev, generator=g).to(torch.bfloat16)
    Y = torch.empty((M, N), device=gpu.dev)
    for word in (0x7F81, 0x7FFF, -0x7F, -1):                  # -0x7f: 0xff81
        X.view(torch.int16)[M - 1, 77] = word
        gpu.ctx.linear_w4g(X, Wp, s, None, 0, gpu.pk.OUT_F32, Y)
        assert torch.isnan(Y[M - 1]).all() and torch.isfinite(Y[:M - 1]).all()
