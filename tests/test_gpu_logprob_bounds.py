"""Bounds of token_logprobs' outputs: no log probability above 0, no entropy below."""
import numpy as np
import pytest

import test_gpu_logprobs as tl
from test_gpu_logprobs import gpu  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bfloat16", "float32"])
@pytest.mark.parametrize("V,B", [(40, 4000), (3000, 400), (128000, 8)])
@pytest.mark.parametrize("rest", [-np.inf, -60.0])
def test_no_probability_above_one(gpu, dt, V, B, rest):  # noqa: F811
    """Rows whose tokens but one have no weight, or next to none: the sum of the weights is that token's own, which is rounded."""
    torch = gpu.torch
    g = torch.Generator(device=gpu.dev).manual_seed(V + B)
    X = torch.full((B, V), float(rest), device=gpu.dev).to(getattr(torch, dt))
    at = torch.randint(0, V, (B,), device=gpu.dev, generator=g)
    top = torch.randn((B,), device=gpu.dev, generator=g) * 20
    top[0], top[1] = 3.3, 20.7
    X.scatter_(1, at[:, None], top[:, None].to(X.dtype))
    for temp in (None, torch.rand((B,), device=gpu.dev, generator=g) * 0.5 + 0.1):
        lp, rank, ent, ids, tlp = tl.run(gpu, X, at.to(torch.int32), temp, 2)
        assert gpu.ctx.stwq_device_status() == 0
        assert (lp <= 0).all() and (tlp <= 0).all() and (ent >= 0).all()
        n = 64
        tl.check(gpu, X[:n], at[:n].to(torch.int32), None if temp is None else temp[:n], 2)


@pytest.mark.parametrize("dt", ["bfloat16", "float32"])
@pytest.mark.parametrize("V", [40, 16384, 128000])
def test_peaked_rows(gpu, dt, V):  # noqa: F811
    torch = gpu.torch
    X, g = tl.logits(gpu, 8, V, dt, V, spread=4.0)
    at = X.float().argmax(-1)
    X.scatter_(1, at[:, None], torch.linspace(18, 60, 8, device=gpu.dev)[:, None].to(X.dtype))
    lp, rank, ent, ids, tlp = tl.run(gpu, X, at.to(torch.int32), None, 5)
    assert (lp <= 0).all() and (tlp <= 0).all() and (ent >= 0).all()
    tl.check(gpu, X, at.to(torch.int32), None, 5)
