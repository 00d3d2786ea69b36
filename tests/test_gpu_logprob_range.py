"""token_logprobs on logits whose differences pass the largest fp32, at temperatures that bring them together again."""
import pytest

import test_gpu_logprobs as tl
from test_gpu_logprobs import gpu  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bfloat16", "float32"])
@pytest.mark.parametrize("V", [50, 3000, 128000])
def test_differences_beyond_the_largest_number(gpu, dt, V):  # noqa: F811
    """Up to 6.6e38 apart at temperatures of 1e38 and more (an infinite one counts as 3.4e38): a few octaves, which all count. The bound of
    the other tests holds: log2(e) / t is a subnormal number there, off by up to 2.8 units of 2^-24 instead of one, over at most 10 octaves,
    which the 40 units that it grants to the exponentials cover beside their own 4."""
    torch = gpu.torch
    g = torch.Generator(device=gpu.dev).manual_seed(V)
    temps = [float("inf"), 3.4e38, 2e38, 1e38]
    X = ((torch.rand((len(temps), V), device=gpu.dev, generator=g) * 2 - 1) * 3.3e38).to(getattr(torch, dt))
    X[:, V // 3], X[:, V // 2] = 3.3e38, -3.3e38
    temp = torch.tensor(temps, device=gpu.dev)
    for at in (V // 3, V // 2, V - 1):
        tl.check(gpu, X, torch.full((len(temps),), at, device=gpu.dev, dtype=torch.int32), temp, 6)
    # with a token at +Inf, at a finite temperature as at the infinite one, nothing else counts
    X[:, 5] = float("inf")
    tl.check(gpu, X, torch.full((len(temps),), 5, device=gpu.dev, dtype=torch.int32), temp, 6)
    tl.check(gpu, X, torch.full((len(temps),), 9, device=gpu.dev, dtype=torch.int32), temp, 6)
