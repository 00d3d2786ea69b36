"""token_logprobs where its running reference m and its octaves m c meet their limits: sums with and without a rounded m c joined in a
thread, between warps and between the blocks of a cluster."""
import numpy as np
import pytest

import test_gpu_logprobs as tl
from test_gpu_logprobs import gpu  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

f32 = np.float32


def neighbours(t, sign, octaves):
    """Two fp32 logits, the larger first, some octaves apart at temperature t, on either side of |x| log2(e) / t = 1e6, up to which the kernel
    keeps x log2(e) / t as a rounded number; the one inside is taken where that rounding is largest."""
    c = f32(1.4426950408889634) / f32(t)
    inside = lambda x: abs(f32(x) * c) < f32(1e6)  # noqa: E731
    edge = f32(1e6) / c
    for _ in range(8):
        edge = np.nextafter(edge, f32(0))
    while inside(edge):
        edge = np.nextafter(edge, f32(np.inf))
    near, best = edge, (-1.0, None, None)                     # `edge`: the least magnitude outside
    for _ in range(400):
        near = np.nextafter(near, f32(0))
        apart = (float(edge) - float(near)) * float(c)
        if octaves[0] <= apart <= octaves[1]:
            off = abs(float(near * c) - float(near) * float(c))
            best = max(best, (off, near, edge))
    assert best[0] > 2.0 ** -7 and inside(best[1]) and not inside(best[2])
    return (best[2], best[1]) if sign > 0 else (-best[1], -best[2])


# where the two stand, in rows of which length, at which offset from 32-byte alignment, octaves between them
PLACES = dict(warps=(1024, 10, 300, 0, (0.05, 2.0)),
              warps_turned=(1024, 300, 10, 0, (0.05, 2.0)),
              end_and_vector=(1024, 7, 0, 1, (0.05, 2.0)),           # seven logits before the first aligned one: both are thread 0's
              two_vectors=(16384, 2048, 0, 0, (5.0, 8.0)),           # thread 0's second vector lifts its reference
              blocks=(128000, 90000, 100, 0, (0.05, 2.0)),
              blocks_turned=(128000, 100, 90000, 0, (0.05, 2.0)))


@pytest.mark.parametrize("place", PLACES)
def test_near_logits_on_both_sides_of_a_million_octaves(gpu, place):  # noqa: F811
    torch = gpu.torch
    V, at_hi, at_lo, shift, octaves = PLACES[place]
    temps, signs = (1e-5, 2e-5, 1e-3, 1.0), (1, -1)
    rows = [(t, s) + neighbours(t, s, octaves) for t in temps for s in signs]
    ld = (V + 15) // 8 * 8                                    # every row at the same offset from an aligned address
    buf = torch.empty((len(rows) * ld + 8,), device=gpu.dev)
    assert buf.data_ptr() % 32 == 0
    X = buf[shift:shift + len(rows) * ld].view(len(rows), ld)[:, :V]
    for b, (t, s, hi, lo) in enumerate(rows):
        X[b] = float(hi) - abs(float(hi)) * 0.5               # far below
        X[b, at_hi], X[b, at_lo] = float(hi), float(lo)
    temp = torch.tensor([r[0] for r in rows], device=gpu.dev)
    for at in (at_hi, at_lo):
        tokens = torch.full((len(rows),), at, device=gpu.dev, dtype=torch.int32)
        for k in (0, 3):
            tl.check(gpu, X, tokens, temp, k)
