"""The serving calls at the limits that their documentation names: lengths next to 2^31, the largest batches, values that are no
numbers."""
import subprocess
import sys

import numpy as np
import pytest

from conftest import ROOT
from test_gpu_serving import run_plan

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


ERR_PAGES, MAX = -12, 2 ** 31 - 1


@pytest.mark.parametrize("S,W,cached,new,table", [
    (715827882, 3, 2147483640, 100, [1, 0, 2]),                  # the row ends after 6 tokens, positions pass 2^31 after 8
    (16, 134217727, 2147483632 - 3, 40, None),                   # the same with a long row
    (MAX, 1, 2 ** 30 + 5, 3, [0]),                               # cached + page size - 1 is beyond 2^31
    (MAX, 1, MAX, 2, [0]), (2 ** 30, 1, 0, 7, [-9])])
def test_page_plan_next_to_2_31(gpu, S, W, cached, new, table):
    torch = gpu.torch
    if table is None:                                            # page 5 everywhere
        row = torch.full((1, W), 5, dtype=torch.int32, device=gpu.dev)
    else:
        row = gpu.T(np.array([table], np.int32))
    e = lambda n: torch.full((n,), -77, dtype=torch.int32, device=gpu.dev)  # noqa: E731
    i32 = lambda *a: gpu.T(np.array(a, np.int32))  # noqa: E731
    cu, kv, slots, pos, used = e(2), e(1), e(new + 2), e(new + 2), e(1)
    gpu.ctx.page_plan(i32(cached), i32(new), i32(1), S, row, cu, kv, slots, pos, used)
    fits = cached + new <= W * S
    assert gpu.ctx.stwq_device_status() == (0 if fits else ERR_PAGES)
    first_new = -(-cached // S)                                  # the first page that has to come from the free list, whose page is 1
    want = []
    for t in range(cached, cached + new):
        page = None if t >= W * S else 1 if t // S >= first_new else 5 if table is None else table[t // S]
        want.append(-1 if page is None or page * S + t % S > MAX else page * S + t % S)
    assert cu.tolist() == [0, new] and kv.item() == min(cached + new, W * S)
    assert slots.tolist() == want + [-1, -1]
    assert pos.tolist() == [min(t, MAX) for t in range(cached, cached + new)] + [-1, -1]
    assert used.item() == -(-min(cached + new, W * S) // S) - first_new
    if table is not None:
        table = [1 if first_new <= i < -(-min(cached + new, W * S) // S) else p for i, p in enumerate(table)]
        assert row.tolist() == [table]


@pytest.mark.parametrize("B", [4084, 4085, 4090, 4095])
def test_page_plan_of_large_batches_in_a_fresh_process(B):
    """The first plan of a process (a larger one before it could have raised the kernel's shared memory limit)."""
    code = f"""
import torch, paper_2601_21238_b200 as pk
z = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")
ctx = pk.Context(0)
slots = z({B})
ctx.page_plan(z({B}), z({B}) + 1, torch.arange({B}, dtype=torch.int32, device="cuda"), 16, z({B}, 1), z({B} + 1), z({B}), slots, z({B}), z(1))
assert ctx.stwq_device_status() == 0
assert torch.equal(slots, 16 * torch.arange({B}, dtype=torch.int32, device="cuda"))
ctx.close()
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
