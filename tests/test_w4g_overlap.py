"""gps_fold_group4 refuses outputs over operands and over each other, on the host, before anything of the context is used."""
import ctypes as C

import pytest
import torch

from paper_2601_21238_b200 import binding as B

N, K, GROUP = 6, 256, 32
BASE = 1 << 20                                                # addresses that nothing reads: refused calls touch no memory
W_BYTES, SCH_BYTES, WP_BYTES = N * K * 4, K * 4, N * K // 2


def fold(W, s_ch, Wp, s_g, s_dtype):
    ctx = C.create_string_buffer(1 << 16)                     # all zeros: no SMs, and nothing to launch on
    return B.load_library().gps_fold_group4(C.addressof(ctx), W, N, K, s_ch, GROUP, Wp, s_g, s_dtype, None)


@pytest.mark.parametrize("s_dtype", [0, 1])
@pytest.mark.parametrize("out,over", [("Wp", "W"), ("Wp", "s_ch"), ("s_g", "W"), ("s_g", "s_ch"), ("s_g", "Wp"), ("Wp", "s_g")])
@pytest.mark.parametrize("end", ["same", "first", "last"])
def test_outputs_over_operands_or_each_other(out, over, end, s_dtype):
    sizes = dict(W=W_BYTES, s_ch=SCH_BYTES, Wp=WP_BYTES, s_g=N * (K // GROUP) * (4 if s_dtype == 0 else 2))
    at = dict(W=BASE, s_ch=2 * BASE, Wp=3 * BASE, s_g=4 * BASE)
    last16 = lambda n: (n - 1) // 16 * 16  # noqa: E731       (the alignment of every operand)
    at[out] = at[over] + dict(same=0, first=-last16(sizes[out]), last=last16(sizes[over]))[end]
    assert fold(**at, s_dtype=s_dtype) == B.ERR_ALIGN


@pytest.mark.skipif(torch.cuda.is_available(), reason="what passes the checks goes on to the device")
def test_neighbours_are_not_refused_for_it():
    """Side by side without a shared byte: whatever comes after the checks (no device is here), it is not a refusal."""
    at = dict(W=BASE, s_ch=BASE + W_BYTES, Wp=BASE + W_BYTES + SCH_BYTES, s_g=BASE + W_BYTES + SCH_BYTES + WP_BYTES)
    assert fold(**at, s_dtype=0) not in (B.ERR_ALIGN, B.ERR_DIM, B.ERR_NULL, B.ERR_BITS)
