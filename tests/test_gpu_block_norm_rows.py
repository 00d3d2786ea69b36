"""block_norm with many rows for each team of warps, against 64 bits: the slots that a team's rows take in turn, rows that are skipped or
reported between live ones, ids and conditioning of their own for every row."""
import numpy as np
import pytest

import test_gpu_block_norm as tn
from test_gpu_block_norm import gpu  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

G, P = 11, 37
ERR_POS_RANGE = -8


def teams(gpu, C):  # noqa: F811
    """The most teams that are at work at once (by the launch's rule for many rows): with R times as many rows each has R or more."""
    sm = gpu.torch.cuda.get_device_properties(0).multi_processor_count
    warps = (C // 8 + 31) // 32
    if warps <= 3:                                            # a warp holds a row, four teams a block
        return 4 * (1024 if warps == 1 else 512) // 128 * sm
    for v in (2, 3):
        t = (warps + v - 1) // v
        if t <= 16 and (v == 3 or 2 * t < 3 * ((warps + 2) // 3)):
            return 512 // (32 * t) * sm
    return sm


def scattered(gpu, M, y, seed):  # noqa: F811
    """Positions and conditioning ids of M rows; which are skipped, which have a bad conditioning id, which a bad position (codes only)."""
    r = np.random.default_rng(seed)
    pos, cond = r.integers(0, P, M), r.integers(0, G, M)
    what = r.random(M)
    dead, bad_c, bad_p = what < 0.15, (what >= 0.15) & (what < 0.2), (what >= 0.2) & (what < 0.25)
    dead[M // 3:M // 3 + M // 4] = True                       # whole teams without a live row, or with one
    dead[M // 3 + M // 8] = False
    dead[[0, 1, M - 1]], bad_c[[2, M - 2]], bad_p[[3, M - 3]] = True, True, True
    bad_c &= ~dead
    bad_p &= ~dead & ~bad_c
    pos[bad_p] = r.choice([P, -2, 1 << 30, -(1 << 31)], int(bad_p.sum()))     # floating outputs need no position: these are live rows
    pos[dead] = -1
    cond[bad_c] = r.choice([G, -1, 1 << 30, -(1 << 31)], int(bad_c.sum()))
    cond[dead & (r.random(M) < 0.5)] = 99
    T = lambda a: gpu.torch.from_numpy(a.astype(np.int32)).to(gpu.dev)  # noqa: E731
    return T(pos), T(cond), dead, bad_c, bad_p if y == "i8" else np.zeros(M, bool)


def check(gpu, a, dead, bad_c, bad_p):  # noqa: F811
    torch = gpu.torch
    H, O = a["H"].clone(), a["O"]
    at = torch.from_numpy(dead).to(gpu.dev)
    a["H"][at] = float("nan")                                 # a skipped row is not read
    if O is not None:
        O[at] = float("nan")
    before = {k: a[k].clone() for k in ("Hout", "Y") if a[k] is not None}
    gpu.ctx.block_norm(**a)
    assert gpu.ctx.stwq_device_status() == (ERR_POS_RANGE if (bad_c | bad_p).any() else 0)
    for k, was in before.items():
        assert torch.equal(a[k][at], was[at])
    bits = {torch.float32: torch.int32, torch.bfloat16: torch.int16}
    rows = torch.from_numpy(np.flatnonzero(bad_c)).to(gpu.dev)
    if a["Hout"] is not None:
        assert torch.equal(a["Hout"][rows].view(bits[H.dtype]), H[rows].view(bits[H.dtype]))
    if a["Y"] is not None:
        assert not a["Y"][rows].any() and not a["Y"][torch.from_numpy(np.flatnonzero(bad_p)).to(gpu.dev)].any()

    summed = np.flatnonzero(~dead & ~bad_c)                   # these have their sum, those without a bad position also their output
    part = lambda t: None if t is None else t[torch.from_numpy(summed).to(gpu.dev)]  # noqa: E731
    h, e, y, ey = tn.reference(dict(a, H=part(H), O=part(O), cond_ids=part(a["cond_ids"])))
    if a["Hout"] is not None:
        tn.check_store(part(a["Hout"]), h, e, H.dtype == torch.bfloat16)
    if a["Y"] is None:
        return
    good = np.flatnonzero(~bad_p[summed])
    got, y, ey = part(a["Y"])[torch.from_numpy(good).to(gpu.dev)], y[good], ey[good]
    if got.dtype != torch.int8:
        tn.check_store(got, y, ey, got.dtype == torch.bfloat16)
        return
    rt = 1 / tn.f64(a["s_tok"])[part(a["pos_ids"]).cpu().numpy()[good]][:, None]
    u, eu = y * rt, ey * rt + 2 * tn.U * np.abs(y * rt)
    assert (np.abs(got.cpu().numpy() - np.clip(u, -128, 127)) <= 0.5 + eu).all()


# C, rows for each team, types of H, O and Y, norms, and whether a floating output is divided by s_ch: a row in a warp (one, two and three
# vectors), in two to sixteen warps; with one slot where two do not fit (16384 with two fp32 operands, 12288 beside s_ch)
FORMS = [(64, 3, "f32", "bf16", "bf16", 1, 1, False), (200, 5, "bf16", "bf16", "i8", 0, 3, True), (64, 32, "bf16", "f32", "f32", 3, 1, False),
         (256, 3, "bf16", "bf16", "f32", 3, 3, True), (264, 4, "f32", "f32", "bf16", 0, 3, False), (512, 7, "f32", "bf16", "i8", 1, 3, True), (512, 3, "bf16", None, "bf16", 0, 1, True),
         (520, 4, "bf16", "bf16", "bf16", 3, 3, False), (640, 6, "f32", "bf16", "i8", 0, 3, True), (768, 3, "f32", "f32", "f32", 1, 0, True),
         (1112, 4, "bf16", None, "i8", 0, 1, True), (1280, 3, "f32", "bf16", "bf16", 0, 3, False), (1280, 9, "bf16", "bf16", None, 3, 0, False),
         (1920, 10, "bf16", "bf16", "i8", 0, 3, True), (2048, 3, "f32", "bf16", "bf16", 3, 3, True), (4096, 4, "bf16", "bf16", "bf16", 1, 1, False),
         (8192, 4, "f32", "f32", "i8", 1, 3, True), (12288, 4, "f32", "f32", "i8", 0, 3, True), (12288, 3, "f32", "f32", "f32", 3, 1, True),
         (12296, 3, "bf16", "bf16", "bf16", 0, 3, False), (16384, 3, "f32", "f32", "bf16", 3, 3, False), (16384, 5, "f32", "f32", "i8", 1, 1, True)]


@pytest.mark.parametrize("C,R,h,o,y,post,pre,s_ch", FORMS)
def test_rows_in_turn(gpu, C, R, h, o, y, post, pre, s_ch):  # noqa: F811
    M = R * teams(gpu, C) - 5
    a = tn.make(gpu, M, C, h=h, o=o, y=y, post=post, pre=pre, G=G, seed=C + R, s_ch=s_ch)
    a["pos_ids"], a["cond_ids"], dead, bad_c, bad_p = scattered(gpu, M, y, C + R)
    check(gpu, a, dead, bad_c, bad_p)


@pytest.mark.parametrize("C,R", [(128, 4), (640, 4), (1920, 4), (16384, 3)])
def test_rows_in_turn_in_place(gpu, C, R):  # noqa: F811
    """The sum replaces H and the output O while the rows behind are on their way: as the same call with buffers of its own, which is checked."""
    M = R * teams(gpu, C) + 3
    a = tn.make(gpu, M, C, h="f32", o="f32", y="f32", post=1, pre=3, G=G, seed=C)
    a["pos_ids"], a["cond_ids"], dead, bad_c, bad_p = scattered(gpu, M, "f32", C)
    H, O = a["H"].clone(), a["O"].clone()
    check(gpu, a, dead, bad_c, bad_p)
    b = dict(a, H=H, O=O, Hout=H, Y=O)
    gpu.ctx.block_norm(**b)
    assert gpu.ctx.stwq_device_status() == ERR_POS_RANGE
    live = gpu.torch.from_numpy(~dead).to(gpu.dev)
    assert gpu.torch.equal(H[live], a["Hout"][live]) and gpu.torch.equal(O[live], a["Y"][live])


@pytest.mark.parametrize("C", [96, 640, 1280, 16384])
def test_one_conditioning_row_and_none(gpu, C):  # noqa: F811
    for G_ in (0, 1):
        a = tn.make(gpu, 4 * teams(gpu, C), C, h="f32", o="f32", y="f32", G=G_, seed=2 * C)
        assert a["cond_ids"] is None
        tn.run_and_check(gpu, a)
