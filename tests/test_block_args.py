"""Argument checks of block_norm, gps_fold_group4, linear_w4g and token_logprobs without a GPU: stand-in tensors go through the
binding, whose library is replaced by one that records the call; and the C entry points refuse what they can see on the host."""
import pytest
import torch

import paper_2601_21238_b200 as pk
from paper_2601_21238_b200 import binding as B
from test_serving_args import BF16, F32, I8, I32, Fake, ctx  # noqa: F401  (ctx: a fixture)

U8 = torch.uint8
M, C, G, P, K, N, V, TOP = 12, 64, 3, 9, 256, 40, 100, 5


def norm():
    ada = lambda: Fake((G, C), BF16, strides=(6 * C, 1))  # noqa: E731
    return dict(H=Fake((M, C)), O=Fake((M, C), BF16), cond_ids=Fake((M,), I32), gate=ada(), scale=ada(), shift=ada(), post_norm=pk.NORM_RMS,
                w_post=Fake((C,)), b_post=None, res_scale=1.0, pre_norm=pk.NORM_LAYER, w_pre=Fake((C,)), b_pre=Fake((C,)), eps=1e-6, Hout=Fake((M, C)),
                pos_ids=Fake((M,), I32), s_ch=Fake((C,)), s_tok=Fake((P,)), bits=8, Y=Fake((M, C), I8))


def fold():
    return dict(W=Fake((N, K)), s_ch=Fake((K,)), Wp=Fake((N, K // 2), U8), s_g=Fake((N, 4), BF16))


def linear():
    return dict(X=Fake((6, K), BF16), Wp=Fake((N, K // 2), U8), s_g=Fake((N, 4)), bias=Fake((N,)), act=0, out_dtype=pk.OUT_BF16, Y=Fake((6, N), BF16))


def logprobs():
    i, f = lambda *s: Fake(s, I32), lambda *s: Fake(s)  # noqa: E731
    return dict(logits=Fake((6, V)), temperature=f(6), tokens=i(6), logprobs=f(6), ranks=i(6), entropy=f(6), top_ids=i(6, TOP), top_logprobs=f(6, TOP))


MAKE = dict(block_norm=norm, gps_fold_group4=fold, linear_w4g=linear, token_logprobs=logprobs)


@pytest.mark.parametrize("name", MAKE)
def test_consistent_arguments_reach_the_library(ctx, name):  # noqa: F811
    a = MAKE[name]()
    if name == "gps_fold_group4":
        ctx._stream = lambda stream: 0
    getattr(ctx, name)(**a)
    assert [n for n, _ in ctx._L.called] == [name]


def test_strides_types_and_sizes_are_passed_on(ctx):  # noqa: F811
    a = norm()
    a.update(H=Fake((M, C), BF16, strides=(200, 1)), Hout=Fake((M, C), BF16, strides=(128, 1)), Y=Fake((M, C), strides=(96, 1)))
    ctx.block_norm(**a)
    got = ctx._L.called[0][1]
    assert got[2:4] == (200, pk.OUT_BF16) and got[5:9] == (C, pk.OUT_BF16, M, C) and got[10] == G and got[14:16] == (6 * C, pk.OUT_BF16)
    assert got[25] == 128 and got[-3:-1] == (96, pk.OUT_F32) and got[29] == P
    b = linear()
    b["X"], b["s_g"] = Fake((6, K), F32, strides=(300, 1)), Fake((N, 2), BF16)
    ctx.linear_w4g(**b)
    got = ctx._L.called[1][1]
    assert got[2:7] == (300, pk.OUT_F32, 6, K, N) and got[9:11] == (pk.OUT_BF16, 128)
    c = logprobs()
    c.update(logits=Fake((6, V), BF16, strides=(131, 1)), temperature=None, ranks=None, entropy=None, top_ids=None, top_logprobs=None)
    ctx.token_logprobs(**c)
    got = ctx._L.called[2][1]
    assert got[2:6] == (pk.OUT_BF16, 131, 6, V) and got[6] is None and got[9:14] == (None, None, 0, None, None)


BAD = [("block_norm", "H", Fake((M, C), torch.float16), B.ERR_BITS), ("block_norm", "H", Fake((M, C), strides=(1, M)), B.ERR_ALIGN), ("block_norm", "H", None, B.ERR_NULL),
       ("block_norm", "O", Fake((M, C + 8), BF16), B.ERR_DIM), ("block_norm", "O", Fake((M, C), I8), B.ERR_BITS), ("block_norm", "Hout", Fake((M, C), BF16), B.ERR_BITS),
       ("block_norm", "Hout", Fake((M - 1, C)), B.ERR_DIM), ("block_norm", "Y", Fake((M, C), I32), B.ERR_BITS), ("block_norm", "Y", Fake((M + 1, C), I8), B.ERR_DIM),
       ("block_norm", "Y", Fake((M, C), I8, strides=(2 * C, 2)), B.ERR_ALIGN), ("block_norm", "Y", Fake((M, C), cuda=False), B.ERR_CUDA),
       ("block_norm", "cond_ids", Fake((M - 1,), I32), B.ERR_DIM), ("block_norm", "cond_ids", None, B.ERR_NULL), ("block_norm", "cond_ids", Fake((M,), torch.int64), B.ERR_BITS),
       ("block_norm", "gate", Fake((G + 1, C), BF16, strides=(6 * C, 1)), B.ERR_DIM), ("block_norm", "scale", Fake((G, C), F32, strides=(6 * C, 1)), B.ERR_DIM),
       ("block_norm", "shift", Fake((G, C), BF16), B.ERR_DIM), ("block_norm", "w_post", Fake((C + 1,)), B.ERR_DIM), ("block_norm", "b_pre", Fake((C,), BF16), B.ERR_BITS),
       ("block_norm", "pos_ids", Fake((M + 1,), I32), B.ERR_DIM), ("block_norm", "s_ch", Fake((P,)), B.ERR_DIM), ("block_norm", "s_tok", Fake((P,), BF16), B.ERR_BITS),
       ("block_norm", "w_pre", Fake((C,), device=1), B.ERR_CUDA),
       ("gps_fold_group4", "Wp", Fake((N, K), U8), B.ERR_DIM), ("gps_fold_group4", "W", Fake((N, K), BF16), B.ERR_BITS), ("gps_fold_group4", "s_g", Fake((N, 5)), B.ERR_DIM),
       ("gps_fold_group4", "s_g", Fake((N + 1, 4)), B.ERR_DIM), ("gps_fold_group4", "s_ch", Fake((N,)), B.ERR_DIM), ("gps_fold_group4", "W", Fake((N, K), strides=(1, N)), B.ERR_ALIGN),
       ("linear_w4g", "X", Fake((6, K), torch.float16), B.ERR_BITS), ("linear_w4g", "X", Fake((6, K), BF16, strides=(1, 6)), B.ERR_ALIGN), ("linear_w4g", "Wp", Fake((N, K), U8), B.ERR_DIM),
       ("linear_w4g", "Wp", Fake((N, K // 2), I8), B.ERR_BITS), ("linear_w4g", "s_g", Fake((N, 3)), B.ERR_DIM), ("linear_w4g", "s_g", Fake((N, 4), torch.float16), B.ERR_BITS),
       ("linear_w4g", "s_g", Fake((N, 0)), B.ERR_DIM), ("linear_w4g", "bias", Fake((K,)), B.ERR_DIM), ("linear_w4g", "Y", Fake((6, N)), B.ERR_BITS), ("linear_w4g", "Y", Fake((7, N), BF16), B.ERR_DIM),
       ("linear_w4g", "Y", Fake((6, N), BF16, strides=(N + 8, 1)), B.ERR_ALIGN), ("linear_w4g", "out_dtype", pk.OUT_INT8, B.ERR_BITS), ("linear_w4g", "Wp", Fake((N, K // 2), U8, device=1), B.ERR_CUDA),
       ("token_logprobs", "logits", Fake((6, V), torch.float16), B.ERR_BITS), ("token_logprobs", "logits", Fake((6, V), strides=(2 * V, 2)), B.ERR_ALIGN),
       ("token_logprobs", "tokens", Fake((6,), torch.int64), B.ERR_BITS), ("token_logprobs", "tokens", Fake((7,), I32), B.ERR_DIM), ("token_logprobs", "temperature", Fake((1,)), B.ERR_DIM),
       ("token_logprobs", "logprobs", Fake((6,), BF16), B.ERR_BITS), ("token_logprobs", "ranks", Fake((6,)), B.ERR_BITS), ("token_logprobs", "entropy", Fake((6, 1)), B.ERR_DIM),
       ("token_logprobs", "top_ids", Fake((6, TOP), torch.int64), B.ERR_BITS), ("token_logprobs", "top_ids", Fake((6, TOP + 1), I32), B.ERR_DIM), ("token_logprobs", "top_logprobs", Fake((5, TOP)), B.ERR_DIM),
       ("token_logprobs", "entropy", Fake((6,), cuda=False), B.ERR_CUDA)]


@pytest.mark.parametrize("name,arg,value,code", BAD)
def test_bad_arguments_are_refused_before_the_library_is_called(ctx, name, arg, value, code):  # noqa: F811
    a = MAKE[name]()
    a[arg] = value
    with pytest.raises(pk.StwqError) as e:
        getattr(ctx, name)(**a)
    assert e.value.code == code and ctx._L.called == []


def test_no_context_is_an_error_of_every_entry_point():
    lib = B.load_library()
    none = lambda fn: fn(*[0.0 if t is B.C.c_float else 0 if t in (B.C.c_int, B.C.c_int64) else None for t in fn.argtypes])  # noqa: E731
    for name in MAKE:
        assert none(getattr(lib, name)) == B.ERR_NULL
