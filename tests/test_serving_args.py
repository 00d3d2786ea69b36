"""Argument checks of the serving calls, without a GPU: stand-in tensors go through the binding, whose library is replaced by
one that records the call. What would make a kernel read or write out of bounds is refused before any pointer is taken."""
import pytest
import torch

import paper_2601_21238_b200 as pk
from paper_2601_21238_b200 import binding as B

I32, F32, BF16, I8 = torch.int32, torch.float32, torch.bfloat16, torch.int8


class Dev:
    index = 0


class Fake:
    """The attributes of a CUDA tensor that the binding reads."""

    def __init__(self, shape, dtype=F32, strides=None, device=0, cuda=True):
        self.shape, self.dtype, self.is_cuda = tuple(shape), dtype, cuda
        self._device = device if cuda else -1
        self.device = Dev() if device == 0 else type("D", (), {"index": device})()
        dense, n = [], 1
        for s in reversed(self.shape):
            dense.insert(0, n)
            n *= s
        self._strides, self._dense = tuple(strides or dense), strides is None or tuple(strides) == tuple(dense)

    def stride(self, k=None):
        return self._strides if k is None else self._strides[k]

    def is_contiguous(self):
        return self._dense

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def get_device(self):
        return self._device

    def data_ptr(self):
        return 4096


class Lib:
    def __init__(self):
        self.called = []

    def __getattr__(self, name):
        return lambda *a: self.called.append((name, a)) or 0


@pytest.fixture
def ctx():
    c = pk.Context.__new__(pk.Context)
    c._torch, c._L, c._h, c.device = torch, Lib(), None, 0
    c._kinds = B._kinds(torch)
    c._i32, c._f32 = I32, F32
    names = ("torch.float32", "torch.bfloat16")
    c._row_kinds = {(names[0],): (F32,), (names[1],): (BF16,), names: (F32, BF16)}
    c._raw_stream = lambda stream: 0
    return c


T, HQ, HK, D, NP, S, NB, W = 12, 4, 2, 64, 5, 16, 3, 2


def plan():
    return dict(cached_lens=Fake((NB,), I32), new_lens=Fake((NB,), I32), free_pages=Fake((7,), I32), page_size=S, block_table=Fake((NB, W), I32),
                cu_new=Fake((NB + 1,), I32), kv_lens=Fake((NB,), I32), slot_map=Fake((T,), I32), pos_ids=Fake((T,), I32), pages_used=Fake((1,), I32))


def dense():
    return dict(QKV=Fake((T, (HQ + 2 * HK) * D), BF16), pos_ids=Fake((T,), I32), Hq=HQ, Hkv=HK, w_q=Fake((D,)), w_k=Fake((HK, D)), norm=pk.NORM_RMS,
                eps=1e-6, cs=Fake((9, D)), rope=pk.ROPE_HALF, Qo=Fake((T, HQ, D), BF16), Ko=Fake((T, HK, D), BF16))


def append(i8=False):
    kind = I8 if i8 else BF16
    return dict(QKV=Fake((T, (HQ + 2 * HK) * D), F32), pos_ids=Fake((T,), I32), slot_map=Fake((T,), I32), Hq=HQ, Hkv=HK, w_q=None, w_k=None, norm=pk.NORM_L2,
                eps=1e-6, cs=Fake((9, 32)), rope=pk.ROPE_PAIRS, s_k=Fake((9,)) if i8 else None, s_v=Fake((HK, D)) if i8 else None, bits=8,
                Qo=Fake((T, HQ, D), BF16), Kp=Fake((NP, HK, S, D), kind), Vp=Fake((NP, HK, S, D), kind))


def attend(i8=False):
    kind = I8 if i8 else BF16
    return dict(Q=Fake((T, HQ, D), BF16), cu_new=Fake((NB + 1,), I32), max_new=8, block_table=Fake((NB, W), I32), kv_lens=Fake((NB,), I32),
                Kp=Fake((NP, HK, S, D), kind), Vp=Fake((NP, HK, S, D), kind), s_k=Fake((32,)) if i8 else None, s_v=Fake((HK, D)) if i8 else None,
                scale=0.125, causal=True, out_dtype=pk.OUT_BF16, O=Fake((T, HQ, D), BF16))


def sample():
    f = lambda: Fake((6,))  # noqa: E731
    return dict(logits=Fake((6, 100)), temperature=f(), top_k=Fake((6,), I32), top_p=f(), min_p=f(), u=f(), tokens=Fake((6,), I32), probs=f(),
                kept=Fake((6,), I32))


MAKE = dict(page_plan=plan, qk_norm_rope=dense, kv_append_paged=append, paged_attention=attend, sample_tokens=sample)


@pytest.mark.parametrize("name", MAKE)
def test_consistent_arguments_reach_the_library(ctx, name):
    getattr(ctx, name)(**MAKE[name]())
    assert [n for n, _ in ctx._L.called] == [name]
    if name in ("kv_append_paged", "paged_attention"):
        getattr(ctx, name)(**MAKE[name](True))
        assert len(ctx._L.called) == 2


def test_strided_rows_and_left_out_limits_are_allowed(ctx):
    a = dense()
    a["QKV"] = Fake((T, (HQ + 2 * HK) * D), BF16, strides=(1024, 1))          # rows of a wider buffer
    a["Qo"], a["Ko"] = Fake((T, HQ, D), BF16, strides=(D, T * D, 1)), Fake((T, HK, D), BF16, strides=(D, T * D, 1))   # head-major
    a["w_q"] = a["w_k"] = a["cs"] = None
    ctx.qk_norm_rope(**a)
    args = ctx._L.called[0][1]
    assert args[2] == 1024 and args[-4:-1] == (D, T * D, pk.OUT_BF16) and args[9:13] == (None, 0, None, 0)
    b = sample()
    b.update(temperature=None, top_k=None, top_p=None, min_p=None, probs=None, kept=None, logits=Fake((6, 100), BF16, strides=(131, 1)))
    ctx.sample_tokens(**b)
    assert ctx._L.called[1][1][3] == 131


BAD = [("page_plan", "cached_lens", Fake((NB + 1,), I32), B.ERR_DIM), ("page_plan", "cu_new", Fake((NB,), I32), B.ERR_DIM),
       ("page_plan", "pos_ids", Fake((T - 1,), I32), B.ERR_DIM), ("page_plan", "block_table", Fake((NB, W), torch.int64), B.ERR_BITS),
       ("page_plan", "free_pages", Fake((7,), I32, cuda=False), B.ERR_CUDA), ("page_plan", "kv_lens", Fake((NB,), I32, device=1), B.ERR_CUDA),
       ("page_plan", "block_table", Fake((NB, W), I32, strides=(1, NB)), B.ERR_ALIGN), ("page_plan", "pages_used", None, B.ERR_NULL),
       ("qk_norm_rope", "QKV", Fake((T, (HQ + 2 * HK) * D + 1), BF16), B.ERR_DIM), ("qk_norm_rope", "QKV", Fake((T, (HQ + 2 * HK) * D), torch.float16), B.ERR_BITS),
       ("qk_norm_rope", "QKV", Fake((T, (HQ + 2 * HK) * D), BF16, strides=(1, T)), B.ERR_ALIGN), ("qk_norm_rope", "pos_ids", Fake((T - 1,), I32), B.ERR_DIM),
       ("qk_norm_rope", "w_q", Fake((D + 1,)), B.ERR_DIM), ("qk_norm_rope", "w_k", Fake((HK + 1, D)), B.ERR_DIM), ("qk_norm_rope", "cs", Fake((9, D), BF16), B.ERR_BITS),
       ("qk_norm_rope", "Ko", Fake((T, HK, D), F32), B.ERR_BITS), ("qk_norm_rope", "Ko", Fake((T, HQ, D), BF16), B.ERR_DIM),
       ("qk_norm_rope", "Qo", Fake((T, HQ, D), BF16, strides=(HQ * D * 2, D * 2, 2)), B.ERR_ALIGN), ("qk_norm_rope", "Qo", Fake((T, HQ, D), BF16, device=1), B.ERR_CUDA),
       ("kv_append_paged", "slot_map", Fake((T + 1,), I32), B.ERR_DIM), ("kv_append_paged", "slot_map", None, B.ERR_NULL),
       ("kv_append_paged", "Vp", Fake((NP, HK, S, D), I8), B.ERR_BITS), ("kv_append_paged", "Vp", Fake((NP + 1, HK, S, D), BF16), B.ERR_DIM),
       ("kv_append_paged", "Kp", Fake((NP, HK + 1, S, D), BF16), B.ERR_DIM), ("kv_append_paged", "Kp", Fake((NP, HK, S, D), F32), B.ERR_BITS),
       ("kv_append_paged", "Qo", Fake((T, HQ, D), F32), B.ERR_BITS), ("kv_append_paged", "Kp", Fake((NP, HK, S), BF16), B.ERR_DIM),
       ("paged_attention", "Q", Fake((T, HQ, D + 16), BF16), B.ERR_DIM), ("paged_attention", "Q", Fake((T, HQ, D), F32), B.ERR_BITS),
       ("paged_attention", "cu_new", Fake((NB,), I32), B.ERR_DIM), ("paged_attention", "kv_lens", Fake((NB + 2,), I32), B.ERR_DIM),
       ("paged_attention", "O", Fake((T, HQ, D), F32), B.ERR_BITS), ("paged_attention", "O", Fake((T - 1, HQ, D), BF16), B.ERR_DIM),
       ("paged_attention", "out_dtype", pk.OUT_INT32, B.ERR_BITS), ("paged_attention", "Kp", Fake((NP, HK, S, D), I8), B.ERR_BITS),
       ("sample_tokens", "logits", Fake((6, 100), torch.float16), B.ERR_BITS), ("sample_tokens", "logits", Fake((6, 100), strides=(200, 2)), B.ERR_ALIGN),
       ("sample_tokens", "u", Fake((5,)), B.ERR_DIM), ("sample_tokens", "u", None, B.ERR_NULL), ("sample_tokens", "top_k", Fake((6,)), B.ERR_BITS),
       ("sample_tokens", "tokens", Fake((6,), torch.int64), B.ERR_BITS), ("sample_tokens", "probs", Fake((7,)), B.ERR_DIM)]


@pytest.mark.parametrize("name,arg,value,code", BAD)
def test_bad_arguments_are_refused_before_the_library_is_called(ctx, name, arg, value, code):
    a = MAKE[name]()
    a[arg] = value
    with pytest.raises(pk.StwqError) as e:
        getattr(ctx, name)(**a)
    assert e.value.code == code and ctx._L.called == []


@pytest.mark.parametrize("name", ["kv_append_paged", "paged_attention"])
@pytest.mark.parametrize("arg,value,code", [("s_k", None, B.ERR_NULL), ("s_v", None, B.ERR_NULL), ("s_v", Fake((HQ, D)), B.ERR_DIM), ("s_k", Fake((9,), BF16), B.ERR_BITS)])
def test_codes_need_their_scales(ctx, name, arg, value, code):
    a = MAKE[name](True)
    a[arg] = value
    with pytest.raises(pk.StwqError) as e:
        getattr(ctx, name)(**a)
    assert e.value.code == code and ctx._L.called == []


def test_no_context_is_an_error_of_every_entry_point():
    lib = B.load_library()
    none = lambda fn: fn(*[0.0 if t is B.C.c_float else 0 if t in (B.C.c_int, B.C.c_int64) else None for t in fn.argtypes])  # noqa: E731
    for name in ("page_plan", "qk_norm_rope", "kv_append_paged", "paged_attention", "sample_tokens", "stwq_reserve_paged_attention"):
        assert none(getattr(lib, name)) == B.ERR_NULL
