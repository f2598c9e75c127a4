"""The extension's microscaled calls against stand-ins for the library: what they hand over, and that a call whose tensors do not hold what the kernels would
address is refused before the library is reached."""
import ctypes

import pytest
import torch

I32, I64, VP, SZ = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
NEED = 4096
BF, F8, E8 = torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu


class Library:
    SIGNATURES = [(ctypes.c_int, [I32, I32, I32, VP, I64, VP, I64, VP, I64, VP])] * 2 + [
        (SZ, [I32] * 3), (ctypes.c_int, [I32] * 3 + [VP, I64] * 4 + [VP, SZ, VP]),
        (ctypes.c_int, [I32] * 8 + [VP, VP, I64, I64] + [VP, VP, I64, I64, I64] * 2 + [VP, I64, VP, VP, VP]), (SZ, [VP]), (ctypes.c_int, [VP] * 12 + [SZ, VP])]

    def __init__(self):
        try:
            from paper_2505_19634_amd import binding
        except ImportError:
            import __graft_entry__
            __graft_entry__.build()
            from paper_2505_19634_amd import binding
        self.made, self.answer = [], 0

        def call(*args):
            self.made.append(args)
            return self.answer

        def attend(desc, *args):   # the descriptor lives as long as the call
            return call(binding.PagedMxDesc.from_buffer_copy(binding.PagedMxDesc.from_address(desc)), *args)
        fs = [call, call, lambda *a: NEED, call, call, lambda *a: NEED, attend]
        self.keep = [ctypes.CFUNCTYPE(res, *args)(f) for (res, args), f in zip(self.SIGNATURES, fs)]
        self.calls = type(binding.load().mx)(*(ctypes.cast(f, VP).value for f in self.keep))


@pytest.fixture()
def library():
    return Library()


WS = torch.zeros(NEED, dtype=torch.uint8)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


def bf(*shape):
    return torch.zeros(shape, dtype=BF)


def convert(**other):
    t = dict(W=bf(5, 96), codes=u8(5, 48), scales=u8(5, 3).view(E8), device=-1, stream=0)
    t.update(other)
    return t


def gemm(**other):
    t = dict(X=bf(3, 96), codes=u8(5, 48), scales=u8(5, 3), out=bf(3, 5), workspace=None, cached=WS, device=-1, stream=0)
    t.update(other)
    return t


def cache(pages=9):
    return dict(K=u8(pages, 2, 16, 64).view(F8), V=u8(pages, 2, 16, 64).view(F8), Ks=u8(pages, 2, 16, 2).view(E8), Vs=u8(pages, 2, 16, 2).view(E8))


def attention(**other):
    t = dict(Q=bf(7, 4, 64), **cache(), table=i32(3, 5), kv_len=i32(3), q_start=i32(4), max_new=None, scale=0.0, out=bf(7, 4, 64), lse=None, workspace=None, cached=WS,
             device=-1, stream=0)
    t.update(other)
    return t


def append(**other):
    t = dict(Knew=bf(7, 2, 64), Vnew=bf(7, 2, 64), **cache(), table=i32(3, 5), kv_len=i32(3), q_start=i32(4), device=-1, stream=0)
    t.update(other)
    return t


def ptrs(a, *names):
    return tuple(a[n].data_ptr() for n in names)


def test_what_a_call_hands_over(library):
    a = convert(W=torch.zeros(5, 128)[:, 16:112], codes=u8(5, 64)[:, :48], scales=u8(5, 7)[:, 2:5])
    assert library.calls.mxfp4_quantize(*a.values()) == 0
    w, c, s = ptrs(a, "W", "codes", "scales")
    assert library.made[0] == (5, 96, 0, w, 128, c, 64, s, 7, None)
    a = convert()
    assert library.calls.mxfp4_dequantize(*a.values()) == 0
    w, c, s = ptrs(a, "W", "codes", "scales")
    assert library.made[1] == (5, 96, 1, c, 48, s, 3, w, 96, None)
    a = gemm(out=bf(3, 9)[:, 2:7], stream=77)
    assert library.calls.skinny_gemm_mxfp4(*a.values()) == 0
    x, c, s, y = ptrs(a, "X", "codes", "scales", "out")
    assert library.made[2] == (3, 5, 96, x, 96, c, 48, s, 3, y, 9, WS.data_ptr(), NEED, 77)
    token = lambda n, d: u8(9, 16, 2, n).transpose(1, 2).view(d)
    a = attention(Q=bf(6, 8, 64).view(3, 2, 8, 64)[:, :, :4], out=bf(3, 2, 4, 64), q_start=None, lse=torch.zeros(6, 4), scale=0.5, K=token(64, F8), V=token(64, F8),
                  Ks=token(2, E8), Vs=token(2, E8), table=i32(3, 8)[:, :5])
    assert library.calls.verify_attention_paged_mxfp8(*a.values()) == 0
    m, *rest = library.made[3]
    d = m.paged
    assert (d.B, d.T, d.max_new, d.Hq, d.Hkv, d.D, d.page_tokens, d.pages, d.columns, d.dtype, d.scale) == (3, 6, 2, 4, 2, 64, 16, 9, 5, 1, 0.5)
    assert (d.q_stride_t, d.q_stride_h, d.o_stride_t, d.o_stride_h, d.table_stride) == (512, 64, 256, 64, 8)
    assert (d.page_stride_p, d.page_stride_h, d.page_stride_t) == (2048, 64, 128) and (m.scale_stride_p, m.scale_stride_h, m.scale_stride_t) == (64, 2, 4)
    assert tuple(rest) == ptrs(a, "Q", "K", "V", "Ks", "Vs", "table", "kv_len") + (None,) + ptrs(a, "out", "lse") + (WS.data_ptr(), NEED, None)
    a = attention(Q=torch.zeros(7, 4, 64), out=torch.zeros(7, 4, 64), max_new=3)
    assert library.calls.verify_attention_paged_mxfp8(*a.values()) == 0
    assert library.made[4][0].paged.dtype == 0 and library.made[4][0].paged.max_new == 3 and library.made[4][8] == a["q_start"].data_ptr()
    a = append()
    assert library.calls.kv_append_paged_mxfp8(*a.values()) == 0
    assert library.made[5] == (3, 7, 2, 64, 16, 9, 5, 1, *ptrs(a, "Knew", "Vnew"), 128, 64, *ptrs(a, "K", "V"), 2048, 1024, 64, *ptrs(a, "Ks", "Vs"), 64, 32, 2,
                               a["table"].data_ptr(), 5, *ptrs(a, "kv_len", "q_start"), None)
    library.answer = -5
    assert library.calls.mxfp4_quantize(*convert().values()) == -5


@pytest.mark.parametrize("name,make", [("verify_attention_paged_mxfp8", attention), ("skinny_gemm_mxfp4", gemm)])
def test_workspaces(library, name, make):
    call = getattr(library.calls, name)
    small = u8(3)
    assert call(*make(cached=None).values()) > 0 and call(*make(cached=small).values()) > 0
    assert not library.made
    assert call(*make(workspace=small, cached=None).values()) == 0     # the caller's own goes to the library as it is
    assert library.made[0][-3:-1] == (small.data_ptr(), 3)


@pytest.mark.parametrize("error,other", [
    (ValueError, dict(W=bf(4, 96))), (ValueError, dict(W=bf(5, 64))), (TypeError, dict(W=torch.zeros(5, 96, dtype=torch.float16))), (ValueError, dict(W=bf(96, 5).t())),
    (ValueError, dict(W=bf(480))), (ValueError, dict(codes=u8(5, 32))), (TypeError, dict(codes=torch.zeros(5, 48))), (ValueError, dict(codes=u8(5, 96)[:, ::2])),
    (ValueError, dict(codes=u8(1, 48).expand(5, -1))), (ValueError, dict(scales=u8(5, 2))), (ValueError, dict(scales=u8(4, 3))), (TypeError, dict(scales=torch.zeros(5, 3))),
    (TypeError, dict(W=None)), (ValueError, dict(device=0)), (ValueError, dict(codes=u8(5, 40), W=bf(5, 80)))])
def test_conversions_refuse(library, error, other):
    for call in (library.calls.mxfp4_quantize, library.calls.mxfp4_dequantize):
        with pytest.raises(error):
            call(*convert(**other).values())
    assert not library.made


@pytest.mark.parametrize("error,other", [
    (ValueError, dict(X=bf(3, 64))), (TypeError, dict(X=torch.zeros(3, 96))), (ValueError, dict(X=bf(96, 3).t())), (ValueError, dict(X=bf(1, 96).expand(3, -1))), (ValueError, dict(out=bf(3, 4))),
    (ValueError, dict(out=bf(4, 5))), (TypeError, dict(out=torch.zeros(3, 5))), (ValueError, dict(out=bf(5, 3).t())), (ValueError, dict(out=bf(1, 5).expand(3, -1))),
    (ValueError, dict(scales=u8(5, 4))), (TypeError, dict(codes=bf(5, 48))), (TypeError, dict(X=None)), (ValueError, dict(device=0))])
def test_product_refuses(library, error, other):
    with pytest.raises(error):
        library.calls.skinny_gemm_mxfp4(*gemm(**other).values())
    assert not library.made


CACHE = [(ValueError, dict(V=u8(8, 2, 16, 64).view(F8))), (TypeError, dict(K=bf(9, 2, 16, 64), V=bf(9, 2, 16, 64))), (TypeError, dict(V=u8(9, 2, 16, 64))),
         (ValueError, dict(V=u8(9, 16, 2, 64).transpose(1, 2).view(F8))), (ValueError, dict(Ks=u8(9, 2, 16, 4).view(E8), Vs=u8(9, 2, 16, 4).view(E8))),
         (ValueError, dict(Ks=u8(9, 2, 8, 2).view(E8), Vs=u8(9, 2, 8, 2).view(E8))), (ValueError, dict(Vs=u8(9, 16, 2, 2).transpose(1, 2).view(E8))), (TypeError, dict(Vs=u8(9, 2, 16, 2))),
         (TypeError, dict(Ks=torch.zeros(9, 2, 16, 2), Vs=torch.zeros(9, 2, 16, 2))), (ValueError, dict(Ks=u8(9, 2, 16, 4)[..., ::2], Vs=u8(9, 2, 16, 4)[..., ::2])),
         (ValueError, dict(Ks=u8(1, 2, 16, 2).expand(9, -1, -1, -1), Vs=u8(1, 2, 16, 2).expand(9, -1, -1, -1))), (ValueError, dict(kv_len=i32(2))), (ValueError, dict(q_start=i32(3))),
         (TypeError, dict(table=torch.zeros(3, 5))), (ValueError, dict(device=0)), (TypeError, dict(Ks=None))]


@pytest.mark.parametrize("error,other", CACHE + [
    (ValueError, dict(out=bf(6, 4, 64))), (TypeError, dict(out=torch.zeros(7, 4, 64))), (TypeError, dict(Q=torch.zeros(7, 4, 64, dtype=torch.float16), out=torch.zeros(7, 4, 64, dtype=torch.float16))),
    (ValueError, dict(Q=bf(7, 4, 128), out=bf(7, 4, 128))), (ValueError, dict(q_start=None)), (ValueError, dict(lse=torch.zeros(27))), (TypeError, dict(scale="large")),
    (TypeError, dict(max_new="many"))])
def test_attention_refuses(library, error, other):
    with pytest.raises(error):
        library.calls.verify_attention_paged_mxfp8(*attention(**other).values())
    assert not library.made


@pytest.mark.parametrize("error,other", CACHE + [
    (ValueError, dict(Vnew=bf(6, 2, 64))), (ValueError, dict(Vnew=bf(7, 4, 64)[:, :2])), (TypeError, dict(Vnew=torch.zeros(7, 2, 64))), (ValueError, dict(Knew=bf(7, 3, 64), Vnew=bf(7, 3, 64))),
    (TypeError, dict(Knew=u8(7, 2, 64), Vnew=u8(7, 2, 64))), (ValueError, dict(Knew=bf(7, 2, 32), Vnew=bf(7, 2, 32)))])
def test_append_refuses(library, error, other):
    with pytest.raises(error):
        library.calls.kv_append_paged_mxfp8(*append(**other).values())
    assert not library.made


def test_wrong_numbers_of_arguments(library):
    for call in ("mxfp4_quantize", "mxfp4_dequantize", "skinny_gemm_mxfp4", "kv_append_paged_mxfp8", "verify_attention_paged_mxfp8"):
        with pytest.raises(TypeError):
            getattr(library.calls, call)(1, 2)
