"""The extension's calls of the paged cache against stand-ins for the library: what they hand over, and that a call whose tensors do not hold what
the kernels would address is refused before the library is reached."""
import ctypes

import pytest
import torch

I32, I64, VP, SZ = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
NEED = 4096
BF = torch.bfloat16


class Library:
    SIGNATURES = [(SZ, [VP]), (ctypes.c_int, [VP] * 10 + [SZ, VP]), (ctypes.c_int, [I32] * 8 + [VP, VP, I64, I64, VP, VP, I64, I64, I64, VP, I64, VP, VP, VP]),
                  (ctypes.c_int, [I32] * 4 + [VP, I64] + [VP] * 6 + [SZ, VP]), (ctypes.c_int, [I32] * 3 + [VP, I64] + [VP] * 4),
                  (ctypes.c_int, [I32] * 4 + [VP, I64] + [VP] * 4), (ctypes.c_int, [I32] * 3 + [VP, I64] + [VP] * 4 + [SZ, VP]),
                  (ctypes.c_int, [VP, I32, I32, I64, I64, I64, VP, I32, VP, VP])]

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
            return call(binding.PagedDesc.from_buffer_copy(binding.PagedDesc.from_address(desc)), *args)
        fs = [lambda *a: NEED, attend] + [call] * 6
        self.keep = [ctypes.CFUNCTYPE(res, *args)(f) for (res, args), f in zip(self.SIGNATURES, fs)]
        self.calls = type(binding.load().paged)(*(ctypes.cast(f, VP).value for f in self.keep))


@pytest.fixture()
def library():
    return Library()


WS = torch.zeros(NEED, dtype=torch.uint8)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def attention(**other):
    t = dict(Q=torch.zeros(7, 4, 64, dtype=BF), K=torch.zeros(9, 2, 16, 64, dtype=BF), V=torch.zeros(9, 2, 16, 64, dtype=BF), table=i32(3, 5), kv_len=i32(3),
             q_start=i32(4), max_new=None, scale=0.0, out=torch.zeros(7, 4, 64, dtype=BF), lse=None, workspace=None, cached=WS, device=-1, stream=0)
    t.update(other)
    return t


def append(**other):
    t = dict(Knew=torch.zeros(7, 2, 64, dtype=BF), Vnew=torch.zeros(7, 2, 64, dtype=BF), K=torch.zeros(9, 2, 16, 64, dtype=BF), V=torch.zeros(9, 2, 16, 64, dtype=BF),
             table=i32(3, 5), kv_len=i32(3), q_start=i32(4), device=-1, stream=0)
    t.update(other)
    return t


def reserve(**other):
    t = dict(table=i32(3, 5), refs=i32(9), kv_len=i32(3), new=i32(3), page=16, copies=i32(3, 2), missing=i32(1), workspace=None, cached=WS, device=-1, stream=0)
    t.update(other)
    return t


def test_what_a_call_hands_over(library):
    qkv = torch.zeros(6, 8, 64, dtype=BF)
    a = attention(Q=qkv.view(3, 2, 8, 64)[:, :, :4], out=torch.zeros(3, 2, 4, 64, dtype=BF), q_start=None, lse=torch.zeros(6, 4), scale=0.5, stream=77,
                  K=torch.zeros(9, 16, 2, 64, dtype=BF).transpose(1, 2), V=torch.zeros(9, 16, 2, 64, dtype=BF).transpose(1, 2), table=i32(3, 8)[:, :5])
    assert library.calls.verify_attention_paged(*a.values()) == 0
    d, *rest = library.made[0]
    assert (d.B, d.T, d.max_new, d.Hq, d.Hkv, d.D, d.page_tokens, d.pages, d.columns, d.dtype, d.scale) == (3, 6, 2, 4, 2, 64, 16, 9, 5, 1, 0.5)
    assert (d.q_stride_t, d.q_stride_h, d.o_stride_t, d.o_stride_h, d.table_stride) == (512, 64, 256, 64, 8)
    assert (d.page_stride_p, d.page_stride_h, d.page_stride_t) == (2048, 64, 128)
    assert rest == [a[n].data_ptr() for n in ("Q", "K", "V", "table", "kv_len")] + [None] + [a[n].data_ptr() for n in ("out", "lse")] + [WS.data_ptr(), NEED, 77]
    a = attention(max_new=3)
    assert library.calls.verify_attention_paged(*a.values()) == 0
    assert library.made[1][0].max_new == 3 and library.made[1][6] == a["q_start"].data_ptr() and library.made[1][8] is None
    assert library.calls.verify_attention_paged(*attention().values()) == 0 and library.made[2][0].max_new == 7
    p = append()
    assert library.calls.kv_append_paged(*p.values()) == 0
    assert library.made[3] == (3, 7, 2, 64, 16, 9, 5, 1, p["Knew"].data_ptr(), p["Vnew"].data_ptr(), 128, 64, p["K"].data_ptr(), p["V"].data_ptr(), 2048, 1024, 64,
                               p["table"].data_ptr(), 5, p["kv_len"].data_ptr(), p["q_start"].data_ptr(), None)
    r = reserve()
    assert library.calls.kv_pages_reserve(*r.values()) == 0
    assert library.made[4] == (3, 5, 9, 16, r["table"].data_ptr(), 5, *(r[n].data_ptr() for n in ("refs", "kv_len", "new", "copies", "missing")), WS.data_ptr(), NEED, None)
    t, refs, n, o = i32(3, 5), i32(9), i32(3), i32(3)
    assert library.calls.kv_pages_fork(t, refs, n, o, -1, 5) == 0 and library.calls.kv_pages_free(t, refs, n, 32, None, -1, 5) == 0
    assert library.made[5] == (3, 5, 9, t.data_ptr(), 5, refs.data_ptr(), n.data_ptr(), o.data_ptr(), 5)
    assert library.made[6] == (3, 5, 9, 32, t.data_ptr(), 5, refs.data_ptr(), n.data_ptr(), None, 5)
    m, c = i32(4, 2), i32(2)
    assert library.calls.kv_pages_compact(t, refs, m, c, None, WS, -1, 5) == 0
    assert library.made[7] == (3, 5, 9, t.data_ptr(), 5, refs.data_ptr(), m.data_ptr(), c.data_ptr(), WS.data_ptr(), NEED, 5)
    pool = torch.zeros(4, 12, 2, 16, 64, dtype=BF)[:, 1:10]
    assert library.calls.kv_pages_copy(pool, m, c, -1, 5) == 0
    assert library.made[8] == (pool.data_ptr(), 4, 9, 12 * 4096, 4096, 4096, m.data_ptr(), 4, c.data_ptr(), 5)
    library.answer = -5
    assert library.calls.kv_pages_fork(t, refs, n, o, -1, 5) == -5


@pytest.mark.parametrize("name,make,at", [("verify_attention_paged", attention, -3), ("kv_pages_reserve", reserve, -3)])
def test_workspaces(library, name, make, at):
    call = getattr(library.calls, name)
    small = torch.zeros(3, dtype=torch.uint8)
    assert call(*make(cached=None).values()) > 0 and call(*make(cached=small).values()) > 0
    assert not library.made
    assert call(*make(workspace=small, cached=None).values()) == 0     # the caller's own goes to the library as it is
    assert library.made[0][at:-1] == (small.data_ptr(), 3)


UNFIT = [
    (ValueError, dict(out=torch.zeros(6, 4, 64, dtype=BF))), (ValueError, dict(out=torch.zeros(7, 4, 32, dtype=BF))), (TypeError, dict(out=torch.zeros(7, 4, 64))),
    (ValueError, dict(Q=torch.zeros(7, 64, 4, dtype=BF).transpose(1, 2))), (ValueError, dict(Q=torch.zeros(1, 4, 64, dtype=BF).expand(7, -1, -1))),
    (ValueError, dict(Q=torch.zeros(7, 64, dtype=BF))), (ValueError, dict(Q=torch.zeros(3, 2, 4, 64, dtype=BF), out=torch.zeros(3, 2, 4, 64, dtype=BF))),
    (TypeError, dict(Q=torch.zeros(7, 4, 64, dtype=torch.float16), out=torch.zeros(7, 4, 64, dtype=torch.float16))), (TypeError, dict(Q=torch.zeros(7, 4, 64), out=torch.zeros(7, 4, 64))),
    (ValueError, dict(V=torch.zeros(8, 2, 16, 64, dtype=BF))), (ValueError, dict(V=torch.zeros(9, 16, 2, 64, dtype=BF).transpose(1, 2))), (TypeError, dict(V=torch.zeros(9, 2, 16, 64))),
    (ValueError, dict(K=torch.zeros(9, 2, 16, 128, dtype=BF), V=torch.zeros(9, 2, 16, 128, dtype=BF))), (ValueError, dict(K=torch.zeros(1, 2, 16, 64, dtype=BF).expand(9, -1, -1, -1),
                                                                                                                   V=torch.zeros(1, 2, 16, 64, dtype=BF).expand(9, -1, -1, -1))),
    (TypeError, dict(table=torch.zeros(3, 5, dtype=torch.int64))), (ValueError, dict(table=i32(5, 3).t())), (ValueError, dict(table=i32(15))), (ValueError, dict(table=i32(1, 5).expand(3, -1))),
    (ValueError, dict(kv_len=i32(2))), (TypeError, dict(kv_len=i32(6)[::2])), (TypeError, dict(kv_len=torch.zeros(3))), (ValueError, dict(q_start=i32(3))),
    (TypeError, dict(q_start=torch.zeros(4, dtype=torch.int64))), (ValueError, dict(q_start=None)), (ValueError, dict(q_start=None, max_new=7)), (ValueError, dict(lse=torch.zeros(27))),
    (TypeError, dict(lse=torch.zeros(28, dtype=BF))), (TypeError, dict(scale="large")), (TypeError, dict(max_new="many")), (TypeError, dict(Q=None)), (ValueError, dict(device=0))]


@pytest.mark.parametrize("error,other", UNFIT)
def test_attention_refuses_tensors_that_do_not_fit(library, error, other):
    with pytest.raises(error):
        library.calls.verify_attention_paged(*attention(**other).values())
    assert not library.made


def test_uniform_tokens_must_lie_evenly_apart(library):
    Q = torch.zeros(3, 4, 4, 64, dtype=BF)[:, :2]
    with pytest.raises(ValueError):
        library.calls.verify_attention_paged(*attention(Q=Q, out=torch.zeros(3, 2, 4, 64, dtype=BF), q_start=None).values())
    one = torch.zeros(3, 4, 4, 64, dtype=BF)[:, :1]   # one token of every branch: any distance
    assert library.calls.verify_attention_paged(*attention(Q=one, out=torch.zeros(3, 1, 4, 64, dtype=BF), q_start=None).values()) == 0
    assert library.made[0][0].q_stride_t == 1024 and library.made[0][0].T == 3


@pytest.mark.parametrize("error,other", [
    (ValueError, dict(Vnew=torch.zeros(6, 2, 64, dtype=BF))), (ValueError, dict(Vnew=torch.zeros(7, 4, 64, dtype=BF)[:, :2])), (TypeError, dict(Vnew=torch.zeros(7, 2, 64))),
    (ValueError, dict(Knew=torch.zeros(7, 3, 64, dtype=BF), Vnew=torch.zeros(7, 3, 64, dtype=BF))), (ValueError, dict(kv_len=i32(2))), (ValueError, dict(q_start=i32(3))),
    (TypeError, dict(table=torch.zeros(3, 5)))])
def test_append_refuses(library, error, other):
    with pytest.raises(error):
        library.calls.kv_append_paged(*append(**other).values())
    assert not library.made


@pytest.mark.parametrize("error,other", [
    (TypeError, dict(refs=torch.zeros(9))), (TypeError, dict(refs=i32(18)[::2])), (ValueError, dict(kv_len=i32(2))), (ValueError, dict(new=i32(2))), (ValueError, dict(copies=i32(2, 2))),
    (TypeError, dict(missing=torch.zeros(1))), (ValueError, dict(missing=i32(0))), (TypeError, dict(page="sixteen"))])
def test_reserve_refuses(library, error, other):
    with pytest.raises(error):
        library.calls.kv_pages_reserve(*reserve(**other).values())
    assert not library.made


def test_the_others_refuse(library):
    t, refs, n = i32(3, 5), i32(9), i32(3)
    bad = [lambda c: c.kv_pages_fork(t, refs, n, i32(2), -1, 0), lambda c: c.kv_pages_fork(t, refs, i32(2), n, -1, 0), lambda c: c.kv_pages_free(t, refs, n, 16, i32(2), -1, 0),
           lambda c: c.kv_pages_compact(t, refs, i32(3, 2), i32(2), None, WS, -1, 0), lambda c: c.kv_pages_compact(t, refs, i32(4, 2), i32(1), None, WS, -1, 0),
           lambda c: c.kv_pages_copy(torch.zeros(3, 4), i32(4, 2), None, -1, 0), lambda c: c.kv_pages_copy(torch.zeros(3, 4, 6, 8)[:, :, :, :4], i32(4, 2), None, -1, 0),
           lambda c: c.kv_pages_copy(torch.zeros(3, 4, 8), i32(8), None, -1, 0), lambda c: c.kv_pages_copy(torch.zeros(1, 4, 8).expand(3, -1, -1), i32(4, 2), None, -1, 0),
           lambda c: c.kv_pages_copy(torch.zeros(3, 4, 8), i32(4, 2), i32(0), -1, 0)]
    for call in bad:
        with pytest.raises(ValueError):
            call(library.calls)
    for call in ("verify_attention_paged", "kv_append_paged", "kv_pages_reserve", "kv_pages_fork", "kv_pages_free", "kv_pages_compact", "kv_pages_copy"):
        with pytest.raises(TypeError):
            getattr(library.calls, call)(1, 2)
    assert not library.made
