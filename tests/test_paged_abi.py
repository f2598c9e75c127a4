"""The paged cache's entry points on the host: geometries and pointers that are refused before anything is launched, and tensors that do not
hold what the kernels would address.  Error paths only: nothing here reaches a launch."""
import ctypes
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ONE = ctypes.c_void_p(4096)   # never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(os.path.join(ROOT, "paper_2505_19634_amd", "liblotts.so")):
        import __graft_entry__
        __graft_entry__.build()
    from paper_2505_19634_amd import binding
    return binding.load()


def desc(**kw):
    from paper_2505_19634_amd.binding import PagedDesc
    d = PagedDesc(16, 64, 4, 40, 8, 128, 64, 1000, 70, 1, 0.0)
    for n, v in kw.items():
        setattr(d, n, v)
    return d


BAD = [dict(B=0), dict(B=4097, T=4097 * 4), dict(T=0), dict(max_new=0), dict(max_new=65), dict(Hq=41), dict(Hkv=0), dict(D=96),
       dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=2048), dict(pages=0), dict(pages=(1 << 24) + 1), dict(columns=0), dict(columns=1 << 24),
       dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_stride_h=124), dict(q_stride_t=4), dict(o_stride_h=64),
       dict(page_stride_t=100), dict(page_stride_t=64), dict(page_stride_p=-8), dict(table_stride=69), dict(T=1 << 20, max_new=1 << 20),
       dict(page_stride_t=1 << 26)]


@pytest.mark.parametrize("kw", BAD)
def test_geometries(lib, kw):
    d = desc(**kw)
    assert lib.verify_attention_paged_workspace_bytes(ctypes.byref(d)) == 0
    assert lib.verify_attention_paged(ctypes.byref(d), *[ONE] * 9, 1 << 40, None) == -2


def test_attention_is_refused(lib):
    d = desc()
    need = lib.verify_attention_paged_workspace_bytes(ctypes.byref(d))
    assert 0 < need < 1 << 30
    assert lib.verify_attention_paged_workspace_bytes(None) == 0
    call = lambda d, *a: lib.verify_attention_paged(None if d is None else ctypes.byref(d), *a, None)
    ok = [ONE] * 7 + [None, ONE, 1 << 40]
    assert call(None, *ok) == -1
    for i in (0, 1, 2, 3, 4, 6, 8):
        a = list(ok)
        a[i] = None
        assert call(d, *a) == -1, i
    assert call(desc(dtype=2), *ok) == -3
    for i in (0, 1, 2, 6, 8):
        a = list(ok)
        a[i] = ctypes.c_void_p(4096 + 8)
        assert call(d, *a) == -2, i
    for i in (3, 4, 5, 7):
        a = list(ok)
        a[i] = ctypes.c_void_p(4096 + 2)
        assert call(d, *a) == -2, i
    a = list(ok)
    a[9] = need - 1
    assert call(d, *a) == -4
    a = list(ok)
    a[5] = None   # without q_start every branch has as many
    assert call(desc(T=63, max_new=4), *a) == -2
    assert call(desc(max_new=5), *a) == -2


def test_append_is_refused(lib):
    names = ("B", "T", "Hkv", "D", "page", "pages", "columns", "dtype", "k", "v", "st", "sh", "kp", "vp", "pp", "ph", "pt", "table", "ts", "len", "q")
    ok = (4, 16, 8, 128, 16, 100, 9, 1, ONE, ONE, 2048, 128, ONE, ONE, 8 * 16 * 128, 16 * 128, 128, ONE, 9, ONE, ONE)
    call = lambda **kw: lib.kv_append_paged(*[kw.get(n, v) for n, v in zip(names, ok)], None)
    for n in ("k", "v", "kp", "vp", "table", "len"):
        assert call(**{n: None}) == -1, n
    assert call(dtype=3) == -3
    for bad in (dict(B=0), dict(B=5000), dict(T=0), dict(Hkv=0), dict(D=4), dict(page=15), dict(page=8), dict(pages=0), dict(columns=0), dict(columns=10),
                dict(st=4), dict(sh=64), dict(pt=120), dict(pp=-16), dict(ts=8), dict(k=ctypes.c_void_p(4104)), dict(vp=ctypes.c_void_p(4104)), dict(T=15, q=None),
                dict(T=(1 << 25) + 4)):
        assert call(**bad) == -2, bad


def test_upkeep_is_refused(lib):
    big = 1 << 40
    assert lib.kv_pages_workspace_bytes(1000) >= 4000 and lib.kv_pages_workspace_bytes(0) == 0 and lib.kv_pages_workspace_bytes((1 << 24) + 1) == 0
    rv = lambda B=4, c=9, p=100, pg=16, t=ONE, ts=9, r=ONE, n=ONE, a=ONE, cp=ONE, m=ONE, w=ONE, wb=big: lib.kv_pages_reserve(B, c, p, pg, t, ts, r, n, a, cp, m, w, wb, None)
    fk = lambda B=4, c=9, p=100, t=ONE, ts=9, r=ONE, n=ONE, a=ONE: lib.kv_pages_fork(B, c, p, t, ts, r, n, a, None)
    fr = lambda B=4, c=9, p=100, pg=16, t=ONE, ts=9, r=ONE, n=ONE, a=ONE: lib.kv_pages_free(B, c, p, pg, t, ts, r, n, a, None)
    cp = lambda B=4, c=9, p=100, t=ONE, ts=9, r=ONE, m=ONE, n=ONE, w=ONE, wb=big: lib.kv_pages_compact(B, c, p, t, ts, r, m, n, w, wb, None)
    for call in (rv, fk, fr, cp):
        for bad in (dict(B=0), dict(B=4097), dict(c=0), dict(c=10), dict(p=0), dict(p=(1 << 24) + 1), dict(t=ctypes.c_void_p(4097)), dict(r=ctypes.c_void_p(4098))):
            assert call(**bad) == -2, bad
        assert call(t=None) == -1 and call(r=None) == -1 and call(n=None) == -1
    assert rv(a=None) == -1 and rv(cp=None) == -1 and rv(m=None) == -1 and rv(w=None) == -1 and fk(a=None) == -1 and cp(m=None) == -1 and cp(w=None) == -1
    assert rv(pg=17) == -2 and fr(pg=8) == -2
    assert rv(wb=399) == -4 and cp(wb=0) == -4
    co = lambda pool=ONE, pl=2, p=10, ps=1 << 20, gs=1 << 16, gb=1 << 16, pr=ONE, n=4: lib.kv_pages_copy(pool, pl, p, ps, gs, gb, pr, n, None, None)
    assert co(pool=None) == -1 and co(pr=None) == -1
    for bad in (dict(pl=0), dict(p=0), dict(n=0), dict(gb=0), dict(gb=24), dict(gs=8), dict(gs=(1 << 16) + 8), dict(ps=-16), dict(ps=8), dict(pool=ctypes.c_void_p(4104))):
        assert co(**bad) == -2, bad
    assert co(n=2 ** 31 - 1, pl=33) == -2   # more pieces than 64 bits might count


def test_binding_refuses_cpu_tensors(lib):
    import paper_2505_19634_amd as lotts
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    kv = torch.zeros(3, 2, 16, 64)
    for call in (lambda: lotts.verify_attention_paged(torch.zeros(2, 4, 64), kv, kv, i(2, 3), i(2), i(3)),
                 lambda: lotts.kv_append_paged(torch.zeros(2, 2, 64), torch.zeros(2, 2, 64), kv, kv, i(2, 3), i(2), i(3)),
                 lambda: lotts.kv_pages_reserve(i(2, 3), i(9), i(2), i(2), 16), lambda: lotts.kv_pages_fork(i(2, 3), i(9), i(2), i(2)),
                 lambda: lotts.kv_pages_free(i(2, 3), i(9), i(2), 16), lambda: lotts.kv_pages_compact(i(2, 3), i(9)),
                 lambda: lotts.kv_pages_copy(torch.zeros(2, 3, 64), i(2, 2))):
        with pytest.raises((ValueError, AssertionError)):
            call()
