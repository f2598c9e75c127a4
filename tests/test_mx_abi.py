"""The microscaled entry points on the host: sizes, pointers and tensors that are refused before anything is launched.  Error paths only."""
import ctypes
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ONE = ctypes.c_void_p(4096)   # never dereferenced


def at(n):
    return ctypes.c_void_p(4096 + n)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(os.path.join(ROOT, "paper_2505_19634_amd", "liblotts.so")):
        import __graft_entry__
        __graft_entry__.build()
    from paper_2505_19634_amd import binding
    return binding.load()


def test_quantise_is_refused(lib):
    q = lambda N=4, K=64, t=1, w=ONE, ld=64, c=ONE, lc=32, s=ONE, ls=2: lib.mxfp4_quantize(N, K, t, w, ld, c, lc, s, ls, None)
    d = lambda N=4, K=64, t=1, w=ONE, ld=64, c=ONE, lc=32, s=ONE, ls=2: lib.mxfp4_dequantize(N, K, t, c, lc, s, ls, w, ld, None)
    for call in (q, d):
        for bad in (dict(w=None), dict(c=None), dict(s=None)):
            assert call(**bad) == -1, bad
        assert call(t=2) == -3
        for bad in (dict(N=0), dict(N=-1), dict(K=0), dict(K=16), dict(K=63), dict(K=33), dict(ld=63), dict(ld=68), dict(lc=31), dict(lc=40), dict(ls=1), dict(w=at(8)), dict(c=at(8)),
                    dict(t=0, ld=66), dict(N=1 << 30, K=64, ld=64), dict(N=2 ** 31 - 1, K=2048, ld=2048, lc=1024, ls=64), dict(ld=-64), dict(ld=1 << 60), dict(lc=1 << 60), dict(ls=1 << 60)):
            assert call(**bad) == -2, bad


def test_product_is_refused(lib):
    need = lib.skinny_gemm_mxfp4_workspace_bytes
    assert need(1, 1, 32) >= 256 and need(0, 8, 64) == 0 and need(257, 8, 64) == 0 and need(4, 0, 64) == 0 and need(4, 8, 48) == 0 and need(4, 8, 0) == 0
    for N, K in ((1003, 1056), (5120, 5120), (55296, 5120), (5120, 27648), (2560, 2048), (64, 28672), (8, 32)):
        sizes = [need(m, N, K) for m in range(1, 257)]
        assert sizes == sorted(sizes), (N, K)   # a workspace for more tokens serves fewer
    g = lambda M=4, N=40, K=64, x=ONE, lx=64, c=ONE, lc=32, s=ONE, ls=2, y=ONE, ly=40, w=ONE, wb=1 << 40: lib.skinny_gemm_mxfp4(M, N, K, x, lx, c, lc, s, ls, y, ly, w, wb, None)
    for bad in (dict(x=None), dict(c=None), dict(s=None), dict(y=None), dict(w=None)):
        assert g(**bad) == -1, bad
    for bad in (dict(M=0), dict(M=257), dict(N=0), dict(K=48), dict(K=-64), dict(lx=63), dict(lx=68), dict(lc=31), dict(lc=40), dict(ls=1), dict(ly=39), dict(x=at(8)), dict(c=at(8)), dict(w=at(8)),
                dict(y=at(1)), dict(N=(1 << 22) + 1, ly=1 << 27), dict(K=(1 << 22) + 32, lx=1 << 23, lc=1 << 22, ls=1 << 18),
                dict(lx=(1 << 22) + 8), dict(lc=(1 << 24) + 16), dict(ls=(1 << 24) + 1), dict(ly=1 << 60)):
        assert g(**bad) == -2, bad
    assert g(wb=need(4, 40, 64) - 1) == -4


def test_append_is_refused(lib):
    names = ("B", "T", "Hkv", "D", "page", "pages", "columns", "dtype", "k", "v", "st", "sh", "kp", "vp", "pp", "ph", "pt", "ks", "vs", "sp", "sch", "sct", "table", "ts", "len", "q")
    ok = (4, 16, 8, 128, 16, 100, 9, 1, ONE, ONE, 2048, 128, ONE, ONE, 8 * 16 * 128, 16 * 128, 128, ONE, ONE, 8 * 16 * 4, 16 * 4, 4, ONE, 9, ONE, ONE)
    call = lambda **kw: lib.kv_append_paged_mxfp8(*[kw.get(n, v) for n, v in zip(names, ok)], None)
    for n in ("k", "v", "kp", "vp", "ks", "vs", "table", "len"):
        assert call(**{n: None}) == -1, n
    assert call(dtype=3) == -3
    for bad in (dict(B=0), dict(B=5000), dict(T=0), dict(Hkv=0), dict(D=16), dict(D=120), dict(page=15), dict(page=8), dict(pages=0), dict(pages=(1 << 24) + 1), dict(columns=0),
                dict(columns=10), dict(st=4), dict(sh=64), dict(sh=120), dict(pt=120), dict(pt=112), dict(pp=-16), dict(ph=8), dict(sct=3), dict(sp=-1), dict(sch=-4), dict(ts=8),
                dict(k=at(8)), dict(vp=at(8)), dict(T=15, q=None), dict(T=(1 << 25) + 4)):
        assert call(**bad) == -2, bad


def desc(scales=(0, 0, 0), **kw):
    from paper_2505_19634_amd.binding import PagedDesc, PagedMxDesc
    d = PagedDesc(16, 64, 4, 40, 8, 128, 64, 1000, 70, 1, 0.0)
    for n, v in kw.items():
        setattr(d, n, v)
    return PagedMxDesc(d, *scales)


BAD = [dict(B=0), dict(B=4097, T=4097 * 4), dict(T=0), dict(max_new=0), dict(max_new=65), dict(Hq=41), dict(Hkv=0), dict(D=96), dict(D=32),
       dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=2048), dict(pages=0), dict(pages=(1 << 24) + 1), dict(columns=0), dict(columns=1 << 24),
       dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_stride_h=124), dict(q_stride_t=4), dict(o_stride_h=64),
       dict(page_stride_t=100), dict(page_stride_t=64), dict(page_stride_t=136), dict(page_stride_p=-16), dict(table_stride=69), dict(T=1 << 20, max_new=1 << 20),
       dict(page_stride_t=1 << 27), dict(scales=(0, 0, 3)), dict(scales=(-1, 0, 0)), dict(scales=(0, -4, 0)), dict(scales=(0, 0, 1 << 27)), dict(scales=(0, 0, 6)), dict(scales=(0, 33, 0)), dict(scales=(66, 0, 0)), dict(scales=(0, 0, 5), D=64)]


@pytest.mark.parametrize("kw", BAD)
def test_geometries(lib, kw):
    d = desc(**kw)
    assert lib.verify_attention_paged_mxfp8_workspace_bytes(ctypes.byref(d)) == 0
    assert lib.verify_attention_paged_mxfp8(ctypes.byref(d), *[ONE] * 11, 1 << 40, None) in (-2, -3)


def test_attention_is_refused(lib):
    d = desc()
    need = lib.verify_attention_paged_mxfp8_workspace_bytes(ctypes.byref(d))
    assert 0 < need < 1 << 30
    assert lib.verify_attention_paged_mxfp8_workspace_bytes(None) == 0
    call = lambda d, *a: lib.verify_attention_paged_mxfp8(None if d is None else ctypes.byref(d), *a, None)
    ok = [ONE] * 9 + [None, ONE, 1 << 40]
    assert call(None, *ok) == -1
    for i in (0, 1, 2, 3, 4, 5, 6, 8, 10):
        a = list(ok)
        a[i] = None
        assert call(d, *a) == -1, i
    assert call(desc(dtype=2), *ok) == -3
    for i in (0, 1, 2, 8, 10):
        a = list(ok)
        a[i] = at(8)
        assert call(d, *a) == -2, i
    for i in (3, 4, 5, 6, 7, 9):
        a = list(ok)
        a[i] = at(2)
        assert call(d, *a) == -2, i
    a = list(ok)
    a[3] = at(1)
    assert call(desc(D=64), *a) == -2
    a = list(ok)
    a[11] = need - 1
    assert call(d, *a) == -4
    a = list(ok)
    a[7] = None   # without q_start every branch has as many
    assert call(desc(T=63, max_new=4), *a) == -2
    assert call(desc(max_new=5), *a) == -2


def test_a_workspace_for_the_largest_call_serves_the_smaller_ones(lib):
    for Hq, Hkv, D in ((16, 2, 128), (40, 8, 128), (32, 8, 64), (5, 1, 64)):
        size = lambda B, n: lib.verify_attention_paged_mxfp8_workspace_bytes(ctypes.byref(desc(B=B, T=B * n, max_new=n, Hq=Hq, Hkv=Hkv, D=D)))
        for n in (1, 2, 4, 9, 20, 70, 300):
            sizes = [size(B, n) for B in (1, 2, 16, 31, 32, 33, 64, 128, 200, 256, 257, 512, 1000)]
            assert sizes == sorted(sizes), (Hq, n)
        for B in (1, 32, 300):
            sizes = [size(B, n) for n in range(1, 80)]
            assert sizes == sorted(sizes), (Hq, B)


def test_binding_refuses_cpu_tensors(lib):
    import paper_2505_19634_amd as lotts
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    u = lambda *s: torch.zeros(s, dtype=torch.uint8)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    for call in (lambda: lotts.mxfp4_quantize(bf(4, 64)), lambda: lotts.mxfp4_dequantize(u(4, 32), u(4, 2)), lambda: lotts.skinny_gemm_mxfp4(bf(2, 64), u(4, 32), u(4, 2)),
                 lambda: lotts.kv_append_paged_mxfp8(bf(2, 2, 64), bf(2, 2, 64), u(3, 2, 16, 64), u(3, 2, 16, 64), u(3, 2, 16, 2), u(3, 2, 16, 2), i(2, 3), i(2), i(3)),
                 lambda: lotts.verify_attention_paged_mxfp8(bf(2, 4, 64), u(3, 2, 16, 64), u(3, 2, 16, 64), u(3, 2, 16, 2), u(3, 2, 16, 2), i(2, 3), i(2), i(3))):
        with pytest.raises((ValueError, AssertionError)):
            call()
