"""What the tests of the paged cache share: a cache whose every unused place is NaN, attention in 64 bits from its definition with the error
that a correct kernel may make, and the upkeep calls in plain Python."""
import math

import numpy as np
import torch

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}   # torch.finfo(type).eps / 2


class Cache:
    """Pages that lie anywhere in a pool, in the given order in memory; new[b] of branch b's length[b] tokens are new."""

    def __init__(self, new, length, Hq, Hkv, D, page, dtype="bf16", layout="head", spare_pages=3, more_columns=2, holes=(), seed=0, device=DEV,
                 std=1.0):
        g = torch.Generator().manual_seed(seed)
        self.new, self.length, self.Hq, self.Hkv, self.D, self.page, self.dtype = list(new), list(length), Hq, Hkv, D, page, dtype
        B, dt = len(new), DTYPES[dtype]
        columns = max(1, max(-(-L // page) for L in length)) + more_columns
        used = sum(-(-L // page) for L in length)
        pages = used + spare_pages
        order = torch.randperm(pages, generator=g).tolist()
        shape = (pages, Hkv, page, D) if layout == "head" else (pages, page, Hkv, D)
        K = torch.full(shape, math.nan, dtype=dt)
        V = torch.full(shape, math.nan, dtype=dt)
        if layout == "token":
            K, V = K.transpose(1, 2), V.transpose(1, 2)
        table = torch.full((B, columns), -1, dtype=torch.int32)
        self.k, self.v, at = [], [], 0
        for b, L in enumerate(length):
            k, v = ((torch.randn(L, Hkv, D, generator=g) * std).to(dt) for _ in range(2))
            for c in range(-(-L // page)):
                e = order[at]
                at += 1
                table[b, c] = e
                rows = k[c * page:(c + 1) * page].shape[0]
                K[e, :, :rows] = k[c * page:(c + 1) * page].transpose(0, 1)
                V[e, :, :rows] = v[c * page:(c + 1) * page].transpose(0, 1)
            self.k.append(k.double())
            self.v.append(v.double())
        self.gone = {}
        for b, c, entry in holes:   # a page that the branch does not have
            table[b, c] = entry if entry < 0 else pages + entry
            self.gone.setdefault(b, []).append(c)
        self.starts = [0] + np.cumsum(self.new).tolist()
        T = self.starts[-1]
        self.q = (torch.randn(T, Hq, D, generator=g) * std).to(dt)
        self.K, self.V, self.table = (t.to(device) for t in (K, V, table)) if layout == "head" else (
            K.transpose(1, 2).contiguous().to(device).transpose(1, 2), V.transpose(1, 2).contiguous().to(device).transpose(1, 2), table.to(device))
        self.Q = self.q.to(device)
        self.kv_len = torch.tensor(length, dtype=torch.int32, device=device)
        self.q_start = torch.tensor(self.starts, dtype=torch.int32, device=device)

    def reference(self, scale=None):
        """O, lse in 64 bits and how far a kernel may be from each: the weights are rounded to the type (a half step each, relative, so a half
        step of the weighted |V|), scores carry fp32 sums of D products and a product with the scale, the sums over the keys one rounding a
        key, and the output is rounded once."""
        G, u = self.Hq // self.Hkv, 2.0 ** -24
        scale = self.D ** -0.5 if scale is None else scale
        O = torch.zeros(self.q.shape, dtype=torch.float64)
        lse = torch.full(self.q.shape[:2], -math.inf, dtype=torch.float64)
        tol, tol_lse = torch.zeros_like(O), torch.zeros_like(lse)
        for b, (n, L) in enumerate(zip(self.new, self.length)):
            if n == 0 or L == 0:
                continue
            at = slice(self.starts[b], self.starts[b] + n)
            seen = torch.arange(L)[None, :] <= (L - n + torch.arange(n))[:, None]
            for c in self.gone.get(b, ()):
                seen[:, c * self.page:(c + 1) * self.page] = False
            for h in range(self.Hq):
                q, k, v = self.q[at, h].double(), self.k[b][:, h // G], self.v[b][:, h // G]
                s = (q @ k.T * scale).masked_fill(~seen, -math.inf)
                size = (q.abs() @ k.abs().T * scale).masked_fill(~seen, 0.0).amax(1, keepdim=True)
                m = s.amax(1, keepdim=True).clamp(min=-1e300)
                e = torch.exp(s - m)
                z = e.sum(1, keepdim=True)
                w = torch.where(z > 0, e / z.clamp(min=1e-300), torch.zeros_like(e))
                O[at, h] = w @ v
                lse[at, h] = torch.where(z > 0, m + torch.log(z), torch.full_like(m, -math.inf))[:, 0]
                off = 2 * (self.D + 8) * u * size + 2 * (L + 16) * u
                rounded = HALF_STEP[self.dtype] if self.dtype == "bf16" else 0.0
                tol[at, h] = (rounded + off) * (w @ v.abs()) * (1 + 2.0 ** -6) + HALF_STEP[self.dtype] * O[at, h].abs() * (1 + 2.0 ** -6)
                tol_lse[at, h] = (off + 4 * u * (1 + size) + 2 * u * lse[at, h].abs().nan_to_num(0, 0, 0)[:, None])[:, 0]
        return O, lse, tol, tol_lse


def check(cache, out, lse=None, scale=None):
    O, ref_lse, tol, tol_lse = cache.reference(scale)
    got = out.cpu().double().reshape(O.shape)
    assert torch.isfinite(got).all(), "not finite"
    worst = ((got - O).abs() - tol).max().item()
    assert worst <= 0, "off by %g more than the tolerance" % worst
    if lse is not None:
        l = lse.cpu().double().reshape(ref_lse.shape)
        assert torch.equal(torch.isinf(l), torch.isinf(ref_lse)) and (l[torch.isinf(l)] < 0).all()
        fine = ~torch.isinf(l)
        assert ((l - ref_lse).abs() <= tol_lse)[fine].all(), ((l - ref_lse).abs() - tol_lse)[fine].max()


# ---- the upkeep calls in plain Python: lists of lists, changed in place --------------------------------------------------------
def is_page(e, pages):
    return 0 <= e < pages


def reserve(table, refs, kv_len, new, page):
    B, columns, pages = len(table), len(table[0]), len(refs)
    copies = [[-1, -1] for _ in range(B)]
    slots = []
    for b in range(B):
        L, n = max(kv_len[b], 0), max(new[b], 0)
        if n and L + n > columns * page:
            return copies, -1
        if n:
            slots += [(b, c) for c in range(L // page, (L + n - 1) // page + 1)]
    wanted = [(b, c) for b, c in slots if not is_page(table[b][c], pages) or refs[table[b][c]] > 1]
    free = [p for p in range(pages) if refs[p] <= 0]
    if len(free) < len(wanted):
        return copies, len(wanted) - len(free)
    lost = []
    for (b, c), p in zip(wanted, free):
        old = table[b][c]
        if is_page(old, pages):
            lost.append(old)
            if c * page < kv_len[b]:
                copies[b] = [old, p]
        table[b][c] = p
        refs[p] = 1
    for p in lost:
        refs[p] -= 1
    for b in range(B):
        kv_len[b] = max(kv_len[b], 0) + max(new[b], 0)
    return copies, 0


def fork(table, refs, kv_len, parent):
    B, pages = len(table), len(refs)
    old, old_len = [list(r) for r in table], list(kv_len)
    for b, f in enumerate(parent):
        if f == b or f >= B:
            continue
        table[b] = list(old[f]) if f >= 0 else [-1] * len(old[b])
        kv_len[b] = old_len[f] if f >= 0 else 0
        for was, now in zip(old[b], table[b]):
            if was != now:
                if is_page(was, pages):
                    refs[was] -= 1
                if is_page(now, pages):
                    refs[now] += 1


def free(table, refs, kv_len, page, keep=None):
    for b, row in enumerate(table):
        L = max(0, kv_len[b] if keep is None else min(kv_len[b], keep[b]))
        for c in range(-(-L // page), len(row)):
            if is_page(row[c], len(refs)):
                refs[row[c]] -= 1
            row[c] = -1
        kv_len[b] = L


def compact(table, refs):
    pages = len(refs)
    live = sum(r > 0 for r in refs)
    src = [p for p in range(live, pages) if refs[p] > 0]
    dst = [p for p in range(live) if refs[p] <= 0]
    new_id = dict(zip(src, dst))
    for s, d in zip(src, dst):
        refs[d], refs[s] = refs[s], 0
    for row in table:
        for c, e in enumerate(row):
            if is_page(e, pages) and e >= live:
                row[c] = new_id.get(e, -1)
    return [list(m) for m in zip(src, dst)], live
