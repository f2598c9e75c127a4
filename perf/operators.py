"""Cases of the paged cache's operators: attention of a chunk of new tokens over pages, the append into pages, and the pages' upkeep.

`listed()` names the cases, `draw()` gives further ones of the same ranges, `prepare()` makes what a program holds before a call, `run()` is
one pass -- through the public entry points where `own` is true, in elementary torch operations where it is not --, `work()` the traffic and
operations that it cannot do without, `exact()` the same outputs in 64 bits.

Kinds:
  attention  verify_attention_paged of one layer: branches with different numbers of new tokens (a prompt's chunk, drafts, one token)
  append     kv_append_paged of one layer
  fork       kv_pages_fork + kv_pages_reserve + kv_pages_copy: a prompt's cache becomes that of many branches, which then take new tokens
  step       kv_pages_reserve + kv_pages_free: the upkeep around one verification step, with the rejected drafts' pages given back
  compact    kv_pages_compact + kv_pages_copy: pages in use move to the front of the pool
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one branch, one new token, a short context: launch and host call are all there is to it
        {"name": "attn_one_token", "kind": "attention", "Hq": 16, "Hkv": 2, "D": 128, "page": 16, "layout": "head", "dtype": "bf16", "lse": False,
         "B": 1, "new": 1, "chunks": 0, "chunk": 0, "shared": 0, "context": 300, "ragged": False},
        # the verification step of the repository's benchmark on pages: 16 branches of a 32B-shaped target forked from one prompt, 3 drafts
        {"name": "attn_32b_b16", "kind": "attention", "Hq": 40, "Hkv": 8, "D": 128, "page": 64, "layout": "head", "dtype": "bf16", "lse": False,
         "B": 16, "new": 4, "chunks": 0, "chunk": 0, "shared": 256, "context": 4096, "ragged": False},
        # the widest branch sweep point, 3B-shaped, branches of different lengths, small pages, tokens in front of heads
        {"name": "attn_3b_b64_ragged", "kind": "attention", "Hq": 16, "Hkv": 2, "D": 128, "page": 16, "layout": "token", "dtype": "bf16", "lse": False,
         "B": 64, "new": 3, "chunks": 0, "chunk": 0, "shared": 1003, "context": 8192, "ragged": True},
        # a whole prompt of odd length, nothing cached before it, 3B-shaped
        {"name": "attn_3b_prompt", "kind": "attention", "Hq": 16, "Hkv": 2, "D": 128, "page": 64, "layout": "head", "dtype": "bf16", "lse": False,
         "B": 1, "new": 0, "chunks": 1, "chunk": 2039, "shared": 0, "context": 2039, "ragged": False},
        # two prompts' chunks behind long cached parts, 32B-shaped: the largest
        {"name": "attn_32b_chunks", "kind": "attention", "Hq": 40, "Hkv": 8, "D": 128, "page": 64, "layout": "head", "dtype": "bf16", "lse": False,
         "B": 2, "new": 0, "chunks": 2, "chunk": 2048, "shared": 0, "context": 10240, "ragged": False},
        # a chunk of a new prompt beside 31 branches in mid generation, heads of 64
        {"name": "attn_mixed_d64", "kind": "attention", "Hq": 32, "Hkv": 8, "D": 64, "page": 32, "layout": "token", "dtype": "bf16", "lse": False,
         "B": 32, "new": 2, "chunks": 1, "chunk": 500, "shared": 0, "context": 4000, "ragged": True},
        # fp32, few short branches, as many KV heads as query heads
        {"name": "attn_f32", "kind": "attention", "Hq": 4, "Hkv": 4, "D": 64, "page": 16, "layout": "head", "dtype": "f32", "lse": True,
         "B": 5, "new": 4, "chunks": 0, "chunk": 0, "shared": 32, "context": 700, "ragged": True},
        # the new tokens of the benchmark's step, and those of a long prompt's chunk beside branches in mid generation
        {"name": "append_32b_b16", "kind": "append", "Hkv": 8, "D": 128, "page": 64, "layout": "head", "dtype": "bf16",
         "B": 16, "new": 4, "chunks": 0, "chunk": 0, "shared": 0, "context": 4096, "ragged": False},
        {"name": "append_chunk", "kind": "append", "Hkv": 8, "D": 128, "page": 16, "layout": "token", "dtype": "bf16",
         "B": 33, "new": 3, "chunks": 2, "chunk": 4001, "shared": 0, "context": 6000, "ragged": True},
        # upkeep of one step of 64 branches with 4 drafts, a pool of every page that a long context takes
        {"name": "step_b64", "kind": "step", "B": 64, "page": 16, "context": 8192, "new": 5, "spare": 0.5},
        # a prompt of odd length becomes 48 branches of a 3B-shaped decoder: its last page is copied for each of them, in every layer
        {"name": "fork_3b_b48", "kind": "fork", "Hkv": 2, "D": 128, "layers": 36, "page": 64, "B": 48, "new": 5, "context": 1003, "dtype": "bf16"},
        # half of the branches have ended: what the others hold goes to the front of an 8-layer pool
        {"name": "compact_b32", "kind": "compact", "Hkv": 8, "D": 128, "layers": 8, "page": 16, "B": 32, "context": 512, "dtype": "bf16"},
    ]


HEADS = [(16, 2, 128), (40, 8, 128), (32, 8, 128), (28, 4, 128), (16, 16, 64), (32, 8, 64)]


def _log(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attention"] * 7 + ["append"] * 2 + ["step", "fork", "compact"])
    page, layout = rng.choice([16, 16, 32, 64, 64, 128, 256]), rng.choice(["head", "token"])
    if kind == "attention":
        Hq, Hkv, D = rng.choice(HEADS)
        c = {"kind": kind, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "layout": layout, "dtype": "bf16", "lse": rng.random() < 0.3}
        form = rng.choice(["steps", "steps", "steps", "prompt", "chunks", "chunks", "mixed", "mixed", "f32"])
        B, new, chunks, chunk, shared, context = 1, 0, 1, 0, 0, 0
        if form == "f32":
            H = rng.choice([(4, 4, 64), (8, 2, 64), (4, 2, 128)])
            c.update(dtype="f32", Hq=H[0], Hkv=H[1], D=H[2])
            B, new, chunks, context = rng.randint(1, 8), rng.randint(1, 9), 0, _log(rng, 20, 1500)
        elif form == "steps":
            B, new, chunks, context = _log(rng, 1, 64), rng.randint(1, 9), 0, _log(rng, 100, 32768)
            shared = rng.choice([0, 0, _log(rng, 1, max(2, context // 2))])
        elif form == "prompt":
            B = chunks = _log(rng, 1, 6)
            chunk = context = _log(rng, 17, 4096)
        elif form == "chunks":
            B = chunks = _log(rng, 1, 4)
            chunk = _log(rng, 17, 2048)
            context = chunk + _log(rng, 1, 12000)
        else:
            B, new, chunks, chunk = _log(rng, 3, 48), rng.randint(1, 6), rng.randint(1, 2), _log(rng, 33, 2048)
            context = chunk + _log(rng, 1, 8000)
        c.update(B=B, new=new, chunks=chunks, chunk=chunk, shared=shared, context=context, ragged=rng.random() < 0.6)
        most = work(listed()[4])["flops"]
        while work(c)["flops"] > most or 4 * c["Hkv"] * c["D"] * c["B"] * c["context"] > 700e6:
            if c["B"] > max(2, c["chunks"] + 1):
                c["B"] = max(c["chunks"], c["B"] // 2)
            else:
                c["chunk"], c["context"], c["shared"] = (c["chunk"] + 1) // 2, c["context"] // 2 + c["new"], c["shared"] // 2
        return c
    if kind == "append":
        _, Hkv, D = rng.choice(HEADS)
        chunks = rng.choice([0, 0, 1, 2])
        chunk = _log(rng, 17, 4096) if chunks else 0
        B = max(chunks, _log(rng, 1, 64))
        return {"kind": kind, "Hkv": Hkv, "D": D, "page": page, "layout": layout, "dtype": rng.choice(["bf16", "bf16", "f32"]), "B": B,
                "new": rng.randint(1, 9), "chunks": chunks, "chunk": chunk, "shared": 0, "context": chunk + _log(rng, 10, 2000 if B > 8 else 8000),
                "ragged": rng.random() < 0.6}
    if kind == "step":
        return {"kind": kind, "B": _log(rng, 1, 256), "page": page, "context": _log(rng, 100, 8192), "new": rng.randint(1, 9), "spare": round(rng.uniform(0.1, 1.0), 2)}
    _, Hkv, D = rng.choice(HEADS)
    layers = _log(rng, 1, 36)
    row = 4 * layers * Hkv * D * page
    if kind == "fork":
        context = _log(rng, 10, 1500)
        B = max(2, min(_log(rng, 2, 64), int(700e6 / row) - context // page - 2))
        while row * (context // page + 2 * B) > 900e6 and row > 2e6:
            layers = max(1, layers // 2)
            row = 4 * layers * Hkv * D * page
        return {"kind": kind, "Hkv": Hkv, "D": D, "layers": layers, "page": page, "B": B, "new": rng.randint(1, 9), "context": context, "dtype": "bf16"}
    B, context = _log(rng, 2, 64), _log(rng, 30, 1500)
    while row * B * (context // page + 1) > 500e6:
        if layers > 1:
            layers //= 2
        elif B > 4:
            B //= 2
        else:
            context //= 2
        row = 4 * layers * Hkv * D * page
    return {"kind": kind, "Hkv": Hkv, "D": D, "layers": layers, "page": page, "B": B, "context": context, "dtype": "bf16"}


# ------------------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _lengths(case):
    """New tokens and all tokens of every branch; a function of the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    new, length = [], []
    for b in range(case["B"]):
        is_chunk = b < case["chunks"]
        n = case["chunk"] if is_chunk else case["new"]
        L = case["context"]
        if case["ragged"]:
            L = rng.randint(max(1, L // 4), L) if b else L
            n = min(n, L)
        new.append(min(n, L))
        length.append(L)
    order = list(range(case["B"]))
    rng.shuffle(order)  # chunks and steps come in any order
    return [new[i] for i in order], [length[i] for i in order]


def _pages(case, length, gen):
    """Page table [B][columns] and its number of pages: whole pages of the shared prompt are the same ones in every branch; the others lie
    anywhere in the pool."""
    page, B = case["page"], case["B"]
    columns = max(-(-L // page) for L in length) + 1
    common = min(case.get("shared", 0), min(length)) // page
    total = common + sum(-(-L // page) - common for L in length)
    ids = torch.randperm(total, generator=gen, device=DEV).to(torch.int32).tolist()
    table, at = [], common
    for L in length:
        own_pages = -(-L // page) - common
        table.append(ids[:common] + ids[at:at + own_pages] + [-1] * (columns - common - own_pages))
        at += own_pages
    return torch.tensor(table, dtype=torch.int32, device=DEV), total


def _cache(case, pages, gen):
    dt = DTYPES[case["dtype"]]
    shape = (pages, case["Hkv"], case["page"], case["D"]) if case["layout"] == "head" else (pages, case["page"], case["Hkv"], case["D"])
    make = lambda: torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16 if dt is torch.bfloat16 else torch.float32)
    K, V = make(), make()
    return (K, V) if case["layout"] == "head" else (K.transpose(1, 2), V.transpose(1, 2))


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    gen, kind = _gen(seed), case["kind"]
    st = {"case": case}
    if kind in ("attention", "append"):
        new, length = _lengths(case)
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        table, pages = _pages(case, length, gen)
        K, V = _cache(case, pages, gen)
        st.update(new=new, length=length, starts=starts, table=table, K=K, V=V, kv_len=_int(length), q_start=_int(starts))
        dt, T = DTYPES[case["dtype"]], starts[-1]
        if kind == "attention":
            st["Q"] = torch.randn((T, case["Hq"], case["D"]), generator=gen, device=DEV, dtype=torch.float32).to(dt)
            st["out"] = torch.empty_like(st["Q"])
            st["lse"] = torch.empty((T, case["Hq"]), dtype=torch.float32, device=DEV) if case["lse"] else None
        else:  # the K and V columns of a projection's output that holds 4 query heads for each KV head too
            H = case["Hkv"]
            qkv = torch.randn((T, 6 * H, case["D"]), generator=gen, device=DEV, dtype=torch.float32).to(dt)
            st["Knew"], st["Vnew"] = qkv[:, 4 * H:5 * H], qkv[:, 5 * H:]
        return st
    B, page = case["B"], case["page"]
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))  # lengths: of the case alone
    if kind == "step":
        length = [rng.randint(max(1, case["context"] // 4), case["context"]) for _ in range(B)]
        table, used = _pages(dict(case, shared=0), length, gen)
        pages = used + int(case["spare"] * used) + 2 * B
        # what is in use lies anywhere among all pages
        where = torch.randperm(pages, generator=gen, device=DEV)[:used].to(torch.int32)
        table = torch.cat([torch.where(table >= 0, where[table.clamp(min=0).long()], table), torch.full((B, 2), -1, dtype=torch.int32, device=DEV)], 1)
        refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
        refs[where.long()] = 1
        st.update(table=table, refs=refs, kv_len=_int(length), start=_int(length), new=torch.full((B,), case["new"], dtype=torch.int32, device=DEV),
                  keep=_int([L + rng.randint(1, case["new"]) for L in length]), copies=torch.empty((B, 2), dtype=torch.int32, device=DEV),
                  missing=torch.empty((1,), dtype=torch.int32, device=DEV))
        return st
    elements = case["Hkv"] * page * case["D"]
    if kind == "fork":
        own_pages = -(-case["context"] // page)
        more = -(-(case["context"] + case["new"]) // page) - case["context"] // page
        pages, columns = own_pages + (B - 1) * more + 3, own_pages + more + 1
        where = torch.randperm(pages, generator=gen, device=DEV)[:own_pages].to(torch.int32)
        table = torch.full((B, columns), -1, dtype=torch.int32, device=DEV)
        table[0, :own_pages] = where
        refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
        refs[where.long()] = 1
        new = torch.full((B,), case["new"], dtype=torch.int32, device=DEV)
        new[0] = 0  # the prompt itself stays as it is
        st.update(table=table, refs=refs, kv_len=_int([case["context"]] + [0] * (B - 1)), new=new, parent=torch.zeros(B, dtype=torch.int32, device=DEV),
                  copies=torch.empty((B, 2), dtype=torch.int32, device=DEV), missing=torch.empty((1,), dtype=torch.int32, device=DEV))
    else:
        length = [rng.randint(max(1, case["context"] // 4), case["context"]) for _ in range(B)]
        table, pages = _pages(dict(case, shared=0), length, gen)
        refs = torch.ones(pages, dtype=torch.int32, device=DEV)
        ended = random.Random(int(seed)).sample(range(B), B // 2)
        for b in ended:
            held = table[b][table[b] >= 0].long()
            refs[held] = 0
            table[b] = -1
        st.update(table=table, refs=refs, moves=torch.empty((pages // 2 + 1, 2), dtype=torch.int32, device=DEV),
                  counts=torch.empty((2,), dtype=torch.int32, device=DEV))
    pool = torch.empty((2 * case["layers"], pages, elements), dtype=torch.bfloat16, device=DEV)
    for plane in pool:
        plane.normal_(generator=gen)
    st["pool"] = pool
    return st


# ------------------------------------------------------------------------------------------------------------------------
def _plain_attention(st):
    case = st["case"]
    Hkv, D, page = case["Hkv"], case["D"], case["page"]
    G = case["Hq"] // Hkv
    out = torch.zeros_like(st["Q"])
    lse = torch.full(st["Q"].shape[:2], -math.inf, dtype=torch.float32, device=DEV)
    for b, (n, L) in enumerate(zip(st["new"], st["length"])):
        ids = st["table"][b, :-(-L // page)].long()
        K = st["K"][ids].permute(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :L].float()
        V = st["V"][ids].permute(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :L].float()
        Kt = K.transpose(1, 2).contiguous()
        rows = max(1, min(n, (1 << 28) // (L * G * Hkv)))
        for i0 in range(0, n, rows):
            i1 = min(n, i0 + rows)
            at = slice(st["starts"][b] + i0, st["starts"][b] + i1)
            q = st["Q"][at].float().view(i1 - i0, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, -1, D)
            s = torch.matmul(q, Kt) * D ** -0.5
            pos = torch.arange(L - n + i0, L - n + i1, device=DEV).repeat_interleave(G)
            s = s.masked_fill(torch.arange(L, device=DEV)[None, :] > pos[:, None], -math.inf)
            m = s.amax(-1, keepdim=True)
            e = torch.exp(s - m)
            z = e.sum(-1, keepdim=True)
            o = torch.matmul(e, V) / z
            out[at] = o.view(Hkv, i1 - i0, G, D).permute(1, 0, 2, 3).reshape(i1 - i0, -1, D).to(out.dtype)
            lse[at] = (m + torch.log(z)).view(Hkv, i1 - i0, G).permute(1, 0, 2).reshape(i1 - i0, -1)
    return {"O": out, "lse": lse} if case["lse"] else {"O": out}


def _plain_append(st):
    page, T = st["case"]["page"], st["starts"][-1]
    tokens = torch.arange(T, device=DEV)
    b = torch.searchsorted(st["q_start"][1:].long().contiguous(), tokens, right=True)
    pos = st["kv_len"].long()[b] - st["q_start"].long()[b + 1] + tokens
    ids = st["table"][b, pos // page].long()
    st["K"][ids, :, pos % page] = st["Knew"]
    st["V"][ids, :, pos % page] = st["Vnew"]
    return {"K": st["K"], "V": st["V"]}


def _entries(table, refs, by):
    """Adds `by` to the references of every page that the table names."""
    held = table.flatten()
    refs.scatter_add_(0, held.clamp(min=0).long(), torch.where(held >= 0, by, 0).to(torch.int32))


def _plain_reserve(table, refs, kv_len, new, page):
    """Lowest free pages, in the order of branches and columns, for what `new` tokens of every branch are written to and is not the branch's
    own; returns the copies and leaves `table`, `refs` and `kv_len` as after the call.  (There is room for all of it.)"""
    B, columns = table.shape
    first, last = kv_len // page, (kv_len + new - 1) // page
    c = torch.arange(columns, device=DEV)[None, :]
    written = (c >= first[:, None]) & (c <= last[:, None]) & (new > 0)[:, None]
    shared = written & (table >= 0) & (refs[table.clamp(min=0).long()] > 1)
    wanted = shared | (written & (table < 0))
    rank = (torch.cumsum(wanted.flatten().int(), 0) - 1).view(B, columns)
    free = torch.argsort((refs > 0).to(torch.int32), stable=True).to(torch.int32)
    fresh = free[rank.clamp(min=0, max=free.numel() - 1).long()]
    kept = shared & (c * page < kv_len[:, None])
    at = first.clamp(max=columns - 1).long()[:, None]
    copy = kept.gather(1, at)
    copies = torch.where(copy, torch.cat([table.gather(1, at), fresh.gather(1, at)], 1), -1)
    _entries(torch.where(shared, table, -1), refs, -1)
    _entries(torch.where(wanted, fresh, -1), refs, 1)
    table.copy_(torch.where(wanted, fresh, table))
    kv_len.add_(new)
    return copies


def _plain_copy(pool, pairs):
    """Copies pages; a pair of -1 stands for no copy (here one of the others once more, or the first page onto itself)."""
    none = pairs[:, :1] < 0
    other = pairs[(~none[:, 0]).int().argmax()].clamp(min=0)
    pairs = torch.where(none, other[None, :], pairs).long()
    pool[:, pairs[:, 1]] = pool[:, pairs[:, 0]]


def _plain_upkeep(st):
    case, kind, table, refs = st["case"], st["case"]["kind"], st["table"], st["refs"]
    if kind == "step":
        st["kv_len"].copy_(st["start"])
        copies = _plain_reserve(table, refs, st["kv_len"], st["new"], case["page"])
        st["kv_len"].copy_(torch.minimum(st["kv_len"], st["keep"]))
        c = torch.arange(table.shape[1], device=DEV)[None, :]
        gone = (c * case["page"] >= st["kv_len"][:, None]) & (table >= 0)
        _entries(torch.where(gone, table, -1), refs, -1)
        table.masked_fill_(gone, -1)
        return {"table": table, "refs": refs, "kv_len": st["kv_len"], "copies": copies}
    if kind == "fork":
        parent = st["parent"].long()
        _entries(table, refs, -1)
        table.copy_(table[parent])
        _entries(table, refs, 1)
        st["kv_len"].copy_(st["kv_len"][parent])
        copies = _plain_reserve(table, refs, st["kv_len"], st["new"], case["page"])
        _plain_copy(st["pool"], copies)
        return {"table": table, "refs": refs, "kv_len": st["kv_len"], "copies": copies, "pool": st["pool"]}
    table, refs = table.clone(), refs.clone()
    used = refs > 0
    live = used.sum()
    ids = torch.arange(refs.numel(), device=DEV)
    movers, holes = used & (ids >= live), ~used & (ids < live)
    n = movers.sum()
    src = torch.argsort((~movers).to(torch.int32), stable=True)  # the pages that move, ascending, and then the others
    dst = torch.argsort((~holes).to(torch.int32), stable=True)
    moves = torch.arange(st["moves"].shape[0], device=DEV) < n
    pairs = torch.where(moves[:, None], torch.stack([src[:moves.numel()], dst[:moves.numel()]], 1), -1).to(torch.int32)
    new_id = ids.clone()
    new_id[src] = torch.where(ids < n, dst, src)
    table.copy_(torch.where(table >= 0, new_id[table.clamp(min=0).long()].to(torch.int32), table))
    moved = torch.zeros_like(refs)
    moved.scatter_add_(0, new_id, torch.where(used, refs, 0))
    _plain_copy(st["pool"], pairs)
    return {"table": table, "refs": moved, "counts": torch.stack([n, live]).to(torch.int32), "pool": st["pool"]}


def run(state):
    case, kind = state["case"], state["case"]["kind"]
    if not own:
        return {"attention": _plain_attention, "append": _plain_append}.get(kind, _plain_upkeep)(state)
    import paper_2505_19634_amd as lotts
    if kind == "attention":
        lotts.verify_attention_paged(state["Q"], state["K"], state["V"], state["table"], state["kv_len"], state["q_start"],
                                     max_new=max(state["new"]), out=state["out"], lse=state["lse"])
        return {"O": state["out"], "lse": state["lse"]} if case["lse"] else {"O": state["out"]}
    if kind == "append":
        lotts.kv_append_paged(state["Knew"], state["Vnew"], state["K"], state["V"], state["table"], state["kv_len"], state["q_start"])
        return {"K": state["K"], "V": state["V"]}
    table, refs = state["table"], state["refs"]
    if kind == "compact":
        table, refs = table.clone(), refs.clone()
        lotts.kv_pages_compact(table, refs, moves=state["moves"], counts=state["counts"])
        lotts.kv_pages_copy(state["pool"], state["moves"], count=state["counts"])
        return {"table": table, "refs": refs, "counts": state["counts"], "pool": state["pool"]}
    kv_len, page = state["kv_len"], case["page"]
    if kind == "step":
        kv_len.copy_(state["start"])
        lotts.kv_pages_reserve(table, refs, kv_len, state["new"], page, copies=state["copies"], missing=state["missing"])
        lotts.kv_pages_free(table, refs, kv_len, page, keep=state["keep"])
        return {"table": table, "refs": refs, "kv_len": kv_len, "copies": state["copies"]}
    lotts.kv_pages_fork(table, refs, kv_len, state["parent"])
    lotts.kv_pages_reserve(table, refs, kv_len, state["new"], page, copies=state["copies"], missing=state["missing"])
    lotts.kv_pages_copy(state["pool"], state["copies"])
    return {"table": table, "refs": refs, "kv_len": kv_len, "copies": state["copies"], "pool": state["pool"]}


def work(case):
    kind, size = case["kind"], 2 if case.get("dtype", "bf16") == "bf16" else 4
    if kind in ("attention", "append"):
        new, length = _lengths(case)
        T, row = sum(new), case["Hkv"] * case["D"] * size
        if kind == "append":
            return {"bytes": 4 * T * row + 4 * (T + 2 * case["B"]), "flops": 0}
        common = min(case["shared"], min(length)) // case["page"] * case["page"]
        visible = sum(n * L - n * (n - 1) // 2 for n, L in zip(new, length))
        return {"bytes": 2 * T * case["Hq"] * case["D"] * size + 2 * row * (common + sum(L - common for L in length)) +
                4 * sum(-(-L // case["page"]) for L in length) + (4 * T * case["Hq"] if case["lse"] else 0),
                "flops": 4 * case["D"] * case["Hq"] * visible}
    B, page = case["B"], case["page"]
    if kind == "step":  # lengths, new tokens, the entries that change hands
        return {"bytes": B * (6 * 4 + 8 + 4 * 4 * (1 + case["new"] // page)), "flops": 0}
    page_bytes = 2 * case["layers"] * case["Hkv"] * case["D"] * page * size
    if kind == "fork":
        copies = B - 1 if case["context"] % page else 0
        return {"bytes": page_bytes * (copies + (1 if copies else 0)) + 4 * B * (-(-case["context"] // page) + 6), "flops": 0}
    mean = 0.625 * case["context"] / page + 0.5  # pages of a branch; half of them have ended, half of what is left lies in the back half
    return {"bytes": int(2 * page_bytes * B * mean / 4 + 8 * B * mean + 8 * B * mean), "flops": 0}


def exact(case, seed):
    """The attention in 64 bits, a KV head at a time; the other kinds move values and whole numbers, and have nothing to compute."""
    if case["kind"] != "attention":
        return None
    if work(case)["flops"] > 2e12:
        return None
    st = prepare(case, seed)
    G, D, page = case["Hq"] // case["Hkv"], case["D"], case["page"]
    O = torch.zeros(st["Q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(st["Q"].shape[:2], dtype=torch.float64, device=DEV)
    for b in range(case["B"]):
        n, L, first = st["new"][b], st["length"][b], st["starts"][b]
        t = torch.arange(L, device=DEV)
        slot = st["table"][b].long()[t // page]
        for h in range(case["Hkv"]):
            k, v = st["K"][slot, h, t % page].double(), st["V"][slot, h, t % page].double()
            for g in range(h * G, h * G + G):
                for i in range(0, n, 1024):
                    q = st["Q"][first + i:first + min(n, i + 1024), g].double()
                    score = (q @ k.T) / math.sqrt(D)
                    last = L - n + i + torch.arange(q.shape[0], device=DEV)
                    score[t[None, :] > last[:, None]] = -math.inf
                    total = torch.logsumexp(score, 1)
                    O[first + i:first + i + q.shape[0], g] = torch.exp(score - total[:, None]) @ v
                    lse[first + i:first + i + q.shape[0], g] = total
    return {"O": O, "lse": lse} if case["lse"] else {"O": O}
