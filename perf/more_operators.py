"""Cases of the microscaled operators: a paged cache held in 8 bits, and weights held in 4.

`listed()` names the cases, `draw()` gives further ones of the same ranges, `prepare()` makes what a program holds before a call, `run()` is
one pass -- through the public entry points where `own` is true, in elementary torch operations where it is not --, `work()` the traffic and
operations that it cannot do without, `exact()` the same outputs in 64 bits.

A microscaled block is 32 neighbouring values of a row with one power of two in common, 2^(s - 127) for the scale byte s: the smallest with which no value of
the block lies behind the largest number of the element type.  MXFP8 has elements of 8 bits (e4m3, up to 448), MXFP4 of 4 (e2m1, up to 6).

Kinds:
  attention  verify_attention_paged_mxfp8 of one layer: branches with different numbers of new tokens over an MXFP8 cache
  append     kv_append_paged_mxfp8 of one layer: the new tokens' K and V are quantised as they are written
  gemm       skinny_gemm_mxfp4: new tokens against an MXFP4 weight matrix
  quantise   mxfp4_quantize and mxfp4_dequantize: a weight matrix to MXFP4, and the values that it then stands for
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 32
# Of an element type: how far the largest number's exponent is from the scale's, its fraction bits, and the scale bytes that are used.
E4M3 = {"exponent": 8, "fraction": 0x600000, "lo": 10, "hi": 246, "most": 448.0}
E2M1 = {"exponent": 2, "fraction": 0x400000, "lo": 2, "hi": 252, "most": 6.0}
NAN_SCALE = 255  # of a block with an infinity or a NaN


def listed():
    return [
        # one branch, one new token, a short context: launch and host call are all there is to it
        {"name": "attn_one_token", "kind": "attention", "Hq": 16, "Hkv": 2, "D": 128, "page": 16, "layout": "head", "dtype": "bf16", "lse": False,
         "B": 1, "new": 1, "chunks": 0, "chunk": 0, "shared": 0, "context": 300, "ragged": False},
        # the verification step of the repository's benchmark: 16 branches of a 32B-shaped target forked from one prompt, 3 drafts
        {"name": "attn_32b_b16", "kind": "attention", "Hq": 40, "Hkv": 8, "D": 128, "page": 64, "layout": "head", "dtype": "bf16", "lse": False,
         "B": 16, "new": 4, "chunks": 0, "chunk": 0, "shared": 256, "context": 4096, "ragged": False},
        # a chunk of a new prompt beside 31 branches of different lengths in mid generation, heads of 64, tokens in front of heads
        {"name": "attn_mixed_d64", "kind": "attention", "Hq": 32, "Hkv": 8, "D": 64, "page": 32, "layout": "token", "dtype": "bf16", "lse": True,
         "B": 32, "new": 2, "chunks": 1, "chunk": 500, "shared": 0, "context": 4000, "ragged": True},
        # two prompts' chunks behind long cached parts, 32B-shaped: the largest
        {"name": "attn_32b_chunks", "kind": "attention", "Hq": 40, "Hkv": 8, "D": 128, "page": 64, "layout": "head", "dtype": "bf16", "lse": False,
         "B": 2, "new": 0, "chunks": 2, "chunk": 2048, "shared": 0, "context": 10240, "ragged": False},
        # the new tokens of the benchmark's step, and those of two prompts' chunks beside branches in mid generation
        {"name": "append_32b_b16", "kind": "append", "Hkv": 8, "D": 128, "page": 64, "layout": "head", "dtype": "bf16",
         "B": 16, "new": 4, "chunks": 0, "chunk": 0, "shared": 0, "context": 1000, "ragged": False},
        {"name": "append_chunk", "kind": "append", "Hkv": 8, "D": 128, "page": 16, "layout": "token", "dtype": "bf16",
         "B": 33, "new": 3, "chunks": 2, "chunk": 4001, "shared": 0, "context": 4100, "ragged": True},
        # one token of plain decoding against the QKV projection of a 3B-shaped decoder
        {"name": "gemm_3b_qkv_1", "kind": "gemm", "M": 1, "N": 2560, "K": 2048},
        # the benchmark's 64 new tokens against gate and up, the largest matrix of a 32B-shaped layer
        {"name": "gemm_32b_gate_up_64", "kind": "gemm", "M": 64, "N": 55296, "K": 5120},
        # 64 branches with 3 drafts each against the down projection: the most tokens of a call
        {"name": "gemm_32b_down_256", "kind": "gemm", "M": 256, "N": 5120, "K": 27648},
        # sizes that fit no tile
        {"name": "gemm_odd", "kind": "gemm", "M": 37, "N": 1003, "K": 1056},
        # a layer's weights as they are loaded, and a small fp32 matrix of odd sizes
        {"name": "quantise_32b_gate_up", "kind": "quantise", "N": 55296, "K": 5120, "dtype": "bf16"},
        {"name": "quantise_odd_f32", "kind": "quantise", "N": 1003, "K": 1056, "dtype": "f32"},
    ]


HEADS = [(16, 2, 128), (40, 8, 128), (32, 8, 128), (28, 4, 128), (16, 16, 64), (32, 8, 64)]
MATRICES = [(2560, 2048), (2048, 2048), (22016, 2048), (2048, 11008), (7168, 5120), (5120, 5120), (55296, 5120), (5120, 27648)]
MOST_WEIGHTS = 290_000_000


def _log(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _matrix(rng):
    N, K = _log(rng, 1, 60000), BLOCK * _log(rng, 1, 900)
    while N * K > MOST_WEIGHTS:
        N //= 2
    return N, K


def draw(rng):
    kind = rng.choice(["attention"] * 6 + ["append"] * 2 + ["gemm"] * 6 + ["quantise"] * 2)
    if kind == "gemm":
        N, K = rng.choice(MATRICES) if rng.random() < 0.4 else _matrix(rng)
        return {"kind": kind, "M": _log(rng, 1, 256), "N": N, "K": K}
    if kind == "quantise":
        N, K = _matrix(rng)
        return {"kind": kind, "N": N, "K": K, "dtype": rng.choice(["bf16", "bf16", "f32"])}
    page, layout = rng.choice([16, 16, 32, 64, 64, 128, 256]), rng.choice(["head", "token"])
    if kind == "append":
        _, Hkv, D = rng.choice(HEADS)
        chunks = rng.choice([0, 0, 1, 2])
        chunk = _log(rng, 17, 4096) if chunks else 0
        B = max(chunks, _log(rng, 1, 64))
        return {"kind": kind, "Hkv": Hkv, "D": D, "page": page, "layout": layout, "dtype": rng.choice(["bf16", "bf16", "f32"]), "B": B,
                "new": rng.randint(1, 9), "chunks": chunks, "chunk": chunk, "shared": 0, "context": chunk + _log(rng, 10, 1000 if B > 8 else 4000),
                "ragged": rng.random() < 0.6}
    Hq, Hkv, D = rng.choice(HEADS)
    c = {"kind": kind, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "layout": layout, "dtype": "bf16", "lse": rng.random() < 0.3}
    form = rng.choice(["steps", "steps", "steps", "prompt", "chunks", "chunks", "mixed", "f32"])
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
    most = work(listed()[3])["flops"]
    while work(c)["flops"] > most or 4 * c["Hkv"] * c["D"] * c["B"] * c["context"] > 700e6:
        if c["B"] > max(2, c["chunks"] + 1):
            c["B"] = max(c["chunks"], c["B"] // 2)
        else:
            c["chunk"], c["context"], c["shared"] = (c["chunk"] + 1) // 2, c["context"] // 2 + c["new"], c["shared"] // 2
    return c


# ------------------------------------------------------------------------------------------------------------------------
def _power(byte):
    """2^(byte - 127) of scale bytes 1 to 254, as float32."""
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _scale_bytes(blocks, kind):
    """[..., 32] float32 -> [...] int32."""
    bits = blocks.abs().amax(-1).view(torch.int32)
    byte = (bits >> 23) - kind["exponent"] + ((bits & 0x7fffff) > kind["fraction"]).to(torch.int32)
    return torch.where((bits >> 23) == 255, NAN_SCALE, byte.clamp(kind["lo"], kind["hi"]))


def _to_mxfp8(x):
    """Codes (float8_e4m3fn) of x's shape and scale bytes (uint8), a thirty-second as many."""
    blocks = x.float().unflatten(-1, (-1, BLOCK))
    byte = _scale_bytes(blocks, E4M3)
    nan = (byte == NAN_SCALE)[..., None]
    y = blocks * _power(torch.where(byte == NAN_SCALE, 127, 254 - byte))[..., None]
    codes = torch.where(nan, math.nan, y.clamp(-E4M3["most"], E4M3["most"])).to(torch.float8_e4m3fn)
    return codes.flatten(-2), byte.to(torch.uint8)


def _to_mxfp4(x):
    """The numbers that the codes of x stand for before they are scaled (float32, [..., blocks, 32]) and scale bytes (int32)."""
    blocks = x.float().unflatten(-1, (-1, BLOCK))
    byte = _scale_bytes(blocks, E2M1)
    a = (blocks.abs() * _power(torch.where(byte == NAN_SCALE, 127, 254 - byte))[..., None]).clamp(max=E2M1["most"])
    up = ((a.view(torch.int32) >> 23) - 127).clamp(min=0)  # numbers from 2^up on are 2^(up - 1) apart
    step = _power(up + 126)
    return torch.copysign(torch.round(a / step) * step, blocks), byte


def _fp8_values(codes, scales):
    """Float32 values of an MXFP8 tensor whose scales are a scale type."""
    return codes.float() * scales.float().repeat_interleave(BLOCK, -1)


def _fp4_values(codes, scales):
    """Float32 values of packed MXFP4 rows: the lower half of a byte comes first."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
    c = codes.to(torch.int32)
    pairs = torch.stack([table[c & 15], table[c >> 4]], -1)
    return pairs.flatten(-2) * scales.float().repeat_interleave(BLOCK, -1)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _lengths(case):
    """New tokens and all tokens of every branch; a function of the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    new, length = [], []
    for b in range(case["B"]):
        n = case["chunk"] if b < case["chunks"] else case["new"]
        L = case["context"]
        if case["ragged"]:
            L = rng.randint(max(1, L // 4), L) if b else L
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
    common = min(case["shared"], min(length)) // page
    total = common + sum(-(-L // page) - common for L in length)
    ids = torch.randperm(total, generator=gen, device=DEV).to(torch.int32).tolist()
    table, at = [], common
    for L in length:
        private = -(-L // page) - common
        table.append(ids[:common] + ids[at:at + private] + [-1] * (columns - common - private))
        at += private
    return torch.tensor(table, dtype=torch.int32, device=DEV), total


def _cache(case, pages, gen):
    """Codes and scales of a cache of normal values whose columns have different sizes, as channels of keys have."""
    shape = (pages, case["Hkv"], case["page"], case["D"]) if case["layout"] == "head" else (pages, case["page"], case["Hkv"], case["D"])
    columns = torch.exp(0.7 * torch.randn(case["D"], generator=gen, device=DEV))
    columns *= math.sqrt(case["D"] / float(columns.square().sum()))
    codes, scales = _to_mxfp8(torch.randn(shape, generator=gen, device=DEV) * columns)
    scales = scales.view(torch.float8_e8m0fnu)
    return (codes, scales) if case["layout"] == "head" else (codes.transpose(1, 2), scales.transpose(1, 2))


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    gen, kind = _gen(seed), case["kind"]
    st = {"case": case}
    if kind in ("gemm", "quantise"):
        W = torch.randn((case["N"], case["K"]), generator=gen, device=DEV) * case["K"] ** -0.5
        if kind == "quantise":
            st["W"] = W.to(DTYPES[case["dtype"]])
            return st
        values, byte = _to_mxfp4(W)
        borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEV)  # between the numbers of codes 0 to 7
        code = (torch.bucketize(values.abs(), borders) + 8 * torch.signbit(values).to(torch.int64)).flatten(-2)
        st["codes"] = (code[:, 0::2] | code[:, 1::2] << 4).to(torch.uint8)
        st["scales"] = byte.to(torch.uint8).view(torch.float8_e8m0fnu)
        st["X"] = (torch.randn((case["M"], case["K"]), generator=gen, device=DEV) * 0.5).to(torch.bfloat16)
        st["Y"] = torch.empty((case["M"], case["N"]), dtype=torch.bfloat16, device=DEV)
        return st
    new, length = _lengths(case)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    table, pages = _pages(case, length, gen)
    K, Ks = _cache(case, pages, gen)
    V, Vs = _cache(case, pages, gen)
    st.update(new=new, length=length, starts=starts, table=table, K=K, V=V, Ks=Ks, Vs=Vs, kv_len=_int(length), q_start=_int(starts))
    dt, T = DTYPES[case["dtype"]], starts[-1]
    if kind == "attention":
        st["Q"] = torch.randn((T, case["Hq"], case["D"]), generator=gen, device=DEV).to(dt)
        st["out"] = torch.empty_like(st["Q"])
        st["lse"] = torch.empty((T, case["Hq"]), dtype=torch.float32, device=DEV) if case["lse"] else None
    else:  # the K and V columns of a projection's output that holds 4 query heads for each KV head too
        H = case["Hkv"]
        qkv = torch.randn((T, 6 * H, case["D"]), generator=gen, device=DEV).to(dt)
        st["Knew"], st["Vnew"] = qkv[:, 4 * H:5 * H], qkv[:, 5 * H:]
    return st


# ------------------------------------------------------------------------------------------------------------------------
def _plain_attention(st):
    case = st["case"]
    Hkv, D, page = case["Hkv"], case["D"], case["page"]
    G, new, length = case["Hq"] // Hkv, st["new"], st["length"]
    out = torch.zeros_like(st["Q"])
    lse = torch.full(st["Q"].shape[:2], -math.inf, dtype=torch.float32, device=DEV)
    for n in sorted(set(new)):  # all branches with as many new tokens at once
        if n == 0:
            continue
        which = [b for b, k in enumerate(new) if k == n]
        L = _int([length[b] for b in which])
        first = _int([st["starts"][b] for b in which]).long()
        ids = st["table"][which, :-(-max(length[b] for b in which) // page)].clamp(min=0).long()
        keys = lambda codes, scales: _fp8_values(codes[ids], scales[ids]).permute(0, 2, 1, 3, 4).flatten(2, 3)
        K, V = keys(st["K"], st["Ks"]), keys(st["V"], st["Vs"])
        rows = first[:, None] + torch.arange(n, device=DEV)
        q = st["Q"][rows].float().view(len(which), n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(len(which), Hkv, n * G, D)
        s = torch.matmul(q, K.transpose(2, 3).contiguous()) * D ** -0.5
        last = (L - n)[:, None] + torch.arange(n, device=DEV).repeat_interleave(G)
        s = s.masked_fill(torch.arange(K.shape[2], device=DEV) > last[:, None, :, None], -math.inf)
        m = s.amax(-1, keepdim=True)
        e = torch.exp(s - m)
        z = e.sum(-1, keepdim=True)
        o = torch.matmul(e, V) / z
        token = lambda x: x.view(len(which), Hkv, n, G, -1).permute(0, 2, 1, 3, 4).reshape(len(which), n, case["Hq"], -1)
        out[rows] = token(o).to(out.dtype)
        lse[rows] = token(m + torch.log(z))[..., 0]
    return {"O": out, "lse": lse} if case["lse"] else {"O": out}


def _plain_append(st):
    page, T = st["case"]["page"], st["starts"][-1]
    tokens = torch.arange(T, device=DEV)
    b = torch.searchsorted(st["q_start"][1:].long().contiguous(), tokens, right=True)
    pos = st["kv_len"].long()[b] - st["q_start"].long()[b + 1] + tokens
    ids, at = st["table"][b, pos // page].long(), pos % page
    for new, codes, scales in (("Knew", "K", "Ks"), ("Vnew", "V", "Vs")):
        c, s = _to_mxfp8(st[new])
        st[codes].view(torch.uint8)[ids, :, at] = c.view(torch.uint8)
        st[scales].view(torch.uint8)[ids, :, at] = s
    return {"K": st["K"], "V": st["V"], "Ks": st["Ks"], "Vs": st["Vs"]}


def run(state):
    case, kind = state["case"], state["case"]["kind"]
    if not own:
        if kind == "attention":
            return _plain_attention(state)
        if kind == "append":
            return _plain_append(state)
        if kind == "gemm":
            return {"Y": torch.matmul(state["X"].float(), _fp4_values(state["codes"], state["scales"]).t()).to(torch.bfloat16)}
        values, byte = _to_mxfp4(state["W"])
        scale = torch.where(byte == NAN_SCALE, math.nan, _power(byte.clamp(max=254)))
        return {"values": (values * scale[..., None]).flatten(-2).to(torch.bfloat16)}
    import paper_2505_19634_amd as lotts
    if kind == "attention":
        lotts.verify_attention_paged_mxfp8(state["Q"], state["K"], state["V"], state["Ks"], state["Vs"], state["table"], state["kv_len"],
                                           state["q_start"], max_new=max(state["new"]), out=state["out"], lse=state["lse"])
        return {"O": state["out"], "lse": state["lse"]} if case["lse"] else {"O": state["out"]}
    if kind == "append":
        lotts.kv_append_paged_mxfp8(state["Knew"], state["Vnew"], state["K"], state["V"], state["Ks"], state["Vs"], state["table"],
                                    state["kv_len"], state["q_start"])
        return {"K": state["K"], "V": state["V"], "Ks": state["Ks"], "Vs": state["Vs"]}
    if kind == "gemm":
        return {"Y": lotts.skinny_gemm_mxfp4(state["X"], state["codes"], state["scales"], out=state["Y"])}
    codes, scales = lotts.mxfp4_quantize(state["W"])
    return {"values": lotts.mxfp4_dequantize(codes, scales)}


def work(case):
    kind, size = case["kind"], 2 if case.get("dtype", "bf16") == "bf16" else 4
    if kind == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": N * K // 2 + N * K // BLOCK + 2 * M * (N + K), "flops": 2 * M * N * K}
    if kind == "quantise":
        n = case["N"] * case["K"]
        return {"bytes": n * size + n // 2 + n // BLOCK + 2 * n, "flops": 0}
    new, length = _lengths(case)
    T, values = sum(new), case["Hkv"] * case["D"]
    row = values + values // BLOCK  # a token's K or V in the cache
    if kind == "append":
        return {"bytes": 2 * T * (values * size + row) + 4 * (T + 2 * case["B"]), "flops": 0}
    common = min(case["shared"], min(length)) // case["page"] * case["page"]
    visible = sum(n * L - n * (n - 1) // 2 for n, L in zip(new, length))
    return {"bytes": 2 * T * case["Hq"] * case["D"] * size + 2 * row * (common + sum(L - common for L in length)) +
            4 * sum(-(-L // case["page"]) for L in length) + (4 * T * case["Hq"] if case["lse"] else 0),
            "flops": 4 * case["D"] * case["Hq"] * visible}


# ------------------------------------------------------------------------------------------------------------------------
def _two(k):
    """2^k in 64 bits, of whole numbers k."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _exact_values(x, top, exponent_of_top, digits, lowest, lo, hi):
    """The values of x's blocks in 64 bits from the definition, with the blocks' exponents: the largest element is `top`, in
    [2^exponent_of_top, 2^(exponent_of_top + 1)), elements have `digits` binary places behind the first and none below 2^lowest."""
    b = x.double().unflatten(-1, (-1, BLOCK))
    most = b.abs().amax(-1)
    e = torch.frexp(most)[1] - 1 - exponent_of_top
    e = torch.where(most > top * _two(e), e + 1, e).clamp(lo, hi)
    y = b / _two(e)[..., None]
    place = (torch.frexp(y)[1] - 1).clamp(min=lowest) - digits
    step = _two(place)
    return (torch.round(y / step) * step).clamp(-top, top), e


def exact(case, seed):
    """Attention a KV head at a time, products and codes from their definitions, all in 64 bits."""
    if work(case)["flops"] > 2e12:
        return None
    st = prepare(case, seed)
    if case["kind"] == "quantise":
        code, e = _exact_values(st["W"], 6.0, 2, 1, 0, -125, 125)
        return {"values": (code * _two(e)[..., None]).flatten(-2)}
    if case["kind"] == "gemm":
        rows = []
        for w, s in zip(st["codes"].split(8192), st["scales"].split(8192)):
            c = torch.stack([w & 15, w >> 4], -1).flatten(1).long()
            up, half = (c & 7) >> 1, (c & 1).double()
            value = torch.where(up == 0, half / 2, (1 + half / 2) * _two(up - 1))
            value = torch.where(c >= 8, -value, value).unflatten(1, (-1, BLOCK)) * s.double()[..., None]
            rows.append(st["X"].double() @ value.flatten(1).t())
        return {"Y": torch.cat(rows, 1)}
    D, page = case["D"], case["page"]
    if case["kind"] == "append":
        for b in range(case["B"]):
            first, n, L = st["starts"][b], st["new"][b], st["length"][b]
            t = torch.arange(L - n, L, device=DEV)
            slot = st["table"][b].long()[t // page]
            for new, codes, scales in (("Knew", "K", "Ks"), ("Vnew", "V", "Vs")):
                code, e = _exact_values(st[new][first:first + n], 448.0, 8, 3, -6, -117, 119)
                st[codes].view(torch.uint8)[slot, :, t % page] = code.flatten(-2).float().to(torch.float8_e4m3fn).view(torch.uint8)
                st[scales].view(torch.uint8)[slot, :, t % page] = (e + 127).to(torch.uint8)
        return {k: st[k].double() for k in ("K", "V", "Ks", "Vs")}
    G = case["Hq"] // case["Hkv"]
    O = torch.zeros(st["Q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(st["Q"].shape[:2], dtype=torch.float64, device=DEV)
    for b in range(case["B"]):
        n, L, first = st["new"][b], st["length"][b], st["starts"][b]
        t = torch.arange(L, device=DEV)
        slot = st["table"][b].long()[t // page]
        for h in range(case["Hkv"]):
            k, v = ((st[c][slot, h, t % page].double().unflatten(-1, (-1, BLOCK)) * st[s][slot, h, t % page].double()[..., None]).flatten(-2)
                    for c, s in (("K", "Ks"), ("V", "Vs")))
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
