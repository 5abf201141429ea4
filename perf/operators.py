"""The operators around the decode step, as they are measured: logit edits, the 4-bit cache, attention over it, its pages.

Each case is run either in its plain form (elementary torch operations in 32 bits) or, with `own` set, through the
calls of paper_2210_15458_b200.binding.  Both read the same inputs.

Cache format (one layer): uint8 [n_pages, heads, page_size / 16, 18 * D].  A tile of 16 tokens of one head holds, in
this order, the key codes [16 tokens][D / 2], the value codes [D / 16 blocks][16 tokens][8], the key scales
[16 tokens][D / 16] and the value scales [D / 16][16 tokens].  A code is 4 bits (sign, 2 exponent bits, 1 mantissa bit;
the even dimension in the low half of its byte), a scale is 8 bits (e4m3) for 16 neighbouring dimensions of a token.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ESIZE = {"bf16": 2, "f32": 4}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
SIXTH = float(np.float32(1.0) / np.float32(6.0))


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # a handful of chat lanes, every edit on: the smallest call of a decode step
        dict(name="edit-8x32000-bf16", kind="edit", lanes=8, V=32000, dtype="bf16", hist=300, mask=True, bias=True),
        # the vocabulary whose rows start off the 16-byte grid; grammar states and penalties, no bias
        dict(name="edit-256x50257-bf16", kind="edit", lanes=256, V=50257, dtype="bf16", hist=1500, mask=True, bias=False),
        # many lanes of a large vocabulary in 32 bits with long histories
        dict(name="edit-1024x128256-f32", kind="edit", lanes=1024, V=128256, dtype="f32", hist=4096, mask=True, bias=True),
        # one new token for each of 256 lanes, keys and values cut out of a fused projection
        dict(name="store-256x1-bf16", kind="store", lanes=256, T=1, Hq=32, H=8, D=128, P=64, ctx=2000, dtype="bf16"),
        # prompts of up to 4096 tokens, left-padded to one length, stored whole
        dict(name="store-8x4096-bf16", kind="store", lanes=8, T=4096, Hq=32, H=8, D=128, P=64, ctx=4096, dtype="bf16"),
        # few lanes, short contexts, small heads and pages: latency
        dict(name="attend-6x1x437-bf16", kind="attend", lanes=6, T=1, Hq=16, H=4, D=64, P=16, ctx=437, own=0, N=1, dtype="bf16"),
        # a batch of single tokens over ragged contexts, heads that share keys and values four to one
        dict(name="attend-128x1x8192-bf16", kind="attend", lanes=128, T=1, Hq=32, H=8, D=128, P=64, ctx=8192, own=0, N=1, dtype="bf16"),
        # every head with its own keys and values, 32-bit queries, one long and several short contexts
        dict(name="attend-12x1x30001-f32", kind="attend", lanes=12, T=1, Hq=8, H=8, D=128, P=32, ctx=30001, own=0, N=1, dtype="f32"),
        # 8 prompts decoded by 32 codes each: the lanes of a prompt share its pages and have a tail of their own
        dict(name="attend-8x32-shared-bf16", kind="attend", lanes=256, T=1, Hq=32, H=8, D=128, P=64, ctx=6144, own=200, N=32, dtype="bf16"),
        # a chunk of two prompts over what is stored of them already, causal
        dict(name="attend-2x2048x8192-bf16", kind="attend", lanes=2, T=2048, Hq=32, H=8, D=128, P=64, ctx=8192, own=0, N=1, dtype="bf16"),
        # 8 prompts handed to 32 codes each (256 lanes), all layers' part pages copied, then one token more for each lane
        dict(name="fork-8to256", kind="fork", parents=8, lanes=256, P=64, ctx=4000, planes=8, page_bytes=73728, free=300),
        # a pool in which finished lanes left holes, packed to its front
        dict(name="compact-1024", kind="compact", lanes=64, P=64, ctx=1500, planes=8, page_bytes=73728, pages=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("edit", "store", "attend", "attend", "shared", "chunk", "fork", "compact"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    D, P = rng.choice((64, 128)), rng.choice((16, 32, 64, 128))
    H = rng.choice((1, 2, 4, 8))
    g = rng.choice((1, 2, 4, 7, 8))
    if kind == "edit":
        V = _log(rng, 500, 128256)
        lanes = _log(rng, 1, max(1, min(1024, 100000000 // V)))
        return dict(kind="edit", lanes=lanes, V=V, dtype=dtype, hist=_log(rng, 1, 4096), mask=rng.random() < 0.7, bias=rng.random() < 0.5)
    if kind == "store":
        T = _log(rng, 1, 4096)
        lanes = _log(rng, 1, max(1, min(256, 32768 // T)))
        return dict(kind="store", lanes=lanes, T=T, Hq=H * g, H=H, D=D, P=P, ctx=T + _log(rng, 1, 2000), dtype=dtype)
    if kind == "attend":
        ctx = _log(rng, 1, 30000)
        lanes = _log(rng, 1, max(1, min(256, 500000 // ctx)))
        return dict(kind="attend", lanes=lanes, T=rng.choice((1, 1, 1, 2, 5)), Hq=H * g, H=H, D=D, P=P, ctx=ctx, own=0, N=1, dtype=dtype)
    if kind == "shared":
        N = _log(rng, 2, 64)
        S = _log(rng, 1, max(1, 256 // N))
        ctx = _log(rng, 200, 6144)
        return dict(kind="attend", lanes=S * N, T=1, Hq=H * g, H=H, D=D, P=P, ctx=ctx, own=_log(rng, 1, 200), N=N, dtype="bf16")
    if kind == "chunk":
        T = _log(rng, 8, 2048)
        ctx = T + _log(rng, 1, 6000)
        return dict(kind="attend", lanes=rng.choice((1, 2)), T=T, Hq=H * g, H=H, D=D, P=P, ctx=ctx, own=0, N=1, dtype="bf16")
    page_bytes = 16 * _log(rng, 64, 4608)
    if kind == "fork":
        parents = _log(rng, 1, 16)
        return dict(kind="fork", parents=parents, lanes=parents * _log(rng, 1, 16), P=P, ctx=_log(rng, 10, 4000), planes=_log(rng, 1, 8),
                    page_bytes=page_bytes, free=_log(rng, 256, 600))
    return dict(kind="compact", lanes=_log(rng, 2, 64), P=P, ctx=_log(rng, 10, 1500), planes=_log(rng, 1, 8), page_bytes=page_bytes, pages=0)


# ---------------------------------------------------------------------------------------------------------------------
# shapes that follow from a case alone (lengths do not depend on the seed, so that the work does not either)
# ---------------------------------------------------------------------------------------------------------------------
def _spread(case, n, lo, hi):
    """n lengths in [lo, hi], the largest among them."""
    r = random.Random("%s" % sorted((k, v) for k, v in case.items() if k != "name"))
    lens = [r.randint(lo, hi) for _ in range(n)]
    lens[r.randrange(n)] = hi
    return lens


def _history(case):
    lens = _spread(case, case["lanes"], 0, case["hist"])
    return lens, [n // 2 for n in lens]


def _contexts(case):
    """(length of each lane, length of each group's shared beginning)."""
    if case["kind"] == "store":
        return _spread(case, case["lanes"], max(1, case["ctx"] * 3 // 4), case["ctx"]), None
    if case["N"] == 1:
        return _spread(case, case["lanes"], max(1, case["T"], case["ctx"] // 3), case["ctx"]), None
    P, N = case["P"], case["N"]
    shared = [n // P * P for n in _spread(case, case["lanes"] // N, case["ctx"] // 2, case["ctx"])]
    tails = _spread(case, case["lanes"], 1, case["own"])
    return [shared[i // N] + t for i, t in enumerate(tails)], shared


def _forked(case):
    """(lengths of the lanes in hand, parent of each lane to come)."""
    n, m = case["parents"], case["lanes"]
    lens = [x + (x % case["P"] == 0) for x in _spread(case, n, max(1, case["ctx"] // 2), case["ctx"])]
    return lens, [i * n // m for i in range(m)]


def _visible(case):
    """Pairs of a query token and a stored token that it may look at."""
    lens, _ = _contexts(case)
    T = case["T"]
    total = 0
    for n in lens:
        first = max(0, T - n)                       # query tokens before the first stored one see nothing
        total += sum(n - T + 1 + i for i in (first, T - 1)) * (T - first) // 2
    return total


def work(case):
    kind = case["kind"]
    if kind == "edit":
        e = ESIZE[case["dtype"]]
        lens, _ = _history(case)
        words = -(-case["V"] // 32)
        b = 2 * case["lanes"] * case["V"] * e + 4 * sum(lens)
        b += (16 * words * 4 if case["mask"] else 0) + (4 * case["V"] if case["bias"] else 0)
        return {"bytes": b, "flops": 4 * case["lanes"] * case["V"]}
    if kind == "store":
        e, n = ESIZE[case["dtype"]], sum(min(case["T"], x) for x in _contexts(case)[0])
        values = 2 * n * case["H"] * case["D"]
        padded = 2 * case["lanes"] * case["T"] * case["H"] * case["D"]
        return {"bytes": int(values * (e + 2 * 0.5625) + padded * e), "flops": 6 * values}
    if kind == "attend":
        lens, shared = _contexts(case)
        tokens = sum(lens) if shared is None else sum(shared) + sum(n - shared[i // case["N"]] for i, n in enumerate(lens))
        qo = 2 * case["lanes"] * case["T"] * case["Hq"] * case["D"] * ESIZE[case["dtype"]]
        return {"bytes": tokens * case["H"] * case["D"] * 18 // 16 + qo, "flops": 4 * case["D"] * case["Hq"] * _visible(case)}
    if kind == "fork":
        lens, parent = _forked(case)
        M = -(-(case["ctx"] + 2) // case["P"])
        copies = (case["lanes"] - case["parents"]) * case["planes"] * case["page_bytes"]
        pages = sum(-(-n // case["P"]) for n in lens)
        return {"bytes": 2 * copies + 8 * pages + 12 * case["lanes"] * M, "flops": case["lanes"] * M}
    lens, pages, live = _holes(case)
    moved, used = _moves(case)
    return {"bytes": 2 * moved * case["planes"] * case["page_bytes"] + 8 * pages + 8 * used, "flops": pages}


def _holes(case):
    """(lengths of the lanes still alive, size of the pool, which lanes of all are alive)."""
    n = case["lanes"]
    lens = [max(1, x) for x in _spread(case, n, max(1, case["ctx"] // 4), case["ctx"])]
    live = [i % 2 == 0 for i in range(n)]
    need = sum(-(-x // case["P"]) for x in lens)
    pages = max(case["pages"], need + need // 8 + 1)
    return lens, pages, live


def _moves(case):
    lens, pages, live = _holes(case)
    used = sum(-(-x // case["P"]) for x, a in zip(lens, live) if a)
    taken = sorted(p for ps, a in zip(_taken(case), live) if a for p in ps)
    return sum(p >= used for p in taken), used


def _taken(case):
    """The pages of each lane of the pool that is compacted: the lanes grew side by side, page by page."""
    lens, pages, _ = _holes(case)
    r = random.Random("pages %s" % sorted((k, v) for k, v in case.items() if k != "name"))
    order = list(range(pages))
    r.shuffle(order)
    got, at = [], 0
    for x in lens:
        n = -(-x // case["P"])
        got.append(order[at:at + n])
        at += n
    return got


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


def _pack(kc, ks, vc, vs):
    """Codes [n, 16, heads, D] (0..15) and scales [n, 16, heads, D / 16] (bytes) of n tiles as [n, heads, 18 D] bytes."""
    n, _, H, D = kc.shape
    kb = (kc[..., 0::2] | (kc[..., 1::2] << 4)).permute(0, 2, 1, 3).reshape(n, H, 8 * D)
    vb = (vc[..., 0::2] | (vc[..., 1::2] << 4)).view(n, 16, H, D // 16, 8).permute(0, 2, 3, 1, 4).reshape(n, H, 8 * D)
    return torch.cat([kb, vb, ks.permute(0, 2, 1, 3).reshape(n, H, D), vs.permute(0, 2, 3, 1).reshape(n, H, D)], dim=-1)


def _quantise(x):
    """f32 [..., D] as codes (uint8) and the scales' bytes, one for 16 values."""
    b = x.reshape(*x.shape[:-1], -1, 16)
    s8 = (b.abs().amax(-1) * SIXTH).clamp(max=448.0).to(torch.float8_e4m3fn)
    s = s8.float()
    y = b * torch.where(s > 0, s.reciprocal(), torch.zeros_like(s)).unsqueeze(-1)
    a = y.abs()
    code = torch.zeros(a.shape, dtype=torch.uint8, device=x.device)
    for edge, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= edge) if up else (a > edge)       # a value half way goes to the even code
    return (code | (torch.signbit(y).to(torch.uint8) << 3)).view(x.shape), s8.view(torch.uint8)


def _tables(lens, shared, N, P, gen):
    """(table, number of pages): pages in random order, the shared ones of a group in every lane's row of it."""
    M = max(-(-n // P) for n in lens) + 1
    first = [0] * len(lens) if shared is None else [shared[i // N] // P for i in range(len(lens))]
    counts = [-(-n // P) - f for n, f in zip(lens, first)]
    groups = 0 if shared is None else sum(s // P for s in shared)
    n = sum(counts) + groups + 3
    order = torch.randperm(n, device=DEV, generator=gen).to(torch.int32).cpu().numpy()
    table = np.full((len(lens), M), -1, dtype=np.int32)
    at = 0
    if shared is not None:
        for s, length in enumerate(shared):
            table[s * N:(s + 1) * N, :length // P] = order[at:at + length // P]
            at += length // P
    for i, c in enumerate(counts):
        table[i, first[i]:first[i] + c] = order[at:at + c]
        at += c
    return torch.from_numpy(table).to(DEV), n


def prepare(case, seed):
    gen = _gen(seed)
    kind = case["kind"]
    st = {"case": case}
    if kind == "edit":
        L, V = case["lanes"], case["V"]
        rank = torch.randperm(V, device=DEV, generator=gen).float()
        x = torch.randn(L, V, device=DEV, generator=gen) * 3.0 - 1.5 * torch.log(rank + 1)
        x[:, int(rank.argmax())] = float("-inf")
        st["logits"] = x.to(DTYPES[case["dtype"]])
        lens, prompts = _history(case)
        u = torch.rand(L, case["hist"], device=DEV, generator=gen)
        st["seq"] = (u ** 3 * V).to(torch.int32).clamp(max=V - 1)
        st["len"], st["prompt"] = _ints(lens), _ints(prompts)
        st["bias"] = torch.where(torch.rand(V, device=DEV, generator=gen) < 0.01, 5.0, 0.0) if case["bias"] else None
        if case["mask"]:
            # 16 grammar states: from a few allowed tokens to nearly all; a lane is in one of them or in none (-1)
            share = torch.tensor([0.0005 * 2.1 ** k for k in range(11)] + [0.95, 0.97, 0.99, 0.999, 1.0], device=DEV).clamp(max=1.0)
            words = -(-V // 32)
            bits = torch.rand(16, words * 32, device=DEV, generator=gen) < share.unsqueeze(1)
            w = (bits.view(16, words, 32).long() << torch.arange(32, device=DEV)).sum(-1)
            st["mask"] = (w - ((w >> 31) << 32)).to(torch.int32)
            st["state"] = torch.randint(-1, 16, (L,), device=DEV, generator=gen, dtype=torch.int32)
        else:
            st["mask"] = st["state"] = None
        return st
    if kind in ("store", "attend"):
        L, T, Hq, H, D, P = (case[k] for k in ("lanes", "T", "Hq", "H", "D", "P"))
        lens, shared = _contexts(case)
        st["table"], n = _tables(lens, shared, case.get("N", 1), P, gen)
        st["len"] = _ints(lens)
        st["shared"] = None if shared is None else _ints(shared)
        st["k_scale"] = 0.2 + 0.05 * torch.rand(H, device=DEV, generator=gen)
        st["v_scale"] = 0.1 + 0.05 * torch.rand(H, device=DEV, generator=gen)
        wide = torch.exp(0.5 * torch.randn(H, D, device=DEV, generator=gen))        # some dimensions are larger than others
        if kind == "store":
            st["pages"] = torch.zeros(n, H, P // 16, 18 * D, dtype=torch.uint8, device=DEV)
            qkv = torch.randn(L, T, Hq + 2 * H, D, device=DEV, generator=gen)
            qkv[:, :, Hq:Hq + H] *= wide
            qkv = qkv.to(DTYPES[case["dtype"]])
            st["k"], st["v"] = qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
            return st
        tiles = n * P // 16
        k = torch.randn(tiles, 16, H, D, device=DEV, generator=gen) * wide / st["k_scale"].view(H, 1)
        kc, ks = _quantise(k)
        del k
        vc, vs = _quantise(torch.randn(tiles, 16, H, D, device=DEV, generator=gen) / st["v_scale"].view(H, 1))
        st["pages"] = _pack(kc, ks, vc, vs).view(n, P // 16, H, 18 * D).transpose(1, 2).contiguous()
        qkv = torch.randn(L, T, Hq + 2 * H, D, device=DEV, generator=gen).to(DTYPES[case["dtype"]])
        st["q"] = qkv[:, :, :Hq]
        return st
    planes, words = case["planes"], case["page_bytes"] // 4
    if kind == "fork":
        lens, parent = _forked(case)
        P = case["P"]
        used = sum(-(-x // P) for x in lens)
        n = used + case["free"] + case["lanes"]
        M = -(-(case["ctx"] + 2) // P)
        order = torch.randperm(n, device=DEV, generator=gen).to(torch.int32).cpu().numpy()
        table = np.full((case["parents"], M), -1, dtype=np.int32)
        at = 0
        for i, x in enumerate(lens):
            c = -(-x // P)
            table[i, :c] = order[at:at + c]
            at += c
        st["parent"] = _ints(parent)
        st["add"] = torch.ones(case["lanes"], dtype=torch.int32, device=DEV)
        st["table_out"] = torch.empty(case["lanes"], M, dtype=torch.int32, device=DEV)
        st["len_out"] = torch.empty(case["lanes"], dtype=torch.int32, device=DEV)
    else:
        lens, n, live = _holes(case)
        # the lanes' pages lie where the case says, but which lane has which depends on the seed
        P = case["P"]
        M = -(-case["ctx"] // P)
        table = np.full((case["lanes"], M), -1, dtype=np.int32)
        for i, (ps, a) in enumerate(zip(_taken(case), live)):
            if a:
                turn = torch.randperm(len(ps), device=DEV, generator=gen).cpu().numpy()
                table[i, :len(ps)] = np.asarray(ps, dtype=np.int32)[turn]
        lens = [x if a else 0 for x, a in zip(lens, live)]
        st["table_out"] = torch.empty(case["lanes"], M, dtype=torch.int32, device=DEV)
    st["table"], st["len"] = torch.from_numpy(table).to(DEV), _ints(lens)
    ref = np.zeros(n, dtype=np.int32)
    np.add.at(ref, table[table >= 0], 1)
    st["ref"] = torch.from_numpy(ref).to(DEV)
    st["ref_out"] = torch.empty_like(st["ref"])
    st["pool"] = torch.randint(-2**31, 2**31 - 1, (planes, n, words), device=DEV, generator=gen, dtype=torch.int32)
    return st


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------------
REPETITION, PRESENCE, FREQUENCY = 1.3, 0.4, 0.15


def _plain_edit(st):
    x = st["logits"].float()
    L, V = x.shape
    at = torch.arange(st["seq"].shape[1], device=DEV)
    tok = st["seq"].long()
    held = at < st["len"].unsqueeze(1)
    seen = torch.zeros(L, V, device=DEV).scatter_add_(1, tok, held.float()) > 0
    count = torch.zeros(L, V, device=DEV).scatter_add_(1, tok, (held & (at >= st["prompt"].unsqueeze(1))).float())
    x = torch.where(seen, torch.where(x > 0, x / torch.full_like(x, REPETITION), x * REPETITION), x)
    x = x - (FREQUENCY * count + PRESENCE * (count > 0).float())
    if st["bias"] is not None:
        x = x + st["bias"]
    if st["mask"] is not None:
        j = torch.arange(V, device=DEV)
        words = st["mask"][st["state"].clamp(min=0).long()][:, j // 32]
        allowed = ((words >> (j % 32).to(torch.int32)) & 1).bool() | (st["state"] < 0).unsqueeze(1)
        x = torch.where(allowed, x, torch.full_like(x, float("-inf")))
    return x.to(st["logits"].dtype)


def _plain_store(st):
    out = []
    T = st["k"].shape[1]
    real = torch.arange(T, device=DEV) >= (T - st["len"]).unsqueeze(1)
    for x, g in ((st["k"], st["k_scale"]), (st["v"], st["v_scale"])):
        code, s = _quantise(x.float() * g.reciprocal().view(-1, 1))
        y = _values(code) * s.view(torch.float8_e4m3fn).float().repeat_interleave(16, dim=-1) * g.view(-1, 1)
        out.append(torch.where(real.view(*real.shape, 1, 1), y, torch.zeros_like(y)).to(x.dtype))
    return tuple(out)


def _values(code):
    """The numbers that codes 0..15 stand for, f32."""
    m = (code & 7).float()
    v = torch.where(m < 4, m * 0.5, torch.where(m < 6, m - 2, m * 2 - 8))
    return torch.where(code >= 8, -v, v)


def _unpack(tiles, D):
    """bytes [..., 18 D] of tiles as keys and values f32 [..., 16, D]."""
    head = tiles.shape[:-1]
    kb, vb, ks, vs = tiles.split([8 * D, 8 * D, D, D], dim=-1)
    kb = kb.reshape(*head, 16, D // 2)
    vb = vb.reshape(*head, D // 16, 16, 8).transpose(-3, -2).reshape(*head, 16, D // 2)
    ks = ks.view(torch.float8_e4m3fn).float().reshape(*head, 16, D // 16)
    vs = vs.contiguous().view(torch.float8_e4m3fn).float().reshape(*head, D // 16, 16).transpose(-2, -1)
    k = _values(torch.stack([kb & 15, kb >> 4], dim=-1).reshape(*head, 16, D // 16, 16)) * ks.unsqueeze(-1)
    v = _values(torch.stack([vb & 15, vb >> 4], dim=-1).reshape(*head, 16, D // 16, 16)) * vs.unsqueeze(-1)
    return k.reshape(*head, 16, D), v.reshape(*head, 16, D)


def _plain_attend(st):
    q, pages, table = st["q"], st["pages"], st["table"]
    L, T, Hq, D = q.shape
    H, P = pages.shape[1], pages.shape[2] * 16
    n = table.shape[1] * P
    tiles = pages[table.clamp(min=0).long()]                                  # [L, M, H, P / 16, 18 D]
    k, v = (x.reshape(L, -1, H, P, D).transpose(1, 2).reshape(L, H, n, D) for x in _unpack(tiles, D))
    k = k * st["k_scale"].view(1, H, 1, 1)
    v = v * st["v_scale"].view(1, H, 1, 1)
    rows = q.float().view(L, T, H, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(L, H, T * (Hq // H), D)
    s = torch.matmul(rows, k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    limit = st["len"].view(L, 1) - T + 1 + torch.arange(T, device=DEV)        # tokens that query token i sees
    limit = limit.repeat_interleave(Hq // H, dim=1).view(L, 1, T * (Hq // H), 1)
    s = torch.where(torch.arange(n, device=DEV) < limit, s, torch.full_like(s, float("-inf")))
    s = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
    o = torch.matmul(s, v) / s.sum(-1, keepdim=True).clamp(min=1e-38)
    return o.view(L, H, T, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(L, T, Hq, D).to(q.dtype)


def _given(need, ref, most):
    """The lowest-numbered free pages, in the order of the lanes: (page for each piece [lanes, most], which lanes got theirs)."""
    free = torch.argsort((ref != 0).to(torch.int8), stable=True)
    upto = torch.cumsum(need, 0)
    ok = (upto <= (ref == 0).sum()) | (need == 0)
    k = torch.arange(most, device=DEV)
    rank = (upto - need).unsqueeze(1) + k
    want = (k < need.unsqueeze(1)) & ok.unsqueeze(1)
    page = free[rank.clamp(max=ref.numel() - 1)]
    return torch.where(want, page, torch.full_like(page, -1)), ok


def _plain_fork(st):
    P = st["case"]["P"]
    table, lens, ref, parent = st["table"], st["len"].long(), st["ref"], st["parent"].long()
    n, M = table.shape
    L = parent.numel()
    at = torch.arange(M, device=DEV)
    child = torch.zeros(n, dtype=torch.long, device=DEV).scatter_add_(0, parent, torch.ones_like(parent))
    held = at * P < lens.unsqueeze(1)
    part = held & ((at + 1) * P > lens.unsqueeze(1))                           # the partly filled last page
    change = torch.where(part, child.unsqueeze(1).clamp(max=1) - 1, child.unsqueeze(1) - 1) * held
    ref = ref.long().scatter_add(0, table.clamp(min=0).long().view(-1), change.view(-1))
    first = torch.full((n,), L, device=DEV).scatter_reduce_(0, parent, torch.arange(L, device=DEV), "amin")
    copy = (first[parent] != torch.arange(L, device=DEV)) & (lens[parent] % P != 0)
    page, _ = _given(copy.long(), ref, 1)
    out = torch.where(held[parent], table[parent], torch.full_like(table[parent], -1)).long()
    src = out.gather(1, (lens[parent] // P).clamp(max=M - 1).unsqueeze(1)).squeeze(1)[copy]
    dst = page[copy].squeeze(1)
    out = torch.where(part[parent] & copy.unsqueeze(1), page, out)
    ref[dst] = 1
    st["pool"][:, dst] = st["pool"][:, src]
    lens = lens[parent]
    # one token more for each lane
    add = st["add"].long()
    have, need = -(-lens // P), -(-(lens + add) // P) - -(-lens // P)
    page, ok = _given(need, ref, 1)
    new = (at == have.unsqueeze(1)) & (page >= 0)
    out = torch.where(new, page, out)
    ref[page[page >= 0]] = 1
    return {"table": out.int(), "len": torch.where(ok, lens + add, lens).int(), "ref": ref.int(), "pool": st["pool"]}


def _plain_compact(st):
    table, ref = st["table"], st["ref"]
    n = ref.numel()
    at = torch.arange(n, device=DEV)
    used = (ref > 0).sum()
    hole, late = (at < used) & (ref == 0), (at >= used) & (ref > 0)
    src, dst = at[late], at[hole]
    to = at.clone()
    to[src] = dst
    st["pool"][:, dst] = st["pool"][:, src]
    out = torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table)
    ref = ref.clone()
    ref[dst] = ref[src]
    ref[src] = 0
    return {"table": out, "ref": ref, "used": used.int(), "pool": st["pool"]}


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        return {"edit": _plain_edit, "store": _plain_store, "attend": _plain_attend, "fork": _plain_fork, "compact": _plain_compact}[kind](st)
    from paper_2210_15458_b200 import binding as B
    if kind == "edit":
        return B.as_logits_edit(st["logits"], seq=st["seq"], length=st["len"], prompt_length=st["prompt"], repetition=REPETITION,
                                presence=PRESENCE, frequency=FREQUENCY, bias=st["bias"], mask=st["mask"], mask_row=st["state"])
    if kind == "store":
        B.as_cache4_append(st["pages"], st["k"], st["v"], st["table"], st["len"], st["k_scale"], st["v_scale"])
        return B.as_cache4_load(st["pages"], st["table"], st["len"], case["T"], st["k_scale"], st["v_scale"], dtype=st["k"].dtype)
    if kind == "attend":
        return B.as_cache4_attend(st["pages"], st["q"], st["table"], st["len"], 1.0 / math.sqrt(case["D"]), st["k_scale"], st["v_scale"],
                                  N=case["N"], shared=st["shared"])
    if kind == "fork":
        B.as_pages_fork(st["parent"], st["table"], st["len"], st["ref"], case["P"], st["pool"], st["table_out"], st["len_out"], st["ref_out"])
        B.as_pages_grow(st["add"], st["table_out"], st["len_out"], st["ref_out"], case["P"])
        return {"table": st["table_out"], "len": st["len_out"], "ref": st["ref_out"], "pool": st["pool"]}
    used = B.as_pages_compact(st["table"], st["ref"], st["pool"], st["table_out"], st["ref_out"])
    return {"table": st["table_out"], "ref": st["ref_out"], "used": used, "pool": st["pool"]}


# ---------------------------------------------------------------------------------------------------------------------
# the operators' definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    kind = case["kind"]
    if kind in ("fork", "compact"):
        return None                                     # whole numbers only
    st = prepare(case, seed)
    if kind == "edit":
        rows = []
        for i in range(case["lanes"]):
            x = st["logits"][i].double()
            words = st["seq"][i, :int(st["len"][i])].long()
            n = torch.bincount(words[int(st["prompt"][i]):], minlength=case["V"]).double()
            was = torch.bincount(words, minlength=case["V"]) > 0
            x[was & (x > 0)] /= REPETITION
            x[was & (st["logits"][i] <= 0)] *= REPETITION
            x -= FREQUENCY * n
            x[n > 0] -= PRESENCE
            if case["bias"]:
                x += st["bias"].double()
            if case["mask"] and int(st["state"][i]) >= 0:
                w = st["mask"][int(st["state"][i])].cpu().numpy().view(np.uint8)
                x[torch.from_numpy(np.unpackbits(w, bitorder="little")[:case["V"]] == 0).to(DEV)] = -math.inf
            rows.append(x)
        return torch.stack(rows)
    level = torch.tensor(LEVELS, dtype=torch.float64, device=DEV)
    e4m3 = torch.arange(127, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn).double()

    def nearest(x, values):
        """Index of the value nearest to x >= 0; half way: the even one."""
        mid = (values[1:] + values[:-1]) / 2
        low, high = torch.searchsorted(mid, x, right=False), torch.searchsorted(mid, x, right=True)
        return torch.where(low % 2 == 0, low, high)

    if kind == "store":
        out = []
        for x, g in ((st["k"], st["k_scale"]), (st["v"], st["v_scale"])):
            got = torch.zeros(x.shape, dtype=torch.float64, device=DEV)
            for i in range(case["lanes"]):
                y = x[i].double() / g.double().view(-1, 1)
                b = y.reshape(*y.shape[:-1], -1, 16)
                s = e4m3[nearest(b.abs().amax(-1) / 6, e4m3)].unsqueeze(-1)
                z = torch.copysign(level[nearest(torch.where(s > 0, b.abs() / s, 0.0), level)], b) * s
                z = z.reshape(y.shape) * g.double().view(-1, 1)
                z[:max(0, case["T"] - int(st["len"][i]))] = 0
                got[i] = z
            out.append(got)
        return tuple(out)
    L, T, Hq, H, D, P = (case[k] for k in ("lanes", "T", "Hq", "H", "D", "P"))
    sign = torch.cat([level, -level])
    byte = torch.cat([e4m3, torch.zeros(129, dtype=torch.float64, device=DEV)])
    o = torch.zeros(L, T, Hq, D, dtype=torch.float64, device=DEV)
    for i in range(L):
        n = int(st["len"][i])
        raw = st["pages"][st["table"][i, :-(-n // P)].long()].long()            # [pages, H, tiles, 18 D]
        raw = raw.permute(1, 0, 2, 3).reshape(H, -1, 18 * D)
        kb = raw[..., :8 * D].reshape(H, -1, D // 2)
        vb = raw[..., 8 * D:16 * D].reshape(H, -1, D // 16, 16, 8).permute(0, 1, 3, 2, 4).reshape(H, -1, D // 2)
        ks = byte[raw[..., 16 * D:17 * D]].reshape(H, -1, D // 16, 1)
        vs = byte[raw[..., 17 * D:]].reshape(H, -1, D // 16, 16).transpose(-1, -2).reshape(H, -1, D // 16, 1)
        k = sign[torch.stack([kb % 16, kb // 16], -1)].reshape(H, -1, D // 16, 16) * ks
        v = sign[torch.stack([vb % 16, vb // 16], -1)].reshape(H, -1, D // 16, 16) * vs
        k = k.reshape(H, -1, D)[:, :n] * st["k_scale"].double().view(H, 1, 1)
        v = v.reshape(H, -1, D)[:, :n] * st["v_scale"].double().view(H, 1, 1)
        for h in range(Hq):
            s = (st["q"][i, :, h].double() @ k[h // (Hq // H)].T) / math.sqrt(D)
            late = torch.arange(n, device=DEV) > torch.arange(n - T, n, device=DEV).unsqueeze(1)
            o[i, :, h] = torch.softmax(s.masked_fill(late, -math.inf), -1).nan_to_num(0.0) @ v[h // (Hq // H)]
    return o
