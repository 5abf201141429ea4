"""The operators of long and of drafted decodes, as they are measured: verification of drafted tokens, attention with a
sliding window, attention weights and eviction by them, pages of lanes that get shorter.

Each case is run either in its plain form (elementary torch operations) or, with `own` set, through the calls of
paper_2210_15458_b200.binding.  Both read the same inputs.

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
ONE_BELOW = 1.0 - 2.0 ** -53
ALIKE = 0.7         # how far draft logits are from the target's: three drafted tokens out of four are accepted
ACCEPTED = 0.75


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # a handful of chat lanes, three drafted tokens each: the smallest call
        dict(name="verify-4x3x32000-bf16", kind="verify", lanes=4, K=3, V=32000, dtype="bf16", temp=1.0, top_k=0, top_p=1.0, drafter=True),
        # 32-bit logits whose rows start off the 16-byte grid, ragged drafts, the nucleus that the decode uses
        dict(name="verify-96x5x50257-f32-nucleus", kind="verify", lanes=96, K=5, V=50257, dtype="f32", temp=0.8, top_k=0, top_p=0.95, drafter=True),
        # many lanes of a large vocabulary
        dict(name="verify-1024x4x128256-bf16", kind="verify", lanes=1024, K=4, V=128256, dtype="bf16", temp=0.8, top_k=0, top_p=1.0, drafter=True),
        # few lanes, short contexts, small heads and pages: latency
        dict(name="window-6x1x437-bf16", kind="window", lanes=6, T=1, Hq=16, H=4, D=64, P=16, ctx=437, window=128, sinks=4, own=0, N=1, dtype="bf16"),
        # a batch of single tokens far behind their beginnings: of up to 30000 tokens each lane sees 4096 and the first 4
        dict(name="window-64x1x30000-bf16", kind="window", lanes=64, T=1, Hq=32, H=8, D=128, P=64, ctx=30000, window=4096, sinks=4, own=0, N=1, dtype="bf16"),
        # a chunk of two prompts over what is stored of them already
        dict(name="window-2x2048x16000-bf16", kind="window", lanes=2, T=2048, Hq=32, H=8, D=128, P=64, ctx=16000, window=4096, sinks=16, own=0, N=1, dtype="bf16"),
        # the weights that one new token of each lane gives to what is stored, added to those of the tokens before it
        dict(name="weigh-64x1x8192-bf16", kind="weigh", lanes=64, T=1, Hq=32, H=8, D=128, P=64, ctx=8192, window=0, sinks=0, add=True, dtype="bf16"),
        # all tokens of the last chunk of two prompts look at the whole of them, before the prompts are cut down
        dict(name="weigh-2x2048x8192-bf16", kind="weigh", lanes=2, T=2048, Hq=32, H=8, D=128, P=64, ctx=8192, window=0, sinks=0, add=False, dtype="bf16"),
        # lanes that are cut back to 2048 tokens whenever they have grown by up to 64
        dict(name="evict-64x2112", kind="evict", lanes=64, H=8, D=128, P=64, ctx=2112, grown=64, keep=2048, first=4, recent=512),
        # prompts of up to 30000 tokens cut down to 4096 before they are handed to their codes
        dict(name="evict-8x30000", kind="evict", lanes=8, H=8, D=128, P=64, ctx=30000, grown=20000, keep=4096, first=4, recent=64),
        # refused drafts leave 1024 lanes
        dict(name="trim-1024x2000", kind="trim", lanes=1024, P=16, ctx=2000, cut=6, window=0),
        # 512 lanes whose windows have moved on, pages behind them given up, a few drafted tokens refused
        dict(name="trim-512x30000-window", kind="trim", lanes=512, P=64, ctx=30000, cut=6, window=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("verify", "verify", "cut", "window", "window", "shared", "chunk", "weigh", "weigh", "evict", "evict", "trim"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    D, P = rng.choice((64, 128)), rng.choice((16, 32, 64, 128))
    H = rng.choice((1, 2, 4, 8))
    g = rng.choice((1, 2, 4, 7, 8))
    if kind in ("verify", "cut"):
        V, K = _log(rng, 500, 128256), rng.randint(1, 8)
        most = 1000000000 // ESIZE[dtype] if kind == "verify" else 100000000
        lanes = _log(rng, 1, max(1, min(1024, most // (V * (2 * K + 1)))))
        top_k = rng.choice((0, _log(rng, 2, 200))) if kind == "cut" else 0
        return dict(kind="verify", lanes=lanes, K=K, V=V, dtype=dtype, temp=rng.choice((0.6, 0.8, 1.0, 1.3)), top_k=top_k,
                    top_p=rng.choice((0.8, 0.9, 0.95)) if kind == "cut" and (top_k == 0 or rng.random() < 0.5) else 1.0, drafter=rng.random() < 0.8)
    if kind in ("window", "shared", "chunk", "weigh"):
        window, sinks = _log(rng, 8, 4096), rng.choice((0, 1, 4, 16, 50, 128))
    if kind == "window":
        T = rng.choice((1, 1, 1, 2, 5))
        ctx = T + _log(rng, 1, 30000) - 1
        lanes = _log(rng, 1, max(1, min(128, 1000000 // ctx)))
        return dict(kind="window", lanes=lanes, T=T, Hq=H * g, H=H, D=D, P=P, ctx=ctx, window=window, sinks=sinks, own=0, N=1, dtype=dtype)
    if kind == "shared":
        N = _log(rng, 2, 64)
        lanes = N * _log(rng, 1, max(1, 128 // N))
        return dict(kind="window", lanes=lanes, T=1, Hq=H * g, H=H, D=D, P=P, ctx=_log(rng, 200, 6144), window=window, sinks=sinks, own=_log(rng, 1, 200), N=N, dtype="bf16")
    if kind == "chunk":
        T = _log(rng, 8, 2048)
        return dict(kind="window", lanes=rng.choice((1, 2)), T=T, Hq=H * min(g, 4), H=H, D=D, P=P, ctx=T + _log(rng, 1, 12000), window=window, sinks=sinks, own=0, N=1, dtype="bf16")
    if kind == "weigh":
        T = rng.choice((1, 1, 2, 32, 64, _log(rng, 8, 2048)))
        ctx = T + _log(rng, 1, 6000)
        lanes = _log(rng, 1, max(1, min(64, 16000000 // (T * ctx))))
        windowed = rng.random() < 0.3
        return dict(kind="weigh", lanes=lanes, T=T, Hq=H * min(g, 4), H=H, D=D, P=P, ctx=ctx, window=window if windowed else 0, sinks=sinks if windowed else 0,
                    add=rng.random() < 0.5, dtype=dtype if T <= 64 else "bf16")
    if kind == "evict":
        keep = _log(rng, 64, 4096)
        ctx = keep + _log(rng, 1, 20000)
        first = rng.choice((0, 4, 16))
        return dict(kind="evict", lanes=_log(rng, 1, max(1, min(64, 240000 // ctx))), H=H, D=D, P=P, ctx=ctx, grown=rng.randint(0, ctx - keep), keep=keep, first=first,
                    recent=_log(rng, 1, keep - first))
    return dict(kind="trim", lanes=_log(rng, 1, 1024), P=P, ctx=_log(rng, 10, 15000), cut=rng.randint(1, 40), window=rng.choice((0, _log(rng, 64, 4096))))


# ---------------------------------------------------------------------------------------------------------------------
# shapes that follow from a case alone (lengths do not depend on the seed, so that the work does not either)
# ---------------------------------------------------------------------------------------------------------------------
def _spread(case, n, lo, hi):
    """n lengths in [lo, hi], the largest among them."""
    r = random.Random("%s" % sorted((k, v) for k, v in case.items() if k != "name"))
    lens = [r.randint(lo, hi) for _ in range(n)]
    lens[r.randrange(n)] = hi
    return lens


def _contexts(case):
    """(length of each lane, length of each group's shared beginning)."""
    if case["kind"] == "evict":
        return _spread(case, case["lanes"], case["ctx"] - case["grown"], case["ctx"]), None
    if case["kind"] == "trim":
        return _spread(case, case["lanes"], max(1, case["ctx"] // 2), case["ctx"]), None
    if case.get("N", 1) == 1:
        return _spread(case, case["lanes"], max(1, case["T"], case["ctx"] // 3), case["ctx"]), None
    P, N = case["P"], case["N"]
    shared = [n // P * P for n in _spread(case, case["lanes"] // N, case["ctx"] // 2, case["ctx"])]
    tails = _spread(case, case["lanes"], 1, case["own"])
    return [shared[i // N] + t for i, t in enumerate(tails)], shared


def _drafts(case):
    return _spread(case, case["lanes"], max(0, case["K"] // 2), case["K"])


def _seen(n, T, window, sinks):
    """(stored tokens that the last T of n tokens look at, pairs of a query token and a token that it looks at)."""
    if not window:
        first = max(0, T - n)
        return n, sum(n - T + 1 + i for i in (first, T - 1)) * (T - first) // 2
    low = max(0, n - T + 1 - window)
    limits = np.arange(max(1, n - T + 1), n + 1)
    pairs = int((np.minimum(limits, window) + np.minimum(sinks, np.maximum(limits - window, 0))).sum())
    return n - low + min(sinks, low), pairs


def work(case):
    kind = case["kind"]
    if kind == "verify":
        # a lane needs the target's rows up to the first refused token, and the draft's rows next to those
        n = _drafts(case)
        rows = sum(sum(ACCEPTED ** i for i in range(m + 1)) + (sum(ACCEPTED ** i for i in range(m)) if case["drafter"] else 0) for m in n)
        b = rows * case["V"] * ESIZE[case["dtype"]] + case["lanes"] * (case["K"] * 12 + 28 + 4 * case["K"] + 4)
        return {"bytes": int(b), "flops": int(4 * rows * case["V"])}
    lens, shared = _contexts(case)
    if kind in ("window", "weigh"):
        T, N = case["T"], case.get("N", 1)
        seen = [_seen(n, T, case["window"], case["sinks"]) for n in lens]
        tokens, pairs = sum(s for s, _ in seen), sum(p for _, p in seen)
        if shared is not None:
            tokens = 0
            for i, n in enumerate(lens):
                low = max(0, n - case["window"])
                b = shared[i // N]
                tokens += n - max(b, low) + max(0, min(case["sinks"], low) - b)
                if i % N == 0:      # once for the group: what its shortest lane's window and the sinks leave of the beginning
                    low = max(0, min(lens[i:i + N]) - case["window"])
                    tokens += max(0, b - low) + min(case["sinks"], low, b)
        rows = case["lanes"] * T * case["Hq"]
        if kind == "window":
            return {"bytes": tokens * case["H"] * case["D"] * 18 // 16 + 2 * rows * case["D"] * ESIZE[case["dtype"]], "flops": 4 * case["D"] * case["Hq"] * pairs}
        b = tokens * case["H"] * (case["D"] * 9 // 16 + (8 if case["add"] else 4)) + rows * (case["D"] * ESIZE[case["dtype"]] + 4)
        return {"bytes": b, "flops": 2 * case["D"] * case["Hq"] * pairs}
    if kind == "evict":
        # weights of the tokens that may go, once; recent tokens move, and some that stay: those behind the new end
        H, read, moved = case["H"], 0, 0
        for n in lens:
            if n > case["keep"]:
                middle, behind = n - case["first"] - case["recent"], n - case["keep"]
                left = case["keep"] - case["first"] - case["recent"]
                read += middle
                moved += case["recent"] + int(min(behind, left) * left / middle)
        return {"bytes": H * (4 * read + 2 * moved * (case["D"] * 18 // 16 + 4) + 4 * sum(lens)), "flops": H * read}
    M = -(-case["ctx"] // case["P"])
    pages = sum(-(-n // case["P"]) for n in lens)
    return {"bytes": 8 * case["lanes"] * M + 16 * case["lanes"] + 8 * pages, "flops": pages}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


def _tiles(n, H, D, k_scale, v_scale, wide, gen):
    """n tiles as bytes [n, H, 18 D]: random keys and values, rounded as the cache stores them."""
    def quantise(x):
        b = x.view(n, 16, H, D // 16, 16)
        s8 = (b.abs().amax(-1) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
        s = s8.float().clamp(min=2.0 ** -9).unsqueeze(-1)
        mid = torch.tensor([(a + b) / 2 for a, b in zip(LEVELS[:-1], LEVELS[1:])], device=DEV)
        code = torch.bucketize((b / s).abs(), mid).to(torch.uint8) | (torch.signbit(b).to(torch.uint8) << 3)
        return code.view(n, 16, H, D), s8.view(torch.uint8)
    kc, ks = quantise(torch.randn(n, 16, H, D, device=DEV, generator=gen) * wide / k_scale.view(H, 1))
    vc, vs = quantise(torch.randn(n, 16, H, D, device=DEV, generator=gen) / v_scale.view(H, 1))
    kb = (kc[..., 0::2] | (kc[..., 1::2] << 4)).permute(0, 2, 1, 3).reshape(n, H, 8 * D)
    vb = (vc[..., 0::2] | (vc[..., 1::2] << 4)).view(n, 16, H, D // 16, 8).permute(0, 2, 3, 1, 4).reshape(n, H, 8 * D)
    return torch.cat([kb, vb, ks.permute(0, 2, 1, 3).reshape(n, H, D), vs.permute(0, 2, 3, 1).reshape(n, H, D)], dim=-1)


def _tables(lens, shared, N, P, gen):
    """(table, number of pages): pages in random order, the shared ones of a group in every lane's row of it."""
    lens = np.asarray(lens)
    begin = np.zeros_like(lens) if shared is None else np.repeat(np.asarray(shared), N) // P
    held = -(-lens // P)
    M = int(held.max()) + 1
    at = np.arange(M)
    groups = 0 if shared is None else int(sum(shared)) // P
    mine = (at >= begin[:, None]) & (at < held[:, None])
    n = int(mine.sum()) + groups + 3
    order = torch.randperm(n, device=DEV, generator=gen).to(torch.int32).cpu().numpy()
    table = np.full((len(lens), M), -1, dtype=np.int32)
    table[mine] = order[groups:groups + int(mine.sum())]
    if shared is not None:
        of_group = at < np.asarray(shared)[:, None] // P
        first = np.full((len(shared), M), -1, dtype=np.int32)
        first[of_group] = order[:groups]
        table = np.where(np.repeat(of_group, N, axis=0), np.repeat(first, N, axis=0), table)
    return torch.from_numpy(np.ascontiguousarray(table)).to(DEV), n


def prepare(case, seed):
    gen = _gen(seed)
    kind = case["kind"]
    st = {"case": case}
    if kind == "verify":
        L, K, V = case["lanes"], case["K"], case["V"]
        dt = DTYPES[case["dtype"]]
        rank = torch.randperm(V, device=DEV, generator=gen).float()
        st["target"] = torch.empty(L, K + 1, V, dtype=dt, device=DEV)
        st["draft"] = torch.empty(L, K, V, dtype=dt, device=DEV) if case["drafter"] else None
        st["drafted"] = torch.empty(L, K, dtype=torch.int32, device=DEV)
        for i in range(K + 1):
            x = torch.randn(L, V, device=DEV, generator=gen) * 3.0 - 1.5 * torch.log(rank + 1)
            st["target"][:, i] = x
            if i < K:
                # what the smaller model thinks, and a token that it draws (of its 20 likeliest where its rows are cut)
                x += ALIKE * torch.randn(L, V, device=DEV, generator=gen)
                if case["drafter"]:
                    st["draft"][:, i] = x
                y, at = torch.topk(x, min(V, 20 if case["top_k"] or case["top_p"] < 1 else 4096), dim=-1)
                noise = -torch.log(-torch.log(torch.rand(y.shape, device=DEV, generator=gen).clamp(1e-9, 1 - 1e-7)))
                st["drafted"][:, i] = at.gather(1, (y / case["temp"] + noise).argmax(-1, keepdim=True)).squeeze(1)
        st["n"] = _ints(_drafts(case))
        st["u"] = torch.rand(L, K, dtype=torch.float64, device=DEV, generator=gen)
        st["codes"] = (torch.arange(L, device=DEV, dtype=torch.float64) + torch.rand(1, dtype=torch.float64, device=DEV, generator=gen)) / L
        return st
    lens, shared = _contexts(case)
    st["table"], n = _tables(lens, shared, case.get("N", 1), case["P"], gen)
    st["len"] = _ints(lens)
    if kind == "trim":
        # a lane keeps all but the last few tokens; with a window, what it can no longer see goes too
        drop = torch.randint(0, case["cut"] + 1, (case["lanes"],), device=DEV, generator=gen, dtype=torch.int32)
        st["keep"] = (st["len"] - drop).clamp(min=0)
        st["gone"] = None
        if case["window"]:
            st["gone"] = torch.stack([torch.full_like(st["len"], 16), (st["keep"] - case["window"]).clamp(min=16)], dim=1)
        used = torch.zeros(n, dtype=torch.int32, device=DEV)
        held = st["table"] >= 0
        used.scatter_add_(0, st["table"][held].long(), torch.ones_like(st["table"][held]))
        st["ref"] = used
        st["out"] = [torch.empty_like(x) for x in (st["table"], st["len"], st["ref"])]
        return st
    H, D, P = case["H"], case["D"], case["P"]
    st["k_scale"] = 0.2 + 0.05 * torch.rand(H, device=DEV, generator=gen)
    st["v_scale"] = 0.1 + 0.05 * torch.rand(H, device=DEV, generator=gen)
    wide = torch.exp(0.5 * torch.randn(H, D, device=DEV, generator=gen))        # some dimensions are larger than others
    all_tiles = n * P // 16
    tiles = _tiles(min(all_tiles, 16384), H, D, st["k_scale"], st["v_scale"], wide, gen)
    which = torch.randint(0, tiles.shape[0], (all_tiles,), device=DEV, generator=gen)
    st["pages"] = tiles[which].view(n, P // 16, H, 18 * D).transpose(1, 2).contiguous()
    del tiles
    L, W = case["lanes"], st["table"].shape[1] * P
    if kind == "evict":
        # sums of attention weights: a few tokens have most of it, some none
        w = torch.exp(2.0 * torch.randn(L, H, W, device=DEV, generator=gen) - 6.0)
        st["weight"] = torch.where(torch.rand(L, H, W, device=DEV, generator=gen) < 0.05, torch.zeros_like(w), w)
        st["weight_out"] = torch.empty_like(w)
        st["keep"] = torch.full_like(st["len"], case["keep"])
        st["first"] = torch.full_like(st["len"], case["first"])
        return st
    T, Hq = case["T"], case["Hq"]
    qkv = torch.randn(L, T, Hq + 2 * H, D, device=DEV, generator=gen).to(DTYPES[case["dtype"]])
    st["q"] = qkv[:, :, :Hq]
    st["shared"] = None if shared is None else _ints(shared)
    if kind == "weigh":
        pos, s, _ = _scores(st, 0)
        st["lse"] = torch.logsumexp(s, -1).view(L, H, T, Hq // H).transpose(1, 2).reshape(L, T, Hq).contiguous()
        w = torch.exp(2.0 * torch.randn(L, H, W, device=DEV, generator=gen) - 3.0)
        st["weight"] = torch.where(torch.arange(W, device=DEV) < st["len"].view(L, 1, 1), w, torch.zeros_like(w))
    return st


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _masses(x, case):
    """Unnormalised probabilities [..., V], 64 bits, of logits under the case's temperature and cuts, and their sums."""
    e = (x.double() - x.amax(-1, keepdim=True).double()).div_(case["temp"]).exp_()
    if case["top_k"] or case["top_p"] < 1:
        order = torch.sort(x, dim=-1, descending=True, stable=True)[1]          # equal logits: the lower index first
        es = e.gather(-1, order)
        if case["top_k"]:
            es[..., case["top_k"]:] = 0
        if case["top_p"] < 1:
            upto = es.cumsum(-1)
            es *= (upto - es) < case["top_p"] * upto[..., -1:]
        e = torch.zeros_like(e).scatter_(-1, order, es)
    return e, e.sum(-1, keepdim=True)


def _plain_verify(st):
    case = st["case"]
    L, K, V = case["lanes"], case["K"], case["V"]
    lane, at = torch.arange(L, device=DEV), torch.arange(K, device=DEV)
    drafted = st["drafted"].long()
    p, zp = _masses(st["target"], case)
    px = (p[:, :K].gather(-1, drafted.unsqueeze(-1)) / zp[:, :K]).squeeze(-1)
    if case["drafter"]:
        q, zq = _masses(st["draft"], case)
        qx = (q.gather(-1, drafted.unsqueeze(-1)) / zq).squeeze(-1)
    else:
        qx = torch.ones_like(px)
    ok = (st["u"] * qx < px) & (at < st["n"].unsqueeze(1))
    a = ok.to(torch.int64).cumprod(1).sum(1)
    r = p[lane, a] / zp[lane, a]
    last = a.clamp(max=K - 1)
    refused = (a < st["n"]).unsqueeze(1)
    if case["drafter"]:
        left = (r - q[lane, last] / zq[lane, last]).clamp(min=0)
    else:
        left = r.scatter(1, drafted[lane, last].unsqueeze(1), 0.0)
    r = torch.where(refused & (left.sum(1, keepdim=True) > 0), left, r)
    upto = r.cumsum(1)
    t = st["codes"].unsqueeze(1) * upto[:, -1:]
    token = ((upto <= t) | (r == 0)).to(torch.int64).cumprod(1).sum(1).clamp(max=V - 1).unsqueeze(1)
    mass = r.gather(1, token)
    code = ((t - (upto.gather(1, token) - mass)) / mass).clamp(0.0, ONE_BELOW).squeeze(1)
    col = torch.arange(K + 1, device=DEV)
    tokens = torch.cat([drafted, token], 1)
    tokens = torch.where(col < a.unsqueeze(1), tokens, torch.where(col == a.unsqueeze(1), token, torch.full_like(tokens, -1)))
    return tokens.int(), a.int(), code


def _values(code):
    """The numbers that codes 0..15 stand for, f32."""
    m = (code & 7).float()
    v = torch.where(m < 4, m * 0.5, torch.where(m < 6, m - 2, m * 2 - 8))
    return torch.where(code >= 8, -v, v)


def _widen(codes, scales, D):
    """Code bytes [..., D / 2] and scale bytes [..., D / 16] as f32 [..., D]."""
    x = _values(torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)).unflatten(-1, (D // 16, 16))
    return (x * scales.contiguous().view(torch.float8_e4m3fn).float().unsqueeze(-1)).flatten(-2)


def _at(st, pos):
    """Where the tokens at pos [L, n] lie: page, tile and place [L, n] (anywhere for positions outside the lane)."""
    P = st["case"]["P"]
    pos = pos.clamp(min=0, max=st["table"].shape[1] * P - 1)
    return st["table"].gather(1, pos // P).clamp(min=0).long(), pos % P // 16, pos % 16


def _keys(st, pos):
    H, D = st["case"]["H"], st["case"]["D"]
    page, tile, t = _at(st, pos)
    codes = st["pages"][..., :8 * D].unflatten(-1, (16, D // 2)).transpose(1, 2)[page, tile, :, t]         # [L, n, H, D / 2]
    scales = st["pages"][..., 16 * D:17 * D].unflatten(-1, (16, D // 16)).transpose(1, 2)[page, tile, :, t]
    return (_widen(codes, scales, D) * st["k_scale"].view(H, 1)).transpose(1, 2)                           # [L, H, n, D]


def _vals(st, pos):
    H, D = st["case"]["H"], st["case"]["D"]
    page, tile, t = _at(st, pos)
    codes = st["pages"][..., 8 * D:16 * D].unflatten(-1, (D // 16, 16, 8)).transpose(1, 2)[page, tile, :, :, t].flatten(-2)
    scales = st["pages"][..., 17 * D:].unflatten(-1, (D // 16, 16)).transpose(1, 2)[page, tile, :, :, t]
    return (_widen(codes, scales, D) * st["v_scale"].view(H, 1)).transpose(1, 2)


def _scores(st, span):
    """(positions [L, n], scores [L, H, T * g, n], -inf where a query token does not look, which positions are real): with a
    window (span > 0) only the first tokens and the last `span`."""
    case, q = st["case"], st["q"]
    L, T, Hq, D = q.shape
    H, window, sinks = case["H"], case["window"], case["sinks"]
    length = st["len"].long().view(L, 1)
    if span:
        late = length - span + torch.arange(span, device=DEV)
        early = torch.arange(sinks, device=DEV).expand(L, sinks)
        pos = torch.cat([torch.where(early < late[:, :1], early, torch.full_like(early, -1)), late], dim=1)
    else:
        pos = torch.arange(st["table"].shape[1] * case["P"], device=DEV).expand(L, -1)
    rows = q.float().view(L, T, H, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(L, H, T * (Hq // H), D)
    s = torch.matmul(rows, _keys(st, pos).transpose(-1, -2)).mul_(1.0 / math.sqrt(D))
    limit = length - T + 1 + torch.arange(T, device=DEV)                       # query token i looks at positions below
    limit = limit.repeat_interleave(Hq // H, dim=1).unsqueeze(2)               # [L, T * g, 1]
    see = (pos >= 0).unsqueeze(1) & (pos.unsqueeze(1) < limit)
    if window:
        see &= (pos.unsqueeze(1) >= limit - window) | (pos.unsqueeze(1) < sinks)
    return pos, s.masked_fill_(~see.unsqueeze(1), float("-inf")), pos >= 0


def _plain_window(st):
    case, q = st["case"], st["q"]
    L, T, Hq, D = q.shape
    H = case["H"]
    pos, s, _ = _scores(st, case["window"] + T - 1)
    s = s.sub_(s.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    o = torch.matmul(s, _vals(st, pos)) / s.sum(-1, keepdim=True).clamp(min=1e-38)
    return o.view(L, H, T, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(L, T, Hq, D).to(q.dtype)


def _plain_weigh(st):
    case = st["case"]
    L, T, Hq, _ = st["q"].shape
    H = case["H"]
    pos, s, _ = _scores(st, 0)
    lse = st["lse"].view(L, T, H, Hq // H).transpose(1, 2).reshape(L, H, T * (Hq // H), 1)
    got = s.sub_(lse).exp_().sum(2)
    length = st["len"].view(L, 1, 1)
    at = pos.unsqueeze(1)
    if case["add"]:
        got = torch.where(at < length - T, st["weight"] + got, got)
    st["weight"].copy_(torch.where(at < length, got, st["weight"]))
    return st["weight"]


def _plain_evict(st):
    case = st["case"]
    H, D, P, R = case["H"], case["D"], case["P"], case["recent"]
    table, w = st["table"], st["weight"]
    L, M = table.shape
    W = M * P
    at = torch.arange(W, device=DEV).view(1, 1, W)
    length, keep, first = (st[k].long().view(L, 1, 1) for k in ("len", "keep", "first"))
    cut = length > keep
    middle = (at >= first) & (at < length - R)
    order = torch.sort(torch.where(middle, w, torch.full_like(w, float("-inf"))), dim=-1, descending=True, stable=True)[1]
    rank = torch.empty_like(order).scatter_(-1, order, at.expand_as(order).contiguous())
    stays = middle & (rank < keep - R - first)
    # the kept tokens behind keep - R go to the places of the others, lowest to lowest; the recent ones follow in their order
    hole = (at >= first) & (at < keep - R) & ~stays
    mover = stays & (at >= keep - R)
    movers = torch.sort((~mover).to(torch.uint8), dim=-1, stable=True)[1]       # positions of the movers, in order, first
    src = torch.where(hole, movers.gather(-1, (hole.long().cumsum(-1) - 1).clamp(min=0)), at)
    src = torch.where((at >= keep - R) & (at < keep), at + length - keep, src)
    src = torch.where(cut, src, at)
    out = torch.where(cut & (at >= keep) & (at < length), torch.zeros_like(w), w.gather(-1, src))
    # a token of a head as bytes [L, H, W, 18 D / 16], gathered, and back into the pages
    tiles = st["pages"][table.clamp(min=0).long()].transpose(1, 2)              # [L, H, M, P / 16, 18 D]
    kb, vb, ks, vs = tiles.split([8 * D, 8 * D, D, D], dim=-1)
    rows = torch.cat([kb.unflatten(-1, (16, D // 2)), vb.unflatten(-1, (D // 16, 16, 8)).transpose(-3, -2).flatten(-2), ks.unflatten(-1, (16, D // 16)),
                      vs.unflatten(-1, (D // 16, 16)).transpose(-2, -1)], dim=-1).reshape(L, H, W, 9 * D // 8)
    rows = rows.gather(2, src.unsqueeze(-1).expand(L, H, W, 9 * D // 8)).view(L, H, M, P // 16, 16, 9 * D // 8)
    kb, vb, ks, vs = rows.split([D // 2, D // 2, D // 16, D // 16], dim=-1)
    tiles = torch.cat([kb.flatten(-2), vb.unflatten(-1, (D // 16, 8)).transpose(-3, -2).flatten(-3), ks.flatten(-2), vs.transpose(-2, -1).flatten(-2)], dim=-1)
    held = table >= 0
    st["pages"][table[held].long()] = tiles.transpose(1, 2)[held]
    return st["pages"], out


def _plain_trim(st):
    P = st["case"]["P"]
    table, length = st["table"], st["len"].long()
    at = torch.arange(table.shape[1], device=DEV) * P
    new = torch.minimum(length, st["keep"].long()).unsqueeze(1)
    held = (table >= 0) & (at < length.unsqueeze(1))
    goes = at >= new
    if st["gone"] is not None:
        goes = goes | ((at >= st["gone"][:, :1]) & (at + P <= torch.minimum(st["gone"][:, 1:].long(), new)))
    drop = (held & goes).to(torch.int32)
    ref = st["ref"].scatter_add(0, table.clamp(min=0).long().view(-1), -drop.view(-1))
    return {"table": torch.where(goes, torch.full_like(table, -1), table), "len": new.squeeze(1).int(), "ref": ref}


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        return {"verify": _plain_verify, "window": _plain_window, "weigh": _plain_weigh, "evict": _plain_evict, "trim": _plain_trim}[kind](st)
    from paper_2210_15458_b200 import binding as B
    if kind == "verify":
        return B.as_step_verify(st["target"], st["draft"], st["drafted"], st["u"], st["codes"], case["temp"], case["top_k"], case["top_p"], n_drafts=st["n"])
    if kind == "window":
        return B.as_cache4_attend(st["pages"], st["q"], st["table"], st["len"], 1.0 / math.sqrt(case["D"]), st["k_scale"], st["v_scale"],
                                  N=case["N"], shared=st["shared"], window=case["window"], sinks=case["sinks"])
    if kind == "weigh":
        B.as_cache4_weigh(st["pages"], st["q"], st["lse"], st["table"], st["len"], 1.0 / math.sqrt(case["D"]), st["weight"], st["k_scale"],
                          window=case["window"] or None, sinks=case["sinks"], add=case["add"])
        return st["weight"]
    if kind == "evict":
        B.as_cache4_evict(st["pages"], st["weight"], st["table"], st["len"], st["keep"], case["recent"], first=st["first"], weight_out=st["weight_out"])
        return st["pages"], st["weight_out"]
    table, length, ref = B.as_pages_trim(st["keep"], st["table"], st["len"], st["ref"], case["P"], gone=st["gone"], table_out=st["out"][0],
                                         length_out=st["out"][1], ref_out=st["out"][2])
    return {"table": table, "len": length, "ref": ref}


# ---------------------------------------------------------------------------------------------------------------------
# the operators' definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    kind = case["kind"]
    if kind in ("evict", "trim"):
        return None                                     # whole numbers and values that only move
    st = prepare(case, seed)
    if kind == "verify":
        return None, None, _exact_codes(case, st)
    L, T, Hq, H, D, P = (case[k] for k in ("lanes", "T", "Hq", "H", "D", "P"))
    level = torch.tensor(LEVELS, dtype=torch.float64, device=DEV)
    sign = torch.cat([level, -level])
    byte = torch.cat([torch.arange(127, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn).double(), torch.zeros(129, dtype=torch.float64, device=DEV)])
    o = torch.zeros(L, T, Hq, D, dtype=torch.float64, device=DEV)
    weight = st["weight"].double() if kind == "weigh" else None
    for i in range(L):
        n = int(st["len"][i])
        raw = st["pages"][st["table"][i, :-(-n // P)].long()].long()            # [pages, H, tiles, 18 D]
        raw = raw.permute(1, 0, 2, 3).reshape(H, -1, 18 * D)
        kb = raw[..., :8 * D].reshape(H, -1, D // 2)
        ks = byte[raw[..., 16 * D:17 * D]].reshape(H, -1, D // 16, 1)
        k = (sign[torch.stack([kb % 16, kb // 16], -1)].reshape(H, -1, D // 16, 16) * ks).reshape(H, -1, D)[:, :n] * st["k_scale"].double().view(H, 1, 1)
        if kind == "window":
            vb = raw[..., 8 * D:16 * D].reshape(H, -1, D // 16, 16, 8).permute(0, 1, 3, 2, 4).reshape(H, -1, D // 2)
            vs = byte[raw[..., 17 * D:]].reshape(H, -1, D // 16, 16).transpose(-1, -2).reshape(H, -1, D // 16, 1)
            v = (sign[torch.stack([vb % 16, vb // 16], -1)].reshape(H, -1, D // 16, 16) * vs).reshape(H, -1, D)[:, :n] * st["v_scale"].double().view(H, 1, 1)
        del raw
        where = torch.arange(n - T, n, device=DEV).unsqueeze(1)                 # the query tokens' own positions
        pos = torch.arange(n, device=DEV)
        hidden = pos > where
        if case["window"]:
            hidden |= (pos <= where - case["window"]) & (pos >= case["sinks"])
        new = pos >= n - T
        if kind == "weigh" and not case["add"]:
            new = torch.ones_like(new)
        if kind == "weigh":
            weight[i, :, :n][:, new] = 0
        for h in range(Hq):
            s = ((st["q"][i, :, h].double() @ k[h // (Hq // H)].T) / math.sqrt(D)).masked_fill(hidden, -math.inf)
            if kind == "window":
                o[i, :, h] = torch.softmax(s, -1).nan_to_num(0.0) @ v[h // (Hq // H)]
            else:
                weight[i, h // (Hq // H), :n] += torch.exp(s - st["lse"][i, :, h].double().unsqueeze(1)).sum(0)
    return o if kind == "window" else weight


def _exact_codes(case, st):
    """The lanes' codes after verification, lane by lane."""
    def probabilities(x):
        e = torch.exp((x.double() - x.double().max()) / case["temp"])
        if case["top_k"] or case["top_p"] < 1:
            keep = torch.argsort(-x.double(), stable=True)[:case["top_k"] or None]
            if case["top_p"] < 1:
                upto = torch.cumsum(e[keep], 0)
                keep = keep[:int((upto < case["top_p"] * upto[-1]).sum()) + 1]
            cut = torch.zeros_like(e)
            cut[keep] = e[keep]
            e = cut
        return e / e.sum()
    codes = st["codes"].clone()
    u, drafted, drafts = st["u"].tolist(), st["drafted"].tolist(), st["n"].tolist()
    for lane, code in enumerate(st["codes"].tolist()):
        rest = None
        for i in range(drafts[lane] + 1):
            p = rest = probabilities(st["target"][lane, i])
            if i == drafts[lane]:
                break
            x = drafted[lane][i]
            if case["drafter"]:
                q = probabilities(st["draft"][lane, i])
            else:
                q = torch.zeros_like(p)
                q[x] = 1.0
            if not u[lane][i] * float(q[x]) < float(p[x]):
                rest = torch.clamp(p - q, min=0.0)
                rest = rest if bool(rest.any()) else p
                break
        upto = torch.cumsum(rest, 0)
        t = code * float(upto[-1])
        token = min(int((upto <= t).sum()), int(rest.nonzero()[-1]))
        below = float(upto[token - 1]) if token else 0.0
        codes[lane] = min(max((t - below) / float(rest[token]), 0.0), ONE_BELOW)
    return codes
