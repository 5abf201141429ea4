"""The 4-bit cache and attention over it, against plain implementations: storing bit for bit, attention in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
LEVEL = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float32)
E4M3 = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127], dtype=np.float32)


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import binding
    return binding


def nearest_even(x, values):
    """Index of the value nearest to x >= 0 (x not above the largest value's half step), half way to the even index."""
    mid = (values[1:].astype(np.float64) + values[:-1]) / 2
    low, high = np.searchsorted(mid, x, side="left"), np.searchsorted(mid, x, side="right")
    return np.where(low % 2 == 0, low, high)


def quantise(x, g):
    """float32 [..., D] as (values that are stored, as float32, codes, scale indices): each step rounded to 32 bits."""
    g = np.float32(g)
    y = x.astype(np.float32) * (np.float32(1) / g)
    y = np.where(np.isnan(y), np.float32(0), y)
    b = y.reshape(*y.shape[:-1], -1, 16)
    top = np.abs(b).max(-1) * (np.float32(1) / np.float32(6))
    si = nearest_even(np.minimum(top, np.float32(448)), E4M3)
    s = E4M3[si]
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        rs = np.where(s > 0, np.float32(1) / s, np.float32(0)).astype(np.float32)
        z = np.abs(b * rs[..., None])
    code = nearest_even(np.minimum(z, np.float32(6)), LEVEL)
    value = np.copysign(LEVEL[code], b) * s[..., None] * g
    return value.reshape(y.shape).astype(np.float32), code, si


def pool(B, lens, H, D, P, shared=None, N=1, seed=0, spare=2):
    """(pages filled with 0xA5, table on the GPU) for lanes of these lengths; the pages in random order."""
    rng = np.random.default_rng(seed)
    M = max(max(-(-n // P) for n in lens), 1) + 1
    first = [0 if shared is None else shared[i // N] // P for i in range(len(lens))]
    total = sum(max(0, -(-n // P) - f) for n, f in zip(lens, first)) + (0 if shared is None else sum(s // P for s in shared)) + spare
    order = rng.permutation(total).astype(np.int32)
    table = np.full((len(lens), M), -1, dtype=np.int32)
    at = 0
    if shared is not None:
        for g, s in enumerate(shared):
            table[g * N:(g + 1) * N, :s // P] = order[at:at + s // P]
            at += s // P
    for i, n in enumerate(lens):
        c = max(0, -(-n // P) - first[i])
        table[i, first[i]:first[i] + c] = order[at:at + c]
        at += c
    pages = B.cache4_pages(total, H, D, P)
    pages.fill_(0xA5)
    return pages, torch.from_numpy(table).cuda()


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,T,H,P", [([1], 1, 1, 16), ([5, 17, 16, 15], 1, 3, 16), ([40, 33, 2, 0, 64], 33, 2, 32), ([200, 129], 100, 8, 64), ([300], 300, 5, 128)])
def test_store_and_load_bit_for_bit(B, dtype, D, lens, T, H, P):
    lanes = len(lens)
    gen = torch.Generator().manual_seed(D + T)
    fused = (torch.randn(lanes, T, 2 * H + 3, D, generator=gen) * torch.exp(2 * torch.randn(lanes, T, 2 * H + 3, 1, generator=gen))).to(DT[dtype])
    k, v = fused.cuda()[:, :, 3:3 + H], fused.cuda()[:, :, 3 + H:]
    gk, gv = 0.1 + torch.rand(H, generator=gen), 0.1 + torch.rand(H, generator=gen)
    pages, table = pool(B, lens, H, D, P)
    status = torch.full((lanes,), 9, dtype=torch.int32, device="cuda")
    B.as_cache4_append(pages, k, v, table, i32(lens), gk.cuda(), gv.cuda(), lane_status=status)
    assert (status == 0).all()
    gotk, gotv = B.as_cache4_load(pages, table, i32(lens), T, gk.cuda(), gv.cuda(), dtype=torch.float32)
    for got, x, g in ((gotk, k, gk), (gotv, v, gv)):
        want = np.stack([quantise(x[:, :, h].float().cpu().numpy(), g[h])[0] for h in range(H)], axis=2)
        for i, n in enumerate(lens):
            want[i, :max(0, T - n)] = 0
        assert np.array_equal(got.cpu().numpy(), want)
    b16 = B.as_cache4_load(pages, table, i32(lens), T, gk.cuda(), gv.cuda(), dtype=torch.bfloat16)
    assert torch.equal(b16[0], gotk.bfloat16()) and torch.equal(b16[1], gotv.bfloat16())
    # token by token gives the same bytes as all at once, and nothing else is written
    again, _ = pool(B, lens, H, D, P)
    for t in range(T):
        B.as_cache4_append(again, k[:, t:t + 1], v[:, t:t + 1], table, i32([max(0, n - T + 1 + t) for n in lens]), gk.cuda(), gv.cuda())
    assert torch.equal(again, pages)
    held = torch.zeros(pages.shape[0], dtype=torch.bool)
    for i, n in enumerate(lens):
        for p in range(max(0, n - T), n):
            held[int(table[i, p // P])] = True
    assert (pages[~held] == 0xA5).all()


def test_layout_of_a_tile(B):
    """Bytes where the header says, for one token."""
    H, D, P = 2, 64, 32
    k = torch.arange(H * D, dtype=torch.float32).view(1, 1, H, D).cuda() / 7
    v = -k
    pages = B.cache4_pages(2, H, D, P)
    B.as_cache4_append(pages, k, v, i32([[1]]), i32([20]))       # position 19: tile 1, token 3
    raw = pages[1, :, 1].cpu().numpy()
    assert not pages[0].any() and not pages[1, :, 0].any()
    for h in range(H):
        for x, code_at, scale_at, neg in ((k, lambda b: 3 * 32 + b * 8, lambda b: 16 * D + 3 * 4 + b, 0),
                                          (v, lambda b: 8 * D + b * 128 + 3 * 8, lambda b: 17 * D + b * 16 + 3, 8)):
            _, code, si = quantise(x[0, 0, h].cpu().numpy()[None], 1.0)
            for b in range(D // 16):
                assert raw[h, scale_at(b)] == si[0, b]
                got = raw[h, code_at(b):code_at(b) + 8]
                want = [int(c) | (neg if float(x[0, 0, h, 16 * b + e]) < 0 else 0) for e, c in enumerate(code[0, b])]
                lo, hi = [g & 15 for g in got], [g >> 4 for g in got]
                both = [c for pair in zip(lo, hi) for c in pair]
                assert [c & 7 for c in both] == [w & 7 for w in want]
                assert all((c >> 3) == (w >> 3) for c, w in zip(both, want) if w & 7)


def test_half_way_values_zeros_and_non_finite(B):
    D, P = 64, 16
    x = torch.zeros(1, 4, 1, D)
    x[0, 0, 0, :16] = torch.tensor([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, 0.])
    x[0, 1, 0, 16] = 1e-9                                            # below the smallest scale: all zero
    x[0, 2, 0, 32], x[0, 2, 0, 33] = float("inf"), 1.0
    x[0, 3, 0, 5], x[0, 3, 0, 6], x[0, 3, 0, 60] = float("nan"), 2.0, -1e30
    pages = B.cache4_pages(1, 1, D, P)
    status = i32([9])
    B.as_cache4_append(pages, x.cuda(), torch.zeros_like(x).cuda(), i32([[0]]), i32([4]), lane_status=status)
    assert int(status) == B.ERR_NUMERIC
    k, v = B.as_cache4_load(pages, i32([[0]]), i32([4]), 4, dtype=torch.float32)
    assert k[0, 0, 0, :16].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0, -1, -1, -2, -2, -4, -4, 0] and not k[0, 0, 0, 16:].any()
    assert not k[0, 1].any() and not v.any()
    assert k[0, 2, 0, 32] == 2688 and k[0, 2, 0, 33] == 0
    want = quantise(np.array([[0, 2.0] + [0] * 14], dtype=np.float32), 1.0)[0]      # 2 / 6 rounds to 0.34375: 6 of them
    assert want[0, 1] == 2.0625 and k[0, 3, 0, 5] == 0 and k[0, 3, 0, 6] == 2.0625 and k[0, 3, 0, 60] == -2688


def attention(q, k, v, lens, scale):
    """float64 attention of q [lanes, T, Hq, D] over lists of k, v [len, H, D]; (out, lse, bound on a score's size, max |v|)."""
    lanes, T, Hq, D = q.shape
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full((lanes, T, Hq), -math.inf, dtype=torch.float64)
    size = 0.0
    for i in range(lanes):
        g = Hq // k[i].shape[1]
        for t in range(T):
            n = lens[i] - T + 1 + t
            if n <= 0:
                continue
            for h in range(Hq):
                kk, x = k[i][:n, h // g].double(), q[i, t, h].double()
                s = kk @ x * scale
                size = max(size, float((kk.abs() @ x.abs()).max() * abs(scale)))
                lse[i, t, h] = torch.logsumexp(s, 0)
                out[i, t, h] = torch.softmax(s, 0) @ v[i][:n, h // g].double()
    return out, lse, size


def bounds(dtype, size, vmax, out):
    """|error| of the output and of lse.  A score is off by at most 2^-21 of the sum of its terms' magnitudes (operands and
    sums in 24 bits, each operand split exactly or to 2^-23), so a weight by e = 2^-21 size + 2^-20; weights are rounded to
    11 bits for bf16 outputs (2^-11), then the result to 8 (2^-8).  Sum and weighted sum each carry the weight's error."""
    e = 2.0 ** -21 * size + 2.0 ** -20
    w = 2.0 ** -11 if dtype == "bf16" else 0.0
    return 2 * (e + w) * vmax + (2.0 ** -8 * out.abs() if dtype == "bf16" else 2.0 ** -22 * vmax), 2 * e + 2.0 ** -20


def filled(B, lens, H, D, P, seed, gk, gv, shared=None, N=1):
    """A cache with random tokens: (pages, table, lists of stored k, v as float32)."""
    gen = torch.Generator().manual_seed(seed)
    pages, table = pool(B, lens, H, D, P, shared, N, seed)
    top = max(max(lens), 1)
    k = torch.randn(len(lens), top, H, D, generator=gen).cuda() * 1.5
    v = torch.randn(len(lens), top, H, D, generator=gen).cuda()
    if shared is not None:
        for i in range(len(lens)):
            s = shared[i // N]
            k[i, top - lens[i]:top - lens[i] + s] = k[i // N * N, top - lens[i // N * N]:][:s]
            v[i, top - lens[i]:top - lens[i] + s] = v[i // N * N, top - lens[i // N * N]:][:s]
    B.as_cache4_append(pages, k, v, table, i32(lens), gk, gv)
    ks, vs = B.as_cache4_load(pages, table, i32(lens), top, gk, gv, dtype=torch.float32)
    return pages, table, [ks[i, top - n:].cpu() for i, n in enumerate(lens)], [vs[i, top - n:].cpu() for i, n in enumerate(lens)]


SHAPES = [  # lens, T, Hq, H, P
    ([1], 1, 1, 1, 16), ([0, 1, 2, 15, 16, 17], 1, 2, 2, 16), ([31, 32, 33, 63, 64, 65], 1, 8, 2, 32), ([100, 7], 1, 7, 1, 64), ([700, 3, 129], 1, 12, 1, 64),
    ([130, 500], 1, 16, 2, 128), ([333, 40], 1, 24, 1, 16), ([5, 1, 0, 90], 3, 4, 2, 16), ([64, 200], 5, 8, 1, 64), ([150, 20], 20, 6, 3, 32),
    ([100, 260], 70, 4, 1, 64), ([400], 130, 5, 1, 16), ([2500], 1, 4, 4, 64), ([1, 4000, 1], 2, 2, 1, 64), ([300, 120], 129, 8, 2, 128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,T,Hq,H,P", SHAPES)
def test_attention(B, dtype, D, lens, T, Hq, H, P):
    gen = torch.Generator().manual_seed(T * 7 + Hq)
    gk, gv = (0.2 + 0.3 * torch.rand(H, generator=gen)).cuda(), (0.2 + 0.3 * torch.rand(H, generator=gen)).cuda()
    pages, table, k, v = filled(B, lens, H, D, P, 5, gk, gv)
    q = (torch.randn(len(lens), T, Hq + 3, D, generator=gen) * 1.5).to(DT[dtype]).cuda()[:, :, 2:2 + Hq]
    scale = 1 / math.sqrt(D)
    lse = torch.empty(len(lens), T, Hq, device="cuda")
    status = torch.full((len(lens),), 9, dtype=torch.int32, device="cuda")
    out = B.as_cache4_attend(pages, q, table, i32(lens), scale, gk, gv, lse=lse, lane_status=status)
    want, wlse, size = attention(q.cpu(), k, v, lens, scale)
    tol, ltol = bounds(dtype, size, max([float(x.abs().max()) for x in v if x.numel()] + [0.0]), want)
    assert (status == 0).all()
    assert ((out.double().cpu() - want).abs() <= tol).all()
    empty = torch.isinf(wlse)
    got = lse.double().cpu()
    assert torch.equal(got[empty], wlse[empty]) and (out.cpu()[empty] == 0).all()
    assert ((got - wlse)[~empty].abs() <= ltol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,Hq,H,D,P,shared,tails", [(2, 2, 1, 64, 16, [32], [1, 9]), (3, 4, 2, 128, 16, [0, 48], [5, 1, 17, 1, 2, 40]), (16, 8, 2, 128, 64, [640], list(range(1, 17))),
                                                      (32, 4, 1, 64, 32, [320], [1] * 31 + [70]), (33, 8, 1, 128, 64, [1024, 64], [1 + i % 7 for i in range(66)]),
                                                      (5, 40, 4, 64, 128, [256], [3, 1, 4, 1, 5])])
def test_shared_beginnings(B, dtype, N, Hq, H, D, P, shared, tails):
    lens = [shared[i // N] + t for i, t in enumerate(tails)]
    gen = torch.Generator().manual_seed(N)
    pages, table, k, v = filled(B, lens, H, D, P, 6, None, None, shared, N)
    q = (torch.randn(len(lens), 1, Hq, D, generator=gen) * 1.5).to(DT[dtype]).cuda()
    scale = 1 / math.sqrt(D)
    lse = torch.empty(len(lens), 1, Hq, device="cuda")
    out = B.as_cache4_attend(pages, q, table, i32(lens), scale, N=N, shared=i32(shared), lse=lse)
    want, wlse, size = attention(q.cpu(), k, v, lens, scale)
    tol, ltol = bounds(dtype, size, max(float(x.abs().max()) for x in v), want)
    assert ((out.double().cpu() - want).abs() <= tol).all()
    assert ((lse.double().cpu() - wlse).abs() <= ltol).all()
    # without the hint, and with one that cannot be (not a multiple of a page, longer than a lane): the same rows
    for hint in (None, i32([s + 1 for s in shared]), i32([1 << 20 for s in shared])):
        other = B.as_cache4_attend(pages, q, table, i32(lens), scale, N=N, shared=hint)
        assert ((other.double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_extreme_scores(B, dtype):
    """Scores far apart: one token takes all the weight, early, late or in the middle; a negative and a zero scale."""
    D, H, P, n = 64, 1, 16, 200
    k = torch.full((1, n, H, D), -4.0)
    v = torch.arange(n).float().view(1, n, 1, 1).expand(1, n, H, D).contiguous() % 7
    for top in (0, 77, 199):
        k[0, :, 0] = -4.0
        k[0, top, 0] = 4.0
        pages, table = pool(B, [n], H, D, P)
        B.as_cache4_append(pages, k.cuda(), v.cuda(), table, i32([n]))
        vs = B.as_cache4_load(pages, table, i32([n]), n, dtype=torch.float32)[1].cpu()
        q = torch.full((1, 1, 2, D), 8.0).to(DT[dtype]).cuda()
        out = B.as_cache4_attend(pages, q, table, i32([n]), 1.0).float().cpu()
        assert torch.equal(out[0, 0], vs[0, top].expand(2, D))
        out = B.as_cache4_attend(pages, q, table, i32([n]), 0.0).float().cpu()
        assert ((out - vs.mean(1, keepdim=True)).abs() < 0.02).all()
        out = B.as_cache4_attend(pages, q, table, i32([n]), -1.0).float().cpu()
        rest = torch.cat([vs[:, :top], vs[:, top + 1:]], 1).mean(1, keepdim=True)
        assert ((out - rest).abs() < 0.02).all()


def test_bad_lengths_and_pages(B):
    lens, H, D, P = [40, 40, 40], 2, 64, 16
    pages, table, k, v = filled(B, lens, H, D, P, 8, None, None)
    q = torch.randn(3, 1, 2, D).cuda()
    good = B.as_cache4_attend(pages, q, table, i32(lens), 0.1)
    status = i32([9, 9, 9])
    bad = table.clone()
    bad[1, 0] = 1 << 20
    out = B.as_cache4_attend(pages, q, bad, i32([40, 40, 1 << 29]), 0.1, lane_status=status)
    assert status.tolist() == [0, B.ERR_INVALID_ARG, B.ERR_INVALID_ARG]
    assert torch.equal(out[0], good[0]) and torch.isfinite(out).all() and not out[2].any()
    before = pages.clone()
    B.as_cache4_append(pages, torch.randn(3, 1, H, D).cuda(), torch.randn(3, 1, H, D).cuda(), torch.full_like(table, -1), i32([1, -5, 1 << 29]), lane_status=status)
    assert status.tolist() == [B.ERR_INVALID_ARG] * 3 and torch.equal(before, pages)
    kk, vv = B.as_cache4_load(pages, torch.full_like(table, 99), i32([1, -5, 1 << 29]), 2, lane_status=status)
    assert status.tolist() == [B.ERR_INVALID_ARG] * 3 and not kk.any() and not vv.any()


def test_pages_past_32_bits(B):
    """Pages whose bytes lie beyond 2^32 of the pool's start."""
    H, D, P = 8, 128, 128
    n = (5 << 30) // (H * (P // 16) * 18 * D)
    pages = B.cache4_pages(n, H, D, P)
    lens = [130, 60]
    table = i32([[n - 1, n - 3], [n - 2, -1]])
    k, v = torch.randn(2, 130, H, D).cuda(), torch.randn(2, 130, H, D).cuda()
    B.as_cache4_append(pages, k, v, table, i32(lens))
    small = B.cache4_pages(3, H, D, P)
    near = i32([[2, 0], [1, -1]])
    B.as_cache4_append(small, k, v, near, i32(lens))
    assert torch.equal(small, pages[n - 3:])
    q = torch.randn(2, 1, 16, D).cuda().bfloat16()
    assert torch.equal(B.as_cache4_attend(pages, q, table, i32(lens), 0.1), B.as_cache4_attend(small, q, near, i32(lens), 0.1))


def test_the_same_call_twice_and_other_streams(B):
    lens = [900, 30, 2000, 1]
    pages, table, k, v = filled(B, lens, 4, 128, 64, 9, None, None)
    q = torch.randn(4, 1, 16, 128).cuda().bfloat16()
    first = B.as_cache4_attend(pages, q, table, i32(lens), 0.09)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = B.as_cache4_attend(pages, q, table, i32(lens), 0.09)
        kk, vv = B.as_cache4_load(pages, table, i32(lens), 3)
        fresh = torch.zeros_like(pages)
        B.as_cache4_append(fresh, kk, vv, table, i32(lens))
    s.synchronize()
    assert torch.equal(first, other)
    for _ in range(3):
        assert torch.equal(first, B.as_cache4_attend(pages, q, table, i32(lens), 0.09))


def test_unaligned_queries_keys_and_values(B):
    """Base pointers that are only element-aligned, a pitch that is odd."""
    H, D, P, lens = 2, 64, 16, [37, 20]
    gen = torch.Generator().manual_seed(4)
    flat = torch.randn(1 + 2 * 2 * (H * D + 3) + 64, generator=gen).bfloat16().cuda()
    x = flat[1:1 + 2 * 2 * (H * D + 3)].view(2, 2, H * D + 3)[:, :, :H * D].unflatten(2, (H, D))
    pages, table = pool(B, lens, H, D, P)
    other, _ = pool(B, lens, H, D, P)
    B.as_cache4_append(pages, x, x, table, i32(lens))
    B.as_cache4_append(other, x.contiguous(), x.contiguous(), table, i32(lens))
    assert torch.equal(pages, other)
    pages, table, k, v = filled(B, lens, H, D, P, 3, None, None)
    assert torch.equal(B.as_cache4_attend(pages, x, table, i32(lens), 0.1), B.as_cache4_attend(pages, x.contiguous(), table, i32(lens), 0.1))


def test_a_wait_that_runs_out_reports_timeout_and_the_next_call_is_fine(B):
    """The kernel for many rows with a bound of a thousand cycles on its waits: it returns, says so, and nothing lingers."""
    lens, T = [700, 900], 300
    pages, table, k, v = filled(B, lens, 2, 128, 64, 11, None, None)
    q = torch.randn(2, T, 8, 128).cuda().bfloat16()
    good = B.as_cache4_attend(pages, q, table, i32(lens), 0.09)
    status = i32([9, 9])
    try:
        B.as_tune(B.TUNE_WAIT_KCYCLES, 1)
        B.as_cache4_attend(pages, q, table, i32(lens), 0.09, lane_status=status)
        torch.cuda.synchronize()
    finally:
        B.as_tune(B.TUNE_WAIT_KCYCLES, 0)
    assert status.tolist() == [B.ERR_TIMEOUT, B.ERR_TIMEOUT]
    again = B.as_cache4_attend(pages, q, table, i32(lens), 0.09, lane_status=status)
    assert torch.equal(again, good) and status.tolist() == [0, 0]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,T,Hq,H,D,P,shared,tails", [(2, 3, 4, 2, 64, 16, [64, 0], [6, 9, 3, 4]), (4, 40, 4, 1, 128, 32, [96], [40, 41, 60, 45]),
                                                       (2, 20, 2, 1, 64, 64, [64], [6, 30]), (3, 70, 4, 1, 64, 16, [160], [1, 70, 200]), (1, 5, 4, 2, 128, 16, [32], [7])])
def test_several_tokens_behind_a_shared_beginning(B, dtype, N, T, Hq, H, D, P, shared, tails):
    """Chunks of T tokens for lanes that share a beginning; some of their rows end within it."""
    lens = [shared[i // N] + t for i, t in enumerate(tails)]
    gen = torch.Generator().manual_seed(T)
    pages, table, k, v = filled(B, lens, H, D, P, 12, None, None, shared, N)
    q = (torch.randn(len(lens), T, Hq, D, generator=gen) * 1.5).to(DT[dtype]).cuda()
    lse = torch.empty(len(lens), T, Hq, device="cuda")
    out = B.as_cache4_attend(pages, q, table, i32(lens), 0.11, N=N, shared=i32(shared), lse=lse)
    want, wlse, size = attention(q.cpu(), k, v, lens, 0.11)
    tol, ltol = bounds(dtype, size, max(float(x.abs().max()) for x in v), want)
    assert ((out.double().cpu() - want).abs() <= tol).all()
    empty = torch.isinf(wlse)
    got = lse.double().cpu()
    assert torch.equal(got[empty], wlse[empty]) and (out.cpu()[empty] == 0).all()
    assert ((got - wlse)[~empty].abs() <= ltol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_lanes_of_many_lengths(B, dtype):
    """Enough items for a warp each, lengths of zero among them."""
    gen = torch.Generator().manual_seed(2)
    lens = torch.randint(0, 150, (700,), generator=gen).tolist()
    lens[0] = lens[350] = lens[699] = 0
    pages, table, k, v = filled(B, lens, 1, 64, 16, 13, None, None)
    q = torch.randn(700, 1, 2, 64, generator=gen).to(DT[dtype]).cuda()
    out = B.as_cache4_attend(pages, q, table, i32(lens), 0.125)
    want, _, size = attention(q.cpu(), k, v, lens, 0.125)
    tol, _ = bounds(dtype, size, max(float(x.abs().max()) for x in v if x.numel()), want)
    assert ((out.double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_long_prompts_bit_for_bit(B, dtype, D):
    """Many tokens a lane in one call: what the definition says, and what the same tokens give in pieces."""
    lens, T, H, P = [1999, 700, 31, 0, 703], 700, 3, 64
    gen = torch.Generator().manual_seed(D)
    k, v = ((torch.randn(len(lens), T, H, D, generator=gen) * torch.exp(2 * torch.randn(len(lens), T, H, 1, generator=gen))).to(DT[dtype]).cuda() for _ in range(2))
    gk, gv = 0.1 + torch.rand(H, generator=gen), 0.1 + torch.rand(H, generator=gen)
    pages, table = pool(B, lens, H, D, P)
    B.as_cache4_append(pages, k, v, table, i32(lens), gk.cuda(), gv.cuda())
    gotk, gotv = B.as_cache4_load(pages, table, i32(lens), T, gk.cuda(), gv.cuda(), dtype=torch.float32)
    for got, x, g in ((gotk, k, gk), (gotv, v, gv)):
        want = np.stack([quantise(x[:, :, h].float().cpu().numpy(), g[h])[0] for h in range(H)], axis=2)
        for i, n in enumerate(lens):
            want[i, :max(0, T - n)] = 0
        assert np.array_equal(got.cpu().numpy(), want)
    again, _ = pool(B, lens, H, D, P)
    for t in range(0, T, 100):
        B.as_cache4_append(again, k[:, t:t + 100].contiguous(), v[:, t:t + 100].contiguous(), table, i32([max(0, n - T + 100 + t) for n in lens]), gk.cuda(), gv.cuda())
    assert torch.equal(again, pages)
