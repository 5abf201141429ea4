"""Attention with a sliding window and visible first tokens, against a plain implementation in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
from tests import test_gpu_cache4 as C  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import binding
    return binding


def seen(n, window, sinks):
    """The positions that a query token looks at whose own is n - 1."""
    p = torch.arange(max(n, 0))
    return p[(p >= n - window) | (p < sinks)]


def attention(q, k, v, lens, scale, window, sinks):
    lanes, T, Hq, D = q.shape
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full((lanes, T, Hq), -math.inf, dtype=torch.float64)
    size = 0.0
    for i in range(lanes):
        H = k[i].shape[1]
        for t in range(T):
            at = seen(lens[i] - T + 1 + t, window, sinks)
            if len(at) == 0:
                continue
            kk, vv = k[i][at].double().repeat_interleave(Hq // H, 1), v[i][at].double().repeat_interleave(Hq // H, 1)
            x = q[i, t].double()
            s = torch.einsum("nhd,hd->hn", kk, x) * scale
            size = max(size, float(torch.einsum("nhd,hd->hn", kk.abs(), x.abs()).max() * abs(scale)))
            lse[i, t] = torch.logsumexp(s, 1)
            out[i, t] = torch.einsum("hn,nhd->hd", torch.softmax(s, 1), vv)
    return out, lse, size


def check(B, dtype, out, lse, q, k, v, lens, scale, window, sinks):
    want, wlse, size = attention(q.cpu(), k, v, lens, scale, window, sinks)
    tol, ltol = C.bounds(dtype, size, max([float(x.abs().max()) for x in v if x.numel()] + [0.0]), want)
    assert ((out.double().cpu() - want).abs() <= tol).all()
    empty, got = torch.isinf(wlse), lse.double().cpu()
    assert torch.equal(got[empty], wlse[empty]) and (out.cpu()[empty] == 0).all()
    assert ((got - wlse)[~empty].abs() <= ltol).all()


SHAPES = [  # lens, T, Hq, H, P, window, sinks
    ([1, 0, 2], 1, 1, 1, 16, 1, 0), ([40, 17, 33, 16], 1, 2, 2, 16, 7, 3), ([200, 64, 65, 90], 1, 8, 2, 32, 32, 16), ([500, 129, 16], 1, 7, 1, 64, 100, 0),
    ([700, 3, 140], 1, 12, 1, 64, 130, 17), ([999, 500], 1, 16, 2, 128, 257, 130), ([333, 41], 1, 24, 1, 16, 20, 1), ([5, 1, 0, 90], 3, 4, 2, 16, 4, 2),
    ([64, 300], 5, 8, 1, 64, 33, 40), ([150, 20], 20, 6, 3, 32, 11, 4), ([600, 260], 70, 4, 1, 64, 129, 5), ([400], 130, 5, 1, 16, 64, 0),
    ([2500, 2100], 1, 4, 4, 64, 1000, 4), ([1, 4000, 1], 2, 2, 1, 64, 512, 100), ([900, 120], 129, 8, 2, 128, 200, 50), ([100], 1, 4, 1, 16, 1000, 4),
    ([100], 1, 4, 1, 16, 1, 1000), ([260], 40, 4, 1, 16, 1 << 30, 0), ([700], 1, 4, 1, 16, 1, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,T,Hq,H,P,window,sinks", SHAPES)
def test_attention(B, dtype, D, lens, T, Hq, H, P, window, sinks):
    gen = torch.Generator().manual_seed(T * 7 + Hq)
    gk, gv = (0.2 + 0.3 * torch.rand(H, generator=gen)).cuda(), (0.2 + 0.3 * torch.rand(H, generator=gen)).cuda()
    pages, table, k, v = C.filled(B, lens, H, D, P, 5, gk, gv)
    q = (torch.randn(len(lens), T, Hq + 3, D, generator=gen) * 1.5).to(C.DT[dtype]).cuda()[:, :, 2:2 + Hq]
    scale = 1 / math.sqrt(D)
    lse = torch.empty(len(lens), T, Hq, device="cuda")
    status = torch.full((len(lens),), 9, dtype=torch.int32, device="cuda")
    out = B.as_cache4_attend(pages, q, table, C.i32(lens), scale, gk, gv, lse=lse, lane_status=status, window=window, sinks=sinks)
    assert (status == 0).all()
    check(B, dtype, out, lse, q, k, v, lens, scale, window, sinks)


SHARED = [
    (2, 1, 2, 1, 64, 16, [32], [1, 9], 20, 2), (3, 1, 4, 2, 128, 16, [0, 48], [5, 1, 17, 1, 2, 40], 30, 4), (16, 1, 8, 2, 128, 64, [640], list(range(1, 17)), 300, 70),
    (32, 1, 4, 1, 64, 32, [320], [1] * 31 + [70], 50, 0), (33, 1, 8, 1, 128, 64, [1024, 64], [1 + i % 7 for i in range(66)], 128, 17),
    (5, 1, 40, 4, 64, 128, [256], [3, 1, 4, 1, 200], 100, 1), (4, 3, 4, 2, 64, 16, [160], [6, 9, 40, 200], 60, 5), (4, 40, 4, 1, 128, 32, [96], [40, 41, 60, 45], 64, 3),
    (2, 1, 4, 2, 64, 16, [160], [100, 90], 64, 0), (64, 1, 4, 1, 64, 128, [1280], [1 + i for i in range(64)], 700, 128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,T,Hq,H,D,P,shared,tails,window,sinks", SHARED)
def test_shared_beginnings(B, dtype, N, T, Hq, H, D, P, shared, tails, window, sinks):
    lens = [shared[i // N] + t for i, t in enumerate(tails)]
    gen = torch.Generator().manual_seed(N)
    pages, table, k, v = C.filled(B, lens, H, D, P, 6, None, None, shared, N)
    q = (torch.randn(len(lens), T, Hq, D, generator=gen) * 1.5).to(C.DT[dtype]).cuda()
    scale = 1 / math.sqrt(D)
    for hint in (C.i32(shared), None):
        lse = torch.empty(len(lens), T, Hq, device="cuda")
        out = B.as_cache4_attend(pages, q, table, C.i32(lens), scale, N=N, shared=hint, lse=lse, window=window, sinks=sinks)
        check(B, dtype, out, lse, q, k, v, lens, scale, window, sinks)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,T,Hq,H,D,P,shared,tails,window,sinks", SHARED)
def test_shared_beginnings_by_groups(B, dtype, N, T, Hq, H, D, P, shared, tails, window, sinks):
    """The same where small windows are read by groups as well."""
    try:
        B.as_tune(B.TUNE_WINDOW_GROUPS, 1)
        test_shared_beginnings(B, dtype, N, T, Hq, H, D, P, shared, tails, window, sinks)
    finally:
        B.as_tune(B.TUNE_WINDOW_GROUPS, 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_windows_that_are_read_by_groups_unasked(B, dtype):
    """64 lanes x 8 heads x 1900 tokens of 144 bytes are more than 2^27 bytes."""
    test_shared_beginnings(B, dtype, 32, 1, 8, 8, 128, 64, [2048, 1984], [1 + i % 9 for i in range(64)], 1900, 4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,Hq", [(1, 4), (1, 12), (30, 4), (70, 4)])
def test_a_window_of_everything_is_plain_attention(B, dtype, T, Hq):
    lens, H, D, P = [300, 77, 130], 1, 128, 32
    pages, table, k, v = C.filled(B, lens, H, D, P, 3, None, None)
    q = torch.randn(3, T, Hq, D, generator=torch.Generator().manual_seed(1)).to(C.DT[dtype]).cuda()
    plain = B.as_cache4_attend(pages, q, table, C.i32(lens), 0.1)
    assert torch.equal(plain, B.as_cache4_attend(pages, q, table, C.i32(lens), 0.1, window=300))
    assert torch.equal(plain, B.as_cache4_attend(pages, q, table, C.i32(lens), 0.1, window=1, sinks=300))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,Hq", [(1, 4), (1, 12), (5, 8), (70, 4)])
def test_what_no_row_sees_does_not_count(B, dtype, T, Hq):
    """Pages in between may be given up (no valid id); NaN scales of tokens in front of the window and behind the sinks."""
    lens, H, D, P, window, sinks = [520, 700], 1, 64, 16, 100, 5
    pages, table, k, v = C.filled(B, lens, H, D, P, 4, None, None)
    q = torch.randn(2, T, Hq, D, generator=torch.Generator().manual_seed(2)).to(C.DT[dtype]).cuda()
    want = B.as_cache4_attend(pages, q, table, C.i32(lens), 0.2, window=window, sinks=sinks)
    spoilt, holes = pages.clone(), table.clone()
    for i, n in enumerate(lens):
        low = n - T + 1 - window
        holes[i, 1:low // P] = -1 if i == 0 else 1 << 30
        for p in [x for x in range(sinks, P)] + [x for x in range(low // P * P, low)]:
            page, tile, t = int(table[i, p // P]), p % P // 16, p % 16
            spoilt[page, :, tile, 16 * D + t * (D // 16):16 * D + (t + 1) * (D // 16)] = 0x7F
            for b in range(D // 16):
                spoilt[page, :, tile, 17 * D + b * 16 + t] = 0x7F
    status = C.i32([9, 9])
    got = B.as_cache4_attend(spoilt, q, holes, C.i32(lens), 0.2, window=window, sinks=sinks, lane_status=status)
    assert status.tolist() == [0, 0] and torch.equal(got, want)


def test_bad_lengths_and_pages(B):
    lens, H, D, P = [40, 40, 40], 2, 64, 16
    pages, table, k, v = C.filled(B, lens, H, D, P, 8, None, None)
    q = torch.randn(3, 1, 2, D).cuda()
    good = B.as_cache4_attend(pages, q, table, C.i32(lens), 0.1, window=10, sinks=2)
    status = C.i32([9, 9, 9])
    bad = table.clone()
    bad[1, 0] = 1 << 20
    out = B.as_cache4_attend(pages, q, bad, C.i32([40, 40, 1 << 29]), 0.1, lane_status=status, window=10, sinks=2)
    assert status.tolist() == [0, B.ERR_INVALID_ARG, B.ERR_INVALID_ARG]
    assert torch.equal(out[0], good[0]) and torch.isfinite(out).all() and not out[2].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,T,Hq,H,D,P,shared,tails,window,sinks", [
    (2, 1, 2, 1, 64, 16, [320, 160], [300, 1, 90, 200], 64, 5), (3, 1, 4, 2, 128, 16, [480], [200, 400, 30], 150, 0), (4, 3, 4, 1, 64, 32, [640], [90, 3, 500, 250], 200, 40),
    (33, 1, 8, 1, 128, 64, [1024], [1 + 37 * (32 - i) % 700 for i in range(33)], 400, 17), (40, 1, 8, 2, 64, 16, [512, 0], [600 - 7 * i for i in range(80)], 333, 1)])
def test_shared_beginnings_that_longer_lanes_have_given_up(B, dtype, N, T, Hq, H, D, P, shared, tails, window, sinks):
    """Each lane gives up what its own window has left behind; a shorter one of its group still sees, and holds, some of it."""
    lens = [shared[i // N] + t for i, t in enumerate(tails)]
    gen = torch.Generator().manual_seed(N)
    pages, table, k, v = C.filled(B, lens, H, D, P, 6, None, None, shared, N)
    q = (torch.randn(len(lens), T, Hq, D, generator=gen) * 1.5).to(C.DT[dtype]).cuda()
    held = table[table >= 0].long()
    ref = torch.bincount(held, minlength=pages.shape[0]).int()
    low = [max(n - T + 1 - window, 0) for n in lens]
    gone = C.i32([[-(-sinks // P) * P, x] for x in low])
    cut, left = table.clone(), ref.clone()
    B.as_pages_trim(None, cut, C.i32(lens), left, P, gone=gone)
    assert any(((cut[i // N * N] < 0) & (cut[i] >= 0))[:shared[i // N] // P].any() for i in range(len(lens)))
    pages[(left == 0).nonzero().flatten()] = 0xFF           # (and pages that nobody holds may hold anything)
    scale, status = 1 / math.sqrt(D), C.i32([9] * len(lens))
    for groups in (0, 1):
        try:
            B.as_tune(B.TUNE_WINDOW_GROUPS, groups)
            lse = torch.empty(len(lens), T, Hq, device="cuda")
            out = B.as_cache4_attend(pages, q, cut, C.i32(lens), scale, N=N, shared=C.i32(shared), lse=lse, window=window, sinks=sinks, lane_status=status)
        finally:
            B.as_tune(B.TUNE_WINDOW_GROUPS, 0)
        assert (status == 0).all()
        check(B, dtype, out, lse, q, k, v, lens, scale, window, sinks)
