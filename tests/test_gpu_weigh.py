"""Attention weights of cached tokens, against a plain implementation in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
from tests import test_gpu_cache4 as C  # noqa: E402
from tests.test_gpu_window import seen  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import binding
    return binding


def weights(q, lse, k, lens, scale, window, sinks):
    """([lanes] of float64 [H, len], bound on a score's size)."""
    lanes, T, Hq, D = q.shape
    got, size = [], 0.0
    for i in range(lanes):
        H = k[i].shape[1]
        w = torch.zeros(H, lens[i], dtype=torch.float64)
        for t in range(T):
            at = seen(lens[i] - T + 1 + t, window, sinks)
            if len(at) == 0:
                continue
            kk, x = k[i][at].double().repeat_interleave(Hq // H, 1), q[i, t].double()
            s = torch.einsum("nhd,hd->hn", kk, x) * scale
            size = max(size, float(torch.einsum("nhd,hd->hn", kk.abs(), x.abs()).max() * abs(scale)))
            z = lse[i, t].double().unsqueeze(1)
            e = torch.where(z == -math.inf, torch.zeros_like(s), torch.exp(s - z))
            w[:, at] += e.view(H, Hq // H, -1).sum(1)
        got.append(w)
    return got, size


def tolerance(size, top, rows, w):
    """A score is off by at most 2^-21 of the sum of its terms' magnitudes (operands and sums in 24 bits, each operand split exactly or
    to 2^-23), the difference to lse by 2^-22 of the larger one, the exponential by 2^-22; a sum of n terms by n 2^-24."""
    return (2.0 ** -21 * size + 2.0 ** -22 * (size + top) + 2.0 ** -22 + rows * 2.0 ** -24) * w + 1e-30


SHAPES = [  # lens, T, Hq, H, P, window, sinks
    ([1, 0, 2], 1, 1, 1, 16, 0, 0), ([40, 17, 33, 16], 1, 2, 2, 16, 0, 0), ([200, 64, 65, 90], 1, 8, 2, 32, 0, 0), ([500, 129, 16], 1, 7, 1, 64, 0, 0),
    ([700, 3, 140], 1, 12, 1, 64, 130, 17), ([999, 500], 1, 16, 2, 128, 0, 0), ([333, 41], 1, 24, 1, 16, 20, 1), ([5, 1, 0, 90], 3, 4, 2, 16, 0, 0),
    ([64, 300], 5, 8, 1, 64, 33, 40), ([150, 20], 20, 6, 3, 32, 0, 0), ([600, 260], 70, 4, 1, 64, 129, 5), ([400], 130, 5, 1, 16, 0, 0),
    ([2500, 2100], 1, 4, 4, 64, 0, 0), ([900, 120], 129, 8, 2, 128, 200, 50), ([300, 200], 200, 4, 2, 16, 0, 0), ([1100], 32, 8, 2, 64, 0, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,T,Hq,H,P,window,sinks", SHAPES)
def test_weights(B, dtype, D, lens, T, Hq, H, P, window, sinks):
    gen = torch.Generator().manual_seed(T * 7 + Hq)
    gk = (0.2 + 0.3 * torch.rand(H, generator=gen)).cuda()
    pages, table, k, v = C.filled(B, lens, H, D, P, 5, gk, None)
    q = (torch.randn(len(lens), T, Hq + 3, D, generator=gen) * 1.5).to(C.DT[dtype]).cuda()[:, :, 2:2 + Hq]
    scale = 1 / math.sqrt(D)
    lanes, W = len(lens), max(lens) + 5
    lse = torch.empty(lanes, T, Hq, device="cuda")
    B.as_cache4_attend(pages, q, table, C.i32(lens), scale, gk, lse=lse, window=window or None, sinks=sinks)
    span = window or 1 << 30
    want, size = weights(q.cpu(), lse.cpu(), k, lens, scale, span, sinks)
    finite = lse[torch.isfinite(lse)]
    top = float(finite.abs().max()) if finite.numel() else 0.0
    old = torch.rand(lanes, H, W, generator=gen)
    first = [min(n, 3 * i) for i, n in enumerate(lens)]
    for add in (True, False):
        for begin in (None, first):
            w = old.cuda()
            status = torch.full((lanes,), 9, dtype=torch.int32, device="cuda")
            B.as_cache4_weigh(pages, q, lse, table, C.i32(lens), scale, w, gk, window=window or None, sinks=sinks, add=add,
                              first=None if begin is None else C.i32(begin), lane_status=status)
            assert (status == 0).all()
            w = w.cpu()
            for i, n in enumerate(lens):
                lo = 0 if begin is None else begin[i]
                new = torch.arange(n) >= n - T if add else torch.ones(n, dtype=torch.bool)
                whole = want[i] + torch.where(new, torch.zeros(1, dtype=torch.float64), old[i, :, :n].double())
                tol = tolerance(size, top, T * Hq // H, want[i]) + 2.0 ** -24 * whole
                assert ((w[i, :, lo:n].double() - whole[:, lo:]).abs() <= tol[:, lo:]).all()
                assert torch.equal(w[i, :, n:], old[i, :, n:]) and torch.equal(w[i, :, :lo], old[i, :, :lo])
    # the same calls give the same bits
    a, b = old.cuda(), old.cuda()
    for x in (a, b):
        B.as_cache4_weigh(pages, q, lse, table, C.i32(lens), scale, x, gk, window=window or None, sinks=sinks)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [2, 40])
def test_rows_that_are_not_numbers(B, dtype, T):
    """lse -inf: the row adds nothing; a NaN in lse or query reaches what the row looks at, and nothing else."""
    n, H, D, P = 100, 2, 64, 16
    pages, table, k, v = C.filled(B, [n, n], H, D, P, 5, None, None)
    q = torch.randn(2, T, 4, D, generator=torch.Generator().manual_seed(3)).to(C.DT[dtype]).cuda()
    lse = torch.empty(2, T, 4, device="cuda")
    B.as_cache4_attend(pages, q, table, C.i32([n, n]), 0.1, lse=lse)
    lse[1, T - 1, :] = -math.inf
    want, size = weights(q.cpu(), lse.cpu(), k, [n, n], 0.1, 1 << 30, 0)
    lse[0, 0, 3] = math.nan
    q[1, 0, 0, 7] = math.nan
    w = torch.zeros(2, H, n, device="cuda")
    B.as_cache4_weigh(pages, q, lse, table, C.i32([n, n]), 0.1, w)
    w = w.cpu()
    upto = n - T + 1
    assert torch.isnan(w[0, 1, :upto]).all() and torch.isnan(w[1, 0, :upto]).all()
    fine = torch.ones(2, H, n, dtype=torch.bool)
    fine[0, 1, :upto] = fine[1, 0, :upto] = False
    tol = tolerance(size, 20.0, T * 2, torch.stack(want))
    # (behind what the broken rows look at the others' sums stand)
    assert ((w.double() - torch.stack(want)).abs() <= tol)[fine].all() and torch.isfinite(w[fine]).all()
    assert not w[1, :, n - 1].any()


def test_bad_lanes(B):
    n, H, D, P = 40, 2, 64, 16
    lens = [n] * 5
    pages, table, k, v = C.filled(B, lens, H, D, P, 8, None, None)
    q = torch.randn(5, 1, 2, D).cuda()
    lse = torch.zeros(5, 1, 2, device="cuda")
    w = torch.full((5, H, 44), 2.0, device="cuda")
    status = C.i32([9] * 5)
    bad = table.clone()
    bad[4, 0] = 1 << 20
    B.as_cache4_weigh(pages, q, lse, bad, C.i32([n, 1 << 29, n, 45, n]), 0.1, w, first=C.i32([0, 0, -1, 0, 0]), lane_status=status)
    E = B.ERR_INVALID_ARG
    assert status.tolist() == [0, E, E, E, E] and (w[1:4] == 2.0).all() and (w[0, :, :n] != 2.0).all() and torch.isfinite(w).all()
    w.fill_(2.0)
    B.as_cache4_weigh(pages, q, lse, table, C.i32(lens), 0.1, w, first=C.i32([41, 40, 0, 0, 0]), lane_status=status)
    assert status.tolist() == [E, 0, 0, 0, 0] and (w[:2] == 2.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,Hq", [(2, 2), (5, 4), (10, 4), (24, 4), (40, 4), (130, 4)])
def test_rows_that_see_nothing_may_hold_anything(B, dtype, T, Hq):
    """Padding in front of a short lane, and rows that the caller has taken out by an lse of -inf."""
    H, D, P = 2, 64, 16
    lens = [T // 2, 150, T + 20, 1, 0]
    pages, table, k, v = C.filled(B, lens, H, D, P, 5, None, None)
    q = torch.randn(5, T, Hq, D, generator=torch.Generator().manual_seed(3)).to(C.DT[dtype]).cuda()
    lse = torch.empty(5, T, Hq, device="cuda")
    B.as_cache4_attend(pages, q, table, C.i32(lens), 0.1, lse=lse)
    lse[1, T // 2:, ::2] = -math.inf
    lse[2] = -math.inf
    W = max(lens)
    old = torch.rand(5, H, W, device="cuda")
    clean, got = old.clone(), old.clone()
    B.as_cache4_weigh(pages, q, lse, table, C.i32(lens), 0.1, clean)
    for i, bad in enumerate((math.nan, math.inf, -math.inf)):
        q[:, :, :, i::3] = torch.where((lse == -math.inf).unsqueeze(3), torch.full_like(q[:, :, :, i::3], bad), q[:, :, :, i::3])
    B.as_cache4_weigh(pages, q, lse, table, C.i32(lens), 0.1, got)
    assert torch.equal(got, clean) and torch.isfinite(got).all()
    own = max(lens[2] - T, 0)
    assert torch.equal(got[2, :, :own], old[2, :, :own]) and not got[2, :, own:lens[2]].any()
