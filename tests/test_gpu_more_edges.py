"""Offsets past 32 bits, no lanes, results that do not depend on scheduling: windowed attention, weights, eviction, trim, verification."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from tests import test_gpu_cache4 as C  # noqa: E402
from tests import test_gpu_evict as E  # noqa: E402
from tests import test_gpu_verify as V  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import binding
    return binding


@pytest.mark.parametrize("T", [1, 40])
def test_pages_past_32_bits(B, T):
    """The same lanes in pages at a pool's beginning and beyond its first 2^32 bytes."""
    H, D, P, Hq = 8, 128, 128, 16
    n = (5 << 30) // (H * (P // 16) * 18 * D)
    pages = B.cache4_pages(n, H, D, P)
    lens = [300, 260]
    low, high = C.i32([[0, 1, 2], [3, 4, 5]]), C.i32([[n - 1, n - 3, n - 5], [n - 2, n - 6, n - 4]])
    gen = torch.Generator().manual_seed(1)
    k, v = torch.randn(2, 300, H, D, generator=gen).cuda(), torch.randn(2, 300, H, D, generator=gen).cuda()
    q = torch.randn(2, T, Hq, D, generator=gen).bfloat16().cuda()
    for t in (low, high):
        B.as_cache4_append(pages, k, v, t, C.i32(lens))
    got = []
    for t in (low, high):
        lse, w = torch.empty(2, T, Hq, device="cuda"), torch.zeros(2, H, 300, device="cuda")
        out = B.as_cache4_attend(pages, q, t, C.i32(lens), 0.1, lse=lse, window=50, sinks=3)
        B.as_cache4_attend(pages, q, t, C.i32(lens), 0.1, lse=lse)
        B.as_cache4_weigh(pages, q, lse, t, C.i32(lens), 0.1, w)
        weigh = w.clone()
        B.as_cache4_evict(pages, w, t, C.i32(lens), C.i32([100, 90]), 20, first=C.i32([2, 2]))
        got.append((out, weigh, w, torch.stack([E.tokens(pages, t, i, h, 90) for i in range(2) for h in range(H)])))
    assert all(torch.equal(a, b) for a, b in zip(*got)) and got[0][1].sum() > 0


@pytest.mark.parametrize("top_p", [1.0, 0.9])
def test_rows_past_32_bits(B, top_p):
    lanes, K, V_ = 12000, 1, 100003
    t = torch.zeros(lanes, K + 1, V_, dtype=torch.bfloat16, device="cuda")
    target, draft, drafted, u, codes = (x.cuda() for x in V.inputs(6, K, V_, "bf16", 3))
    t[-6:] = target
    d = torch.zeros(lanes, K, V_, dtype=torch.bfloat16, device="cuda")
    d[-6:] = draft
    all_drafted, all_u, all_codes = drafted[:1].expand(lanes, K).contiguous(), u[:1].expand(lanes, K).contiguous(), codes[:1].expand(lanes).contiguous()
    all_drafted[-6:], all_u[-6:], all_codes[-6:] = drafted, u, codes
    want = B.as_step_verify(target, draft, drafted, u, codes, 1.0, 0, top_p)
    got = B.as_step_verify(t, d, all_drafted, all_u, all_codes, 1.0, 0, top_p)
    assert torch.equal(got[0][-6:], want[0]) and torch.equal(got[1][-6:], want[1]) and (got[2][-6:] - want[2]).abs().max() < 1e-9
    # rows of zeros: every token alike, so that the draft is accepted; the code takes token floor(code V) where nothing is cut
    assert (got[1][:-6] == 1).all()
    if top_p == 1.0:
        assert (got[0][:-6, 1] == int(float(codes[0]) * V_)).all()


def test_no_lanes(B):
    pages = B.cache4_pages(4, 2, 64, 16)
    table, n = torch.empty(0, 3, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    q, w = torch.empty(0, 1, 2, 64, device="cuda"), torch.empty(0, 2, 48, device="cuda")
    assert B.as_cache4_attend(pages, q, table, n, 1.0, window=4).shape == q.shape
    B.as_cache4_weigh(pages, q, torch.empty(0, 1, 2, device="cuda"), table, n, 1.0, w)
    B.as_cache4_evict(pages, w, table, n, n)
    x = torch.empty(0, 3, 8, device="cuda")
    tokens, accepted, codes = B.as_step_verify(x, x[:, :2], torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, dtype=torch.float64, device="cuda"),
                                               torch.empty(0, dtype=torch.float64, device="cuda"))
    assert tokens.shape == (0, 3) and accepted.numel() == codes.numel() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top_p", [1.0, 0.9])
def test_the_same_call_gives_the_same_bits(B, dtype, top_p):
    """Tokens with p near q go through a list whose order depends on timing; rows behind a refusal may or may not be read."""
    target, draft, drafted, u, codes = (x.cuda() for x in V.inputs(200, 3, 20011, dtype, 7, alike=1e-3))
    u.fill_(0.9995)                                 # (many are refused, with little left of p - q)
    first = B.as_step_verify(target, draft, drafted, u, codes, 1.0, 0, top_p)
    assert (first[1] < 3).any()
    for _ in range(20):
        again = B.as_step_verify(target, draft, drafted, u, codes, 1.0, 0, top_p)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("offset", [1e4, -3e5, 1e12, 1e30])
@pytest.mark.parametrize("temp", [1e-3, 1.0, 1e4])
def test_logits_far_from_zero(B, offset, temp):
    """p and q depend on differences of logits alone; far out those are multiples of a float's spacing."""
    target, draft, drafted, u, codes = V.inputs(40, 2, 300, "f32", 11)
    target, draft = target + offset, draft + offset
    V.check(B, target, draft, drafted, u, codes, temp, 0, 1.0)
    V.check(B, target, draft, drafted, u, codes, temp, 0, 0.9)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temp", [1e-300, 1e-40, 1e-29, 1e29, 1e40, 1e300])
@pytest.mark.parametrize("lanes", [3, 700])
def test_temperatures_next_to_nothing_and_beyond_measure(B, dtype, temp, lanes):
    """The largest logit alone, or all that are not masked alike."""
    target, draft, drafted, u, codes = V.inputs(lanes, 2, 300, dtype, 13)
    target[:, :, 7:200] = float("-inf")
    draft[:, :, 5:150] = float("-inf")
    with np.errstate(over="ignore"):
        V.check(B, target, draft, drafted, u, codes, temp, 0, 1.0)
        V.check(B, target, None, drafted, u, codes, temp, 0, 1.0)


@pytest.mark.parametrize("window", [None, 150])
def test_a_wait_that_runs_out_reports_timeout_and_the_next_call_is_fine(B, window):
    """The kernels for many rows with a bound of a thousand cycles on their waits, their scratch full of what is no answer."""
    lens, T, H, sinks = [2700, 1900], 300, 2, 5
    pages, table, k, v = C.filled(B, lens, H, 128, 64, 11, None, None)
    q = torch.randn(2, T, 8, 128).cuda().bfloat16()
    lse, weight = torch.empty(2, T, 8, device="cuda"), torch.zeros(2, H, 2700, device="cuda")
    good = B.as_cache4_attend(pages, q, table, C.i32(lens), 0.09, lse=lse, window=window, sinks=sinks if window else 0)
    kw = dict(window=window, sinks=sinks if window else 0, add=False)
    B.as_cache4_weigh(pages, q, lse, table, C.i32(lens), 0.09, weight, **kw)
    statuses = [C.i32([9, 9]), C.i32([9, 9])]
    work = torch.full((B.as_cache4_weigh_work_bytes(pages, B.BF16, 2, T, 8),), 0x7F, dtype=torch.uint8, device="cuda")
    try:
        B.as_tune(B.TUNE_WAIT_KCYCLES, 1)
        B.as_cache4_attend(pages, q, table, C.i32(lens), 0.09, window=window, sinks=sinks if window else 0, lane_status=statuses[0])
        B.as_cache4_weigh(pages, q, lse, table, C.i32(lens), 0.09, torch.zeros_like(weight), lane_status=statuses[1], work=work, **kw)
        torch.cuda.synchronize()
    finally:
        B.as_tune(B.TUNE_WAIT_KCYCLES, 0)
    assert all(s.tolist() == [B.ERR_TIMEOUT, B.ERR_TIMEOUT] for s in statuses)
    again = torch.zeros_like(weight)
    B.as_cache4_weigh(pages, q, lse, table, C.i32(lens), 0.09, again, lane_status=statuses[1], work=work, **kw)
    assert torch.equal(again, weight) and statuses[1].tolist() == [0, 0] and weight.sum() > 0
    assert torch.equal(B.as_cache4_attend(pages, q, table, C.i32(lens), 0.09, window=window, sinks=sinks if window else 0, lane_status=statuses[0]), good)
    assert statuses[0].tolist() == [0, 0]


def test_weights_of_a_call_whose_waits_run_out_are_old_or_right(B):
    """Bounds that some of the kernel's runs keep and others do not, the scratch full of what is no answer."""
    lens, T, H, Hq = [6000, 4100, 777], 300, 2, 8
    pages, table, k, v = C.filled(B, lens, H, 128, 64, 11, None, None)
    q = torch.randn(3, T, Hq, 128, generator=torch.Generator().manual_seed(2)).cuda().bfloat16()
    lse, old = torch.empty(3, T, Hq, device="cuda"), 1 + torch.rand(3, H, 6000, device="cuda")
    B.as_cache4_attend(pages, q, table, C.i32(lens), 0.09, lse=lse)
    for add in (True, False):
        right = old.clone()
        B.as_cache4_weigh(pages, q, lse, table, C.i32(lens), 0.09, right, add=add)
        found = []
        for kcycles in (1, 2, 3, 4, 5, 6, 8, 10, 13, 16, 20, 25, 32, 40, 50, 64, 80, 100) * 3:
            w, status = old.clone(), C.i32([9] * 3)
            work = torch.full((B.as_cache4_weigh_work_bytes(pages, B.BF16, 3, T, Hq),), 0x7F, dtype=torch.uint8, device="cuda")
            try:
                B.as_tune(B.TUNE_WAIT_KCYCLES, kcycles)
                B.as_cache4_weigh(pages, q, lse, table, C.i32(lens), 0.09, w, add=add, lane_status=status, work=work)
                torch.cuda.synchronize()
            finally:
                B.as_tune(B.TUNE_WAIT_KCYCLES, 0)
            out = status.tolist()
            found.append((kcycles, out, int(((w != old) & (w != right)).sum())))
            assert out in ([0] * 3, [B.ERR_TIMEOUT] * 3)
            assert out != [0] * 3 or torch.equal(w, right)
        assert any(out != [0] * 3 for _, out, _ in found) and all(n == 0 for _, _, n in found), found


@pytest.mark.parametrize("rise,other", [(0.5, 3.0), (3.0, 0.5), (20.0, 18.0), (200.0, 190.0)])
def test_long_rows_that_rise_all_the_way(B, rise, other):
    """Rows of nearly 2^20 tokens, summed by one CTA to a lane, whose running maxima go up at every step; u at and around the border."""
    lanes, V_ = 240, (1 << 20) - 5
    t, d = torch.linspace(-rise, 0, V_, device="cuda"), torch.linspace(-other, 0, V_, device="cuda")
    x = V_ - 9 if rise < other else V_ // 2 if rise < 10 else V_ - 40000
    # (64-bit sums on the GPU; both probabilities are within 1e-12 of themselves)
    px, qx = (float(torch.softmax(r.double(), 0)[x]) for r in (t, d))
    if px > qx:
        t, d, px, qx = d, t, qx, px
    delta = torch.tensor([s * 2.0 ** -(8 + k / 4) for k in range(lanes // 2) for s in (1, -1)], dtype=torch.float64)
    u = (px / qx * (1 + delta)).view(lanes, 1)
    assert u.max() < 1
    target = t.expand(lanes, 2, V_).contiguous()
    draft = d.expand(lanes, 1, V_).contiguous()
    drafted = torch.full((lanes, 1), x, dtype=torch.int32, device="cuda")
    codes = torch.full((lanes,), 0.37, dtype=torch.float64, device="cuda")
    tokens, accepted, _ = B.as_step_verify(target, draft, drafted, u.cuda(), codes)
    sure = delta.abs() > 1e-11
    assert torch.equal((accepted.cpu() == 1)[sure], (delta < 0)[sure]) and int(sure.sum()) > 200
