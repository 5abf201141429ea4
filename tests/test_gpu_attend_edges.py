"""Attention over the 4-bit cache where its inputs are at their edges, in every kernel: rows of few and of many queries, with and
without a shared beginning."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
# query rows on the same tokens: a tile of 8 rows, of 16, of 128 and of 256 (in 32 bits all are cut into tiles of 8)
ROWS = [1, 7, 12, 64, 300]


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import binding
    return binding


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def cache(B, lanes, n, D, P=64, seed=0, k=None, v=None):
    """Lanes of n tokens, one head, that hold the same pages: (pages, table, lengths, stored k, v [n, D] as float64)."""
    g = torch.Generator().manual_seed(seed)
    k = torch.randn(n, D, generator=g) * 1.5 if k is None else k
    v = torch.randn(n, D, generator=g) if v is None else v
    M = -(-n // P)
    pages = B.cache4_pages(M, 1, D, P)
    row = torch.randperm(M, generator=g).to(torch.int32).view(1, M).cuda()
    B.as_cache4_append(pages, k.view(1, n, 1, D).cuda(), v.view(1, n, 1, D).cuda(), row, i32([n]))
    ks, vs = B.as_cache4_load(pages, row, i32([n]), n, dtype=torch.float32)
    return pages, row.expand(lanes, M).contiguous(), i32([n] * lanes), ks[0, :, 0].double().cpu(), vs[0, :, 0].double().cpu()


def poisoned(q, rows, how):
    bad = q.clone()
    for j in rows:
        flat = bad.view(-1, q.shape[-1])[j]
        if how == "nan":
            flat[5] = float("nan")
        elif how == "all_nan":
            flat[:] = float("nan")
        else:
            flat[3], flat[40] = float("inf"), float("-inf")
    return bad


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["nan", "all_nan", "inf"])
@pytest.mark.parametrize("rows", ROWS)
def test_a_query_that_is_not_finite_makes_its_own_row_nan(B, dtype, rows, how):
    D, n = 64, 700
    pages, table, length, k, v = cache(B, 1, n, D)
    g = torch.Generator().manual_seed(rows)
    q = torch.randn(1, 1, rows, D, generator=g).to(DT[dtype]).cuda()
    hit = sorted({0, rows // 2, rows - 1}) if rows > 2 else [0]
    lse, blse = (torch.empty(1, 1, rows, device="cuda") for _ in range(2))
    clean = B.as_cache4_attend(pages, q, table, length, 0.125, lse=lse)
    got = B.as_cache4_attend(pages, poisoned(q, hit, how), table, length, 0.125, lse=blse)
    rest = [r for r in range(rows) if r not in hit]
    assert torch.isnan(got[0, 0, hit]).all() and torch.isnan(blse[0, 0, hit]).all()
    assert torch.equal(got[0, 0, rest], clean[0, 0, rest]) and torch.equal(blse[0, 0, rest], lse[0, 0, rest])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,g", [(2, 1), (3, 4), (16, 4), (40, 8)])
def test_the_same_behind_a_shared_beginning(B, dtype, N, g):
    D, n, P = 128, 700, 64
    pages, table, length, k, v = cache(B, N, n, D, P)
    gen = torch.Generator().manual_seed(N)
    q = torch.randn(N, 1, g, D, generator=gen).to(DT[dtype]).cuda()
    bad = poisoned(q, [1, N * g - 1], "all_nan")
    lse = torch.empty(N, 1, g, device="cuda")
    for shared in (i32([640]), i32([64]), None):
        clean = B.as_cache4_attend(pages, q, table, length, 0.1, N=N, shared=shared)
        got = B.as_cache4_attend(pages, bad, table, length, 0.1, N=N, shared=shared, lse=lse)
        hit = torch.zeros(N * g, dtype=torch.bool)
        hit[[1, N * g - 1]] = True
        assert torch.isnan(got.view(N * g, D)[hit.cuda()]).all() and torch.equal(torch.isnan(lse.view(-1)).cpu(), hit)
        assert torch.equal(got.view(N * g, D)[~hit.cuda()], clean.view(N * g, D)[~hit.cuda()])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [3, 90, 300])
def test_rows_that_see_nothing_stay_zero_beside_rows_that_are_nan(B, dtype, T):
    """More query tokens than the lane has: the first ones are padding, whatever their queries hold."""
    D, n = 64, 2
    pages, table, length, k, v = cache(B, 1, n, D, 16)
    q = torch.full((1, T, 2, D), float("nan")).to(DT[dtype]).cuda()
    q[:, -1] = 1.0
    lse = torch.empty(1, T, 2, device="cuda")
    out = B.as_cache4_attend(pages, q, table, length, 0.125, lse=lse)
    assert (out[0, :T - n] == 0).all() and (lse[0, :T - n] == -math.inf).all()
    assert torch.isnan(out[0, T - n:-1]).all() and torch.isfinite(out[0, -1]).all()


def test_a_page_table_so_wide_that_units_for_warps_could_not_be_counted(B):
    """512 items of lanes whose tables have room for 2^29 tokens: a run for each CTA, the same rows as with a table that is cut."""
    lanes, H, T, Hq, D, P, n = 8, 8, 8, 64, 64, 128, 300
    g = torch.Generator().manual_seed(5)
    M = (1 << 22) - 1
    wide = torch.full((lanes, M), -1, dtype=torch.int32, device="cuda")
    wide[:, :3] = torch.randperm(3 * lanes, generator=g).to(torch.int32).view(lanes, 3).cuda()
    pages = B.cache4_pages(3 * lanes, H, D, P)
    k, v = (torch.randn(lanes, n, H, D, generator=g).cuda() for _ in range(2))
    length = i32([n - i for i in range(lanes)])
    B.as_cache4_append(pages, k, v, wide, length)
    q = torch.randn(lanes, T, Hq, D, generator=g).cuda()
    near = B.as_cache4_attend(pages, q, wide[:, :3].contiguous(), length, 0.125)
    # two results, each off by at most what sums and weights of 24 bits are (scores here are below 100)
    tol = 2 * (2 * (2.0 ** -21 * 100 + 2.0 ** -20) + 2.0 ** -22) * float(v.abs().max()) * 1.2
    assert ((B.as_cache4_attend(pages, q, wide, length, 0.125) - near).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("peak", [0, 15000, 29999])
@pytest.mark.parametrize("down", [25.5, 30.0])
@pytest.mark.parametrize("many", [False, True])
def test_one_peak_and_a_long_tail(B, dtype, rows, peak, down, many):
    """One token stands above 29999 others, each of which has 2^-down of its weight; only the others have a value.  Their part
    of the result is theirs together, however small each is: n 2^-25.5 is 6.3e-4 of all weight.

    Relative error of that part: scores as in the other tests (e, in numerator and sum), sums in 32 bits of n / 8 weights
    (2^-24 each) and of n / 16 products (2^-23 each, cut off by the tensor cores), and the output's rounding (2^-22; bf16: 2^-8, and 2^-11 of a weight);
    absolute: a weight is held to 2^-25 in units in which the largest is at least 2^7 (32 bits: 2^12).
    Many lanes: an item's tokens are then seen by one run, or few, in place of all of them."""
    D, n = 64, 30000
    k, v = torch.zeros(n, D), torch.ones(n, D)
    k[peak], v[peak] = 1.0, 0.0
    g, N = (rows, 1) if rows < 300 else (30, 10)
    pages, table, length, ks, vs = cache(B, N, n, D, 64, 1, k, v)
    size = down * math.log(2.0)
    scale = size / float(ks[peak].sum())
    q = torch.ones(N, 1, g, D).to(DT[dtype]).cuda()
    w = 2.0 ** -down * (n - 1)
    v1 = float(vs[(peak + 1) % n, 0])
    want, wlse = w * v1 / (1 + w), size + math.log1p(w)
    e = 2.0 ** -21 * size + 2.0 ** -20
    rel = 2 * e + n / 8 * 2.0 ** -24 + n / 16 * 2.0 ** -23 + (2.0 ** -8 + 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22)
    tol = want * rel + n * v1 * 2.0 ** (-37 if dtype == "f32" else -32)
    if many:
        copies = (600 if rows < 64 else 200) // N
        table, length, q = table.repeat(copies, 1), length.repeat(copies), q.repeat(copies, 1, 1, 1)
    lanes = q.shape[0]
    lse = torch.empty(lanes, 1, g, device="cuda")
    for shared in (None,) if N == 1 else (None, i32([n // 64 * 64] * (lanes // N)), i32([n // 128 * 64] * (lanes // N))):
        out = B.as_cache4_attend(pages, q, table, length, scale, N=N, shared=shared, lse=lse)
        assert float((out.double() - want).abs().max()) <= tol
        assert float((lse.double() - wlse).abs().max()) <= 2 * e + n / 8 * 2.0 ** -24 + 2.0 ** -20


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("fill", [0x7F, 0xFF])
def test_what_lies_behind_the_last_token_does_not_count(B, dtype, D, rows, fill):
    """Pages that end inside a tile, the rest of them filled with bytes whose scales are NaN: the same bits as with zeros."""
    P, lens = 128, [1, 15, 17, 33, 129, 250, 511]
    g = torch.Generator().manual_seed(D)
    k, v = (torch.randn(len(lens), 511, 2, D, generator=g).cuda() for _ in range(2))
    table = torch.randperm(4 * len(lens), generator=g).to(torch.int32).view(len(lens), 4).cuda()
    q = torch.randn(len(lens), 1, 2 * rows, D, generator=g).to(DT[dtype]).cuda()
    got = []
    for byte in (0, fill):
        pages = B.cache4_pages(4 * len(lens), 2, D, P)
        pages.fill_(byte)
        B.as_cache4_append(pages, k, v, table, i32(lens))
        lse = torch.empty(len(lens), 1, 2 * rows, device="cuda")
        got.append((B.as_cache4_attend(pages, q, table, i32(lens), 0.125, lse=lse), lse))
    assert torch.isfinite(got[0][0]).all() and torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
