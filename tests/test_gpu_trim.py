"""as_pages_trim against a plain page-by-page model: exact equality."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import binding
    return binding


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def model(table, lens, ref, P, keep, gone):
    """(table, lengths, ref, status) of lists; the reference counts are judged as they were."""
    out, n_out, r_out, status = [list(r) for r in table], list(lens), list(ref), []
    for i, n in enumerate(lens):
        k = n if keep is None else keep[i]
        left = min(n, k)
        rows = range(-(-n // P)) if 0 <= n <= len(table[i]) * P else []
        bad = not 0 <= n <= len(table[i]) * P or k < 0 or any(not -1 <= table[i][m] < len(ref) for m in rows)
        if not bad and left < n and left % P and table[i][left // P] >= 0:
            bad = ref[table[i][left // P]] > 1
        status.append(-1 if bad else 0)
        if bad:
            continue
        lo, hi = (0, 0) if gone is None else gone[i]
        for m in range(len(table[i])):
            if m * P >= left or (m * P >= lo and (m + 1) * P <= min(hi, left)):
                if m in rows and table[i][m] >= 0:
                    r_out[table[i][m]] -= 1
                out[i][m] = -1
        n_out[i] = left
    return out, n_out, r_out, status


def make(rng, lanes, P, M, share):
    """Lanes that share full leading pages now and then; some pages given up before."""
    lens = [rng.choice((0, 1, P, rng.randint(0, M * P))) for _ in range(lanes)]
    ids = list(range(lanes * M + 3))
    rng.shuffle(ids)
    ref, table = [0] * len(ids), []
    for i, n in enumerate(lens):
        row = []
        for m in range(-(-n // P)):
            other = rng.randrange(i) if i and share else None
            if other is not None and lens[other] >= (m + 1) * P <= n and rng.random() < 0.5 and table[other][m] >= 0:
                row.append(table[other][m])
            elif rng.random() < 0.05:
                row.append(-1)
            else:
                row.append(ids.pop())
            if row[-1] >= 0:
                ref[row[-1]] += 1
        table.append(row + [-1] * (M - len(row)))
    return table, lens, ref


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("seed", range(12))
def test_against_the_model(B, seed, in_place):
    rng = random.Random(seed)
    lanes, P, M = rng.choice((1, 5, 40, 300)), rng.choice((1, 16, 24, 64)), rng.choice((1, 7, 150))
    table, lens, ref = make(rng, lanes, P, M, seed % 2)
    keep = None if seed % 5 == 4 else [rng.choice((n, n + 3, max(0, n - rng.randint(0, 20)), rng.randint(0, n), 0)) for n in lens]
    gone = None if seed % 3 == 0 else [rng.choice(((0, 0), (P, n - 5), (-7, n + 100), (rng.randint(0, n), rng.randint(0, n)))) for n in lens]
    want = model(table, lens, ref, P, keep, gone)
    t, n, r = i32(table), i32(lens), i32(ref)
    outs = (t, n, r) if in_place else tuple(torch.full_like(x, 99) for x in (t, n, r))
    status = i32([9] * lanes)
    got = B.as_pages_trim(None if keep is None else i32(keep), t, n, r, P, gone=None if gone is None else i32(gone), table_out=outs[0], length_out=outs[1],
                          ref_out=outs[2], lane_status=status)
    assert all(a.data_ptr() == b.data_ptr() for a, b in zip(got, outs))
    assert (got[0].tolist(), got[1].tolist(), got[2].tolist(), status.tolist()) == want
    if not in_place:
        assert t.tolist() == table and n.tolist() == lens and r.tolist() == ref


def test_bad_lanes_and_no_lanes(B):
    P = 16
    table, lens, ref = [[0, 1, 2, -1], [3, 99, 4, -1], [5, 6, -1, -1], [0, 7, -1, -1], [8, -1, -1, -1]], [40, 40, 1000, 20, 10], [2, 1, 1, 1, 1, 1, 1, 1, 1, 0]
    keep = [8, 8, 8, 8, -2]
    want = model(table, lens, ref, P, keep, None)
    assert want[3] == [-1] * 5                      # (page 0 is held twice and would end up partly filled)
    t, n, r, status = i32(table), i32(lens), i32(ref), i32([9] * 5)
    B.as_pages_trim(i32(keep), t, n, r, P, lane_status=status)
    assert (t.tolist(), n.tolist(), r.tolist(), status.tolist()) == want
    # down to whole pages it may be cut, and to nothing
    keep = [16, 40, 0, 0, 0]
    lens[2] = 20
    want = model(table, lens, ref, P, keep, None)
    n = i32(lens)
    B.as_pages_trim(i32(keep), t, n, r, P, lane_status=status)
    assert (t.tolist(), n.tolist(), r.tolist(), status.tolist()) == want
    empty = torch.empty(0, 4, dtype=torch.int32, device="cuda")
    out = torch.full_like(r, 5)
    B.as_pages_trim(i32([]), empty, i32([]), r, P, ref_out=out)
    assert torch.equal(out, r)


def test_trimmed_lanes_grow_again(B):
    P = 16
    t, n, r = i32([[-1] * 6] * 3), i32([0] * 3), i32([0] * 20)
    B.as_pages_grow(i32([50, 70, 33]), t, n, r, P)
    B.as_pages_trim(i32([48, 60, 33]), t, n, r, P, gone=i32([[0, 0], [16, 48], [0, 16]]))
    assert n.tolist() == [48, 60, 33] and int(r.sum()) == 3 + 2 + 2
    B.as_pages_grow(i32([1, 10, 0]), t, n, r, P)
    assert n.tolist() == [49, 70, 33]
    held = torch.bincount(t[t >= 0].long(), minlength=20)
    assert torch.equal(held.int(), r)
    B.as_pages_trim(i32([0] * 3), t, n, r, P)
    assert not r.any() and (t == -1).all()


def test_a_lane_cut_into_what_it_has_given_up(B):
    """Its last page is partly filled and not there: it cannot grow before it is cut to a page's end."""
    P = 16
    t, n, r = i32([[-1] * 8] * 4), i32([0] * 4), i32([0] * 40)
    B.as_pages_grow(i32([100, 100, 100, 40]), t, n, r, P)
    B.as_pages_trim(None, t, n, r, P, gone=i32([[16, 64], [16, 64], [16, 64], [0, 0]]))
    status = i32([9] * 4)
    B.as_pages_trim(i32([40, 48, 70, 40]), t, n, r, P, lane_status=status)
    assert status.tolist() == [0] * 4 and n.tolist() == [40, 48, 70, 40]
    held = (t.clone(), n.clone(), r.clone())
    B.as_pages_grow(i32([5, 0, 0, 0]), t, n, r, P, lane_status=status)
    assert status.tolist() == [B.ERR_INVALID_ARG, 0, 0, 0]
    assert all(torch.equal(a, b) for a, b in zip(held, (t, n, r)))
    B.as_pages_grow(i32([0, 5, 5, 10]), t, n, r, P, lane_status=status)
    assert status.tolist() == [0] * 4 and n.tolist() == [40, 53, 75, 50]
    B.as_pages_trim(i32([32, 53, 75, 50]), t, n, r, P)
    B.as_pages_grow(i32([20, 1, 1, 1]), t, n, r, P, lane_status=status)
    assert status.tolist() == [0] * 4 and n.tolist() == [52, 54, 76, 51]
    # every token that came in by growing has a page, and the counts are right
    for i, (a, b) in enumerate(((32, 52), (48, 54), (70, 76), (40, 51))):
        assert all(int(t[i, p // P]) >= 0 for p in range(a, b))
    assert torch.equal(torch.bincount(t[t >= 0].long(), minlength=40).int(), r)
