"""Eviction from the 4-bit cache against a plain model on lists of tokens: exact equality."""
import random

import pytest

torch = pytest.importorskip("torch")
from tests import test_gpu_cache4 as C  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import binding
    return binding


def tokens(pages, table, lane, head, n):
    """[n, 18 D / 16] bytes: what is stored of the lane's tokens."""
    D, P = pages.shape[3] // 18, pages.shape[2] * 16
    t = pages[table[lane, :-(-n // P)].long(), head].view(-1, 18 * D)
    kb, vb, ks, vs = t.split([8 * D, 8 * D, D, D], 1)
    m = t.shape[0]
    rows = torch.cat([kb.reshape(m, 16, D // 2), vb.reshape(m, D // 16, 16, 8).transpose(1, 2).reshape(m, 16, D // 2), ks.reshape(m, 16, D // 16),
                      vs.reshape(m, D // 16, 16).transpose(1, 2)], 2)
    return rows.reshape(m * 16, -1)[:n]


def model(w, n, keep, first, recent):
    """For each of the lane's places the position that its token comes from, and the weights afterwards (w: floats of one head)."""
    if n <= keep:
        return list(range(n)), list(w)
    middle = range(first, n - recent)
    order = sorted(middle, key=lambda t: (w[t] != w[t], -w[t] if w[t] == w[t] else 0.0, t))
    stay = set(order[:keep - first - recent])
    end = keep - recent
    src = list(range(n))
    for hole, mover in zip([t for t in range(first, end) if t not in stay], [t for t in middle if t in stay and t >= end]):
        src[hole] = mover
    for t in range(end, keep):
        src[t] = t + n - keep
    return src, [w[src[t]] if t < keep else 0.0 for t in range(n)] + list(w[n:])


def run(B, lens, keeps, firsts, recent, H, D, P, weight, in_place, seed=1, ref=None):
    pages, table, _, _ = C.filled(B, lens, H, D, P, seed, None, None)
    before = pages.clone()
    w = weight.cuda()
    out = w if in_place else torch.full_like(w, 77.0)
    status = C.i32([9] * len(lens))
    got = B.as_cache4_evict(pages, w, table, C.i32(lens), C.i32(keeps), recent, first=None if firsts is None else C.i32(firsts),
                            weight_out=None if in_place else out, lane_status=status, ref=ref)
    assert got.data_ptr() == out.data_ptr() and (in_place or torch.equal(w.cpu().view(torch.int32), weight.view(torch.int32)))
    return before.cpu(), pages.cpu(), table.cpu(), got.cpu(), status.tolist()


CASES = [  # lens, keep, first, recent, H, D, P
    ([1, 2, 3], 1, 0, 1, 1, 64, 16), ([40, 17, 16, 15], 16, 2, 3, 2, 64, 16), ([100, 64, 65, 63], 64, 4, 20, 3, 128, 32), ([300, 1000], 250, 16, 100, 1, 128, 64),
    ([500], 499, 0, 0, 2, 64, 128), ([500], 20, 4, 16, 2, 128, 128), ([2200, 1800], 1000, 0, 1000, 1, 64, 16), ([9000], 4000, 10, 50, 1, 64, 64),
    ([70, 10], 0, 0, 0, 2, 64, 16), ([3000], 100, 0, 10, 2, 128, 16), ([2112, 2049], 2048, 4, 512, 2, 128, 64), ([6000], 5000, 0, 1, 1, 128, 128)]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("lens,keep,first,recent,H,D,P", CASES)
@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
def test_evict(B, kind, lens, keep, first, recent, H, D, P, in_place):
    gen = torch.Generator().manual_seed(len(lens) * 10 + keep)
    W = max(lens) + 3
    w = torch.exp(2 * torch.randn(len(lens), H, W, generator=gen))
    if kind == "ties":
        w = (w * 2).floor().clamp(max=5)
    if kind == "odd":
        r = torch.rand(w.shape, generator=gen)
        w = torch.where(r < 0.1, torch.zeros_like(w), w)
        w[(r > 0.1) & (r < 0.2)] = float("inf")
        w[(r > 0.2) & (r < 0.3)] = float("nan")
        w[(r > 0.3) & (r < 0.5)] *= -1
        w[(r > 0.5) & (r < 0.55)] = -0.0
        w[(r > 0.55) & (r < 0.6)] = float("-inf")
    before, pages, table, out, status = run(B, lens, [keep] * len(lens), [first] * len(lens), recent, H, D, P, w, in_place)
    assert status == [0] * len(lens)
    want = before.clone()
    for i, n in enumerate(lens):
        for h in range(H):
            src, wo = model(w[i, h].tolist(), n, keep, first, recent)
            old, new = tokens(before, table, i, h, n), tokens(pages, table, i, h, n)
            kept = min(n, keep)
            assert torch.equal(new[:kept], old[src[:kept]]) and torch.equal(new[kept:], old[kept:])
            same = torch.tensor(wo)
            assert torch.equal(torch.nan_to_num(out[i, h], 123.0), torch.nan_to_num(same, 123.0))
    held = torch.zeros(pages.shape[0], dtype=torch.bool)
    held[table[table >= 0].long()] = True
    assert torch.equal(pages[~held], want[~held])


def test_ragged_arguments(B):
    """Every lane with its own end and beginning; random shapes."""
    rng = random.Random(3)
    for trial in range(6):
        H, D, P = rng.choice((1, 3)), rng.choice((64, 128)), rng.choice((16, 64))
        lens = [rng.randint(0, 1500) for _ in range(7)]
        recent = rng.randint(0, 40)
        firsts = [rng.randint(0, 30) for _ in lens]
        keeps = [f + recent + rng.randint(0, 1200) for f in firsts]
        w = torch.rand(7, H, max(lens) + 1, generator=torch.Generator().manual_seed(trial))
        before, pages, table, out, status = run(B, lens, keeps, firsts, recent, H, D, P, w, trial % 2 == 0, seed=trial)
        assert status == [0] * 7
        for i, n in enumerate(lens):
            for h in range(H):
                src, wo = model(w[i, h].tolist(), n, keeps[i], firsts[i], recent)
                kept = min(n, keeps[i])
                assert torch.equal(tokens(pages, table, i, h, n)[:kept], tokens(before, table, i, h, n)[src[:kept]])
                assert torch.equal(out[i, h], torch.tensor(wo))


def test_refused_lanes_keep_what_they_have(B):
    H, D, P, n = 2, 64, 16, 100
    lens = [n] * 8
    pages, table, _, _ = C.filled(B, lens, H, D, P, 2, None, None)
    ref = torch.zeros(pages.shape[0], dtype=torch.int32, device="cuda")
    ref[table[table >= 0].long()] = 1
    ref[table[5, 2].long()] = 2                     # in front of the new end, behind the protected beginning
    ref[table[6, 0].long()] = 2                     # within the protected beginning: not written
    ref[table[7, 6].long()] = 2                     # behind the new end: not written
    w = torch.rand(8, H, 104, device="cuda")
    broken = table.clone()
    broken[4, 3] = 1 << 20
    before, w0, status = pages.clone(), w.clone(), C.i32([9] * 8)
    B.as_cache4_evict(pages, w, broken, C.i32([n, 105, n, n, n, n, n, n]), C.i32([-1, 60, 60, 20, 60, 60, 60, 60]), 10, first=C.i32([0, 0, -1, 16, 0, 0, 16, 0]),
                      ref=ref, lane_status=status)
    E = B.ERR_INVALID_ARG
    assert status.tolist() == [E, E, E, E, E, E, 0, 0]
    assert torch.equal(w[:6], w0[:6]) and not torch.equal(w[6], w0[6]) and not torch.equal(w[7], w0[7])
    mine = torch.unique(table[6:][table[6:] >= 0]).long()
    rest = torch.ones(pages.shape[0], dtype=torch.bool, device="cuda")
    rest[mine] = False
    assert torch.equal(pages[rest], before[rest]) and torch.equal(pages[table[6, 0].long()], before[table[6, 0].long()])
    assert torch.equal(pages[table[7, 6].long()], before[table[7, 6].long()])


def spoilt(w, kind, gen):
    """Weights with many equal ones, or with zeros, infinities, NaN and negative ones among them."""
    if kind == "ties":
        return (w * 2).floor().clamp(max=5)
    if kind == "odd":
        r = torch.rand(w.shape, generator=gen)
        w = torch.where(r < 0.1, torch.zeros_like(w), w)
        for lo, x in ((0.1, float("inf")), (0.2, float("nan")), (0.5, -0.0), (0.55, float("-inf"))):
            w[(r > lo) & (r < lo + 0.05)] = x
    return w


def compare(B, lens, keeps, firsts, recent, H, D, P, W, kind, in_place, lanes=None):
    """The call against the model, in these lanes (None: all); what no lane holds stays."""
    gen = torch.Generator().manual_seed(len(lens) + recent)
    w = spoilt(torch.exp(2 * torch.randn(len(lens), H, W, generator=gen)), kind, gen)
    before, pages, table, out, status = run(B, lens, keeps, firsts, recent, H, D, P, w, in_place)
    assert status == [0] * len(lens)
    for i in range(len(lens)) if lanes is None else lanes:
        n, kept = lens[i], min(lens[i], keeps[i])
        for h in range(H):
            src, wo = model(w[i, h].tolist(), n, keeps[i], firsts[i], recent)
            assert torch.equal(torch.nan_to_num(out[i, h], 123.0), torch.nan_to_num(torch.tensor(wo), 123.0))
            if n > 0:
                old, new = tokens(before, table, i, h, n), tokens(pages, table, i, h, n)
                assert torch.equal(new[:kept], old[src[:kept]]) and torch.equal(new[kept:], old[kept:])
    free = torch.ones(pages.shape[0], dtype=torch.bool)
    free[table[table >= 0].long()] = False
    assert torch.equal(pages[free], before[free])


def ragged(n, top, recent, seed):
    """(lengths, ends, beginnings) of n lanes: some shorter than they may be, some cut by one, some to next to nothing."""
    rng = random.Random(seed)
    lens = [rng.choice((0, 1, top, rng.randint(1, top))) for _ in range(n)]
    firsts = [rng.choice((0, rng.randint(0, 40))) for _ in lens]
    keeps = [f + recent + rng.choice((0, 1, max(0, m - f - recent - 1), rng.randint(0, top))) for f, m in zip(firsts, lens)]
    return lens, keeps, firsts


# More lanes and heads than SMs take small thread blocks if a lane's weights fit those, else large ones; half as many large ones; fewer clusters of them.
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
@pytest.mark.parametrize("lanes,H,D,P,top,recent", [(38, 4, 64, 16, 1500, 40), (80, 2, 128, 64, 700, 0), (310, 1, 64, 32, 130, 17), (200, 3, 128, 16, 90, 20), (75, 2, 64, 128, 8100, 500),
                                                    (30, 3, 128, 32, 1500, 33), (100, 1, 64, 16, 3000, 1000), (37, 4, 64, 64, 400, 0), (160, 1, 64, 64, 8500, 64)])
def test_many_lanes_and_heads(B, lanes, H, D, P, top, recent, kind, in_place):
    lens, keeps, firsts = ragged(lanes, top, recent, lanes)
    W = max(lens) + 2
    compare(B, lens, keeps, firsts, recent, H, D, P, W, kind, in_place, None if top <= 1500 else range(0, lanes, 9))


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
@pytest.mark.parametrize("lens,keeps,firsts,recent,H,D,P", [
    ([40000, 300], [20000, 100], [7, 3], 90, 1, 64, 64), ([50001], [1000], [0], 0, 2, 64, 128), ([37000, 36000, 40], [36999, 35000, 30], [100, 0, 2], 20, 1, 128, 16),
    ([60000], [30000], [16], 25000, 1, 64, 64),
    # (middles of 35549, 35550 and 35551 tokens)
    ([36000, 36001, 36002], [20000, 20000, 35000], [51, 51, 51], 400, 1, 64, 64)])
def test_middles_beyond_shared_memory(B, lens, keeps, firsts, recent, H, D, P, kind, in_place):
    """Weights that do not fit a thread block's shared memory are read again, while places among them are being filled."""
    compare(B, lens, keeps, firsts, recent, H, D, P, max(lens) + 5, kind, in_place)


@pytest.mark.parametrize("in_place", [True, False])
def test_a_long_middle_among_many_lanes(B, in_place):
    lens = [39000 if i == 41 else 37111 if i == 3 else 10 + 13 * i for i in range(80)]
    keeps = [20000 if i == 41 else 3000 if i == 3 else 5 + 12 * i for i in range(80)]
    compare(B, lens, keeps, [2] * 80, 3, 1, 64, 64, 39000, "ties", in_place)
