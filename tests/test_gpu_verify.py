"""The step over drafted tokens against a plain implementation in 64 bits, and against as_step."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ONE_BELOW = 1.0 - 2.0 ** -53


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import binding
    return binding


def probabilities(x, temp, top_k, top_p):
    """float64 probabilities of a row of logits."""
    x = x.astype(np.float64)
    order = np.argsort(-x, kind="stable")
    order = order[np.isfinite(x[order])]
    if top_k > 0:
        order = order[:top_k]
    e = np.exp((x[order] - x[order[0]]) / temp)
    if 0 < top_p < 1:
        upto = np.cumsum(e)
        m = int(np.searchsorted(upto, top_p * upto[-1])) + 1
        order, e = order[:m], e[:m]
    p = np.zeros(x.shape)
    p[order] = e / math.fsum(e)
    return p


def verify(target, draft, drafted, n, u, c, temp, top_k, top_p):
    """(tokens, accepted, code, how near the nearest decision or interval end was, probability of the last token, the mass that it was
    taken from) of one lane."""
    near, tokens = 1.0, []
    for i in range(n + 1):
        p = rest = probabilities(target[i], temp, top_k, top_p)
        if i == n:
            break
        x = drafted[i]
        q = np.zeros_like(p)
        if draft is None:
            q[x] = 1.0
        else:
            q = probabilities(draft[i], temp, top_k, top_p)
        near = min(near, abs(u[i] * q[x] - p[x]) / max(p[x], u[i] * q[x], 1e-300)) if p[x] or u[i] * q[x] else near
        if not u[i] * q[x] < p[x]:
            rest = np.maximum(p - q, 0.0)
            if not rest.any():
                rest = p
            break
        tokens.append(x)
    mass = math.fsum(rest)
    rest = rest / mass
    upto = np.cumsum(rest)
    c = min(c, ONE_BELOW)
    at = min(int(np.searchsorted(upto, c, side="right")), int(np.flatnonzero(rest)[-1]))
    low = upto[at] - rest[at]
    near = min(near, abs(c - low) if at > np.flatnonzero(rest)[0] else 1.0, abs(upto[at] - c) if at < np.flatnonzero(rest)[-1] else 1.0)
    code = min(max((c - low) / rest[at], 0.0), ONE_BELOW)
    return tokens + [at], len(tokens), code, near, rest[at], mass


def inputs(lanes, K, V, dtype, seed, spread=2.0, alike=0.7):
    gen = torch.Generator().manual_seed(seed)
    target = torch.randn(lanes, K + 1, V, generator=gen) * spread
    draft = target[:, :K] + alike * torch.randn(lanes, K, V, generator=gen)
    target, draft = target.to(DT[dtype]), draft.to(DT[dtype])
    noise = -torch.log(-torch.log(torch.rand(lanes, K, V, generator=gen).clamp(1e-9, 1 - 1e-7)))
    drafted = (draft.float() + noise).argmax(-1).int()
    u = torch.rand(lanes, K, generator=gen, dtype=torch.float64)
    codes = (torch.arange(lanes, dtype=torch.float64) + 0.37) / lanes
    return target, draft, drafted, u, codes


def check(B, target, draft, drafted, u, codes, temp, top_k, top_p, n=None, **kw):
    lanes, K = drafted.shape
    status = torch.full((lanes,), 9, dtype=torch.int32, device="cuda")
    tokens, accepted, out = B.as_step_verify(target.cuda(), None if draft is None else draft.cuda(), drafted.cuda(), u.cuda(), codes.cuda(), temp, top_k, top_p,
                                             n_drafts=None if n is None else torch.tensor(n, dtype=torch.int32).cuda(), lane_status=status, **kw)
    assert (status == 0).all()
    tokens, accepted, out = tokens.cpu(), accepted.cpu(), out.cpu()
    V = kw.get("V", target.shape[2])
    t64, d64 = target.float().numpy()[:, :, :V], None if draft is None else draft.float().numpy()[:, :, :V]
    for i in range(lanes):
        m = K if n is None else n[i]
        want, a, code, near, p, mass = verify(t64[i], None if draft is None else d64[i], drafted[i].tolist(), m, u[i].tolist(), float(codes[i]), temp, top_k, top_p)
        # Probabilities p, q and their sums are within 1e-13 of the formula's, relative to themselves, on both sides.  A difference
        # p - q is then off by 1e-13 (p + q), a sum of them by 2e-13, and divided by the mass of max(p - q, 0), the sum of all, by
        # 2e-13 / mass: so are the interval's ends, and the code, between them, by twice that over the interval's length p.
        if near < 1e-11 / mass:
            continue
        assert int(accepted[i]) == a and tokens[i].tolist() == want + [-1] * (K - a)
        assert abs(float(out[i]) - code) <= 1e-12 / (p * mass)


CUTS = [(1.0, 0, 1.0), (0.7, 0, 0.9), (1.3, 40, 1.0), (0.9, 30, 0.8), (1.0, 1, 1.0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temp,top_k,top_p", CUTS)
@pytest.mark.parametrize("lanes,K,V", [(5, 3, 1), (7, 2, 2), (40, 4, 33), (33, 1, 1000), (9, 8, 4099), (3, 40, 257), (6, 3, 50257)])
def test_against_the_formula(B, dtype, temp, top_k, top_p, lanes, K, V):
    target, draft, drafted, u, codes = inputs(lanes, K, V, dtype, V + K)
    check(B, target, draft, drafted, u, codes, temp, top_k, top_p)
    check(B, target, None, drafted, u, codes, temp, top_k, top_p, n=[(3 * i) % (K + 1) for i in range(lanes)])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top_k,top_p", [(0, 1.0), (0, 0.9)])
def test_strides_and_ragged_drafts(B, dtype, top_k, top_p):
    lanes, K, V, wide = 12, 3, 1003, 1021
    target, draft, drafted, u, codes = inputs(lanes, K, wide, dtype, 5)
    drafted = drafted % V
    n = [i % (K + 1) for i in range(lanes)]
    # rows behind a lane's last draft do not count, whatever they hold
    for i in range(lanes):
        target[i, n[i] + 1:] = float("nan")
        draft[i, n[i]:] = float("inf")
        drafted[i, n[i]:] = 1 << 30
        u[i, n[i]:] = float("nan")
    check(B, target, draft, drafted, u, codes, 0.8, top_k, top_p, n=n, V=V)
    # cut out of wider rows at an odd place
    flat = torch.zeros(lanes, (K + 1), wide + 7).to(DT[dtype])
    flat[:, :, 3:3 + wide] = target
    got = B.as_step_verify(flat.cuda()[:, :, 3:3 + V], draft.cuda()[:, :, :V], drafted.cuda(), u.cuda(), codes.cuda(), 0.8, top_k, top_p,
                           n_drafts=torch.tensor(n, dtype=torch.int32).cuda())
    want = B.as_step_verify(target.cuda(), draft.cuda(), drafted.cuda(), u.cuda(), codes.cuda(), 0.8, top_k, top_p, n_drafts=torch.tensor(n, dtype=torch.int32).cuda(), V=V)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert (got[2] - want[2]).abs().max() < 1e-9    # (chunks start elsewhere: sums differ in their last bits)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top_k,top_p", [(0, 1.0), (5, 1.0), (0, 0.9)])
def test_ties_and_masked_tokens(B, dtype, top_k, top_p):
    """Logits of a few values only, -inf among them."""
    gen = torch.Generator().manual_seed(3)
    lanes, K, V = 64, 3, 300
    target = torch.randint(-2, 3, (lanes, K + 1, V), generator=gen).float()
    draft = torch.randint(-2, 3, (lanes, K, V), generator=gen).float()
    target[torch.rand(target.shape, generator=gen) < 0.3] = -math.inf
    draft[torch.rand(draft.shape, generator=gen) < 0.3] = -math.inf
    drafted = torch.randint(0, V, (lanes, K), generator=gen).int()
    u = torch.rand(lanes, K, generator=gen, dtype=torch.float64)
    codes = torch.rand(lanes, generator=gen, dtype=torch.float64)
    check(B, target.to(DT[dtype]), draft.to(DT[dtype]), drafted, u, codes, 1.0, top_k, top_p)
    # drafted tokens that the target masks are never accepted, u = 0 included; those it keeps always are then
    u[:] = 0
    tokens, accepted, _ = B.as_step_verify(target.to(DT[dtype]).cuda(), draft.to(DT[dtype]).cuda(), drafted.cuda(), u.cuda(), codes.cuda(), 1.0)
    ok = torch.isfinite(target[:, :K].gather(2, drafted.long().unsqueeze(2)).squeeze(2))
    assert torch.equal(accepted.cpu(), ok.int().cumprod(1).sum(1).int())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_draft_equal_to_target(B, dtype):
    """p = q: u < 1 accepts everything, and the last token is as_step's."""
    lanes, K, V = 20, 4, 5000
    target, _, drafted, u, codes = inputs(lanes, K, V, dtype, 8)
    t = target.cuda()
    tokens, accepted, out = B.as_step_verify(t, t[:, :K].contiguous(), drafted.cuda(), u.cuda(), codes.cuda(), 0.9)
    assert (accepted == K).all() and torch.equal(tokens[:, :K].cpu(), drafted)
    want, wcode = B.as_step(t[:, K].contiguous(), codes.cuda(), 0.9)
    assert torch.equal(tokens[:, K], want) and (out - wcode).abs().max() < 1e-9
    # no drafts at all: the step itself
    one = t[:, :1].contiguous()
    tokens, accepted, out = B.as_step_verify(one, None, drafted[:, :0].cuda(), u[:, :0].contiguous().cuda(), codes.cuda(), 0.9, 0, 0.95)
    want, wcode = B.as_step(one[:, 0].contiguous(), codes.cuda(), 0.9, 0, 0.95)
    assert not accepted.any() and torch.equal(tokens[:, 0], want) and (out - wcode).abs().max() < 1e-9


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decisions_next_to_their_border(B, dtype):
    """u q(x) one part in 10^9 above and below p(x): finer than 32 bits resolve."""
    lanes, K, V = 64, 1, 3001
    target, draft, drafted, u, codes = inputs(lanes, K, V, dtype, 9)
    t, d = target.float().numpy(), draft.float().numpy()
    want = []
    for i in range(lanes):
        x = int(drafted[i, 0])
        p, q = probabilities(t[i, 0], 0.9, 0, 1.0)[x], probabilities(d[i, 0], 0.9, 0, 1.0)[x]
        if p >= q:                                  # swap the two: the border has to be below 1
            target[i, 0], draft[i, 0] = draft[i, 0].clone(), target[i, 0].clone()
            p, q = q, p
        u[i, 0] = p / q * (1 + (1e-9 if i % 2 else -1e-9))
        want.append(0 if i % 2 else 1)
    _, accepted, _ = B.as_step_verify(target.cuda(), draft.cuda(), drafted.cuda(), u.cuda(), codes.cuda(), 0.9)
    assert accepted.tolist() == want


def test_a_very_small_residual_and_none(B):
    """p and q alike but for one token; a draft with all its mass on one token."""
    V = 1000
    x = torch.randn(1, 2, V, generator=torch.Generator().manual_seed(1))
    q = x[:, :1].clone()
    q[0, 0, 700] += 1e-3                            # the draft likes 700 a little more: refused there, the rest is spread over all others
    drafted = torch.tensor([[700]], dtype=torch.int32)
    for c in (0.0, 0.5, 0.999999, 1.0):
        check(B, x, q, drafted, torch.tensor([[1 - 2.0 ** -53]], dtype=torch.float64), torch.tensor([c], dtype=torch.float64), 1.0, 0, 1.0)
    # the draft has all its mass on one token
    q[:] = -math.inf
    q[0, 0, 3] = 0.0
    for c in (0.0, 0.25, 1.0):
        check(B, x, q, torch.tensor([[3]], dtype=torch.int32), torch.tensor([[0.999]], dtype=torch.float64), torch.tensor([c], dtype=torch.float64), 1.0, 0, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top_p", [1.0, 0.9])
def test_lane_errors(B, dtype, top_p):
    lanes, K, V = 14, 2, 600
    target, draft, drafted, u, codes = inputs(lanes, K, V, dtype, 4)
    u[:] = 0.0                                      # everything is accepted that the cut leaves
    n = [K] * lanes
    good = B.as_step_verify(target.cuda(), draft.cuda(), drafted.cuda(), u.cuda(), codes.cuda(), 1.0, 0, top_p)
    target[1, 0, 5] = math.nan
    target[2, 1, 5] = math.inf
    target[3, 2] = -math.inf
    draft[4, 1, 9] = math.nan
    drafted[5, 1] = V
    drafted[6, 0] = -1
    u[7, 0] = 1.0
    u[8, 1] = math.nan
    codes[9] = -0.1
    codes[10] = math.nan
    n[11] = K + 1
    n[12] = -1
    status = torch.full((lanes,), 9, dtype=torch.int32, device="cuda")
    tokens, accepted, out = B.as_step_verify(target.cuda(), draft.cuda(), drafted.cuda(), u.cuda(), codes.cuda(), 1.0, 0, top_p,
                                             n_drafts=torch.tensor(n, dtype=torch.int32).cuda(), lane_status=status)
    N, I = B.ERR_NUMERIC, B.ERR_INVALID_ARG
    # (what is broken counts if the lane gets as far as its place)
    place = {1: 0, 2: 1, 3: 2, 4: 1, 5: 1, 6: 0, 7: 0, 8: 1, 9: 0, 10: 0, 11: 0, 12: 0}
    code = [0, N, N, N, N, I, I, N, N, N, N, I, I, 0]
    want = [c if i in place and place[i] <= int(good[1][i]) else 0 for i, c in enumerate(code)]
    assert status.tolist() == want and (top_p < 1 or want == code)
    for i in range(lanes):
        if want[i] == 0:
            assert torch.equal(tokens[i], good[0][i]) and int(accepted[i]) == int(good[1][i]) and float(out[i]) == float(good[2][i])
        else:
            assert (tokens[i] == -1).all() and int(accepted[i]) == 0
            assert float(out[i]) == float(codes[i]) or math.isnan(float(codes[i]))
    # behind a refusal none of it counts
    target, draft, drafted, u, codes = inputs(lanes, K, V, dtype, 4)
    target[:, 0] = target[:, 0].scatter(1, drafted[:, :1].long(), -math.inf)
    target[:, 1:] = math.nan
    draft[:, 1:] = math.nan
    drafted[:, 1] = -7
    u[:, 1] = math.nan
    tokens, accepted, out = B.as_step_verify(target.cuda(), draft.cuda(), drafted.cuda(), u.cuda(), codes.cuda(), 1.0, 0, top_p, lane_status=status)
    assert not status.any() and not accepted.any() and (tokens[:, 0] >= 0).all() and (tokens[:, 1:] == -1).all()


def test_tokens_are_distributed_as_the_targets(B):
    """Drafts drawn from q, verified: the first token's frequencies are p's (a chi-square of 7 degrees of freedom)."""
    gen = torch.Generator().manual_seed(12)
    lanes, V = 40000, 8
    p, q = torch.randn(V, generator=gen) * 1.5, torch.randn(V, generator=gen)
    drafted = torch.multinomial(torch.softmax(q, 0), lanes, replacement=True, generator=gen).int().view(lanes, 1)
    u, codes = torch.rand(lanes, 1, generator=gen, dtype=torch.float64), torch.rand(lanes, generator=gen, dtype=torch.float64)
    target = p.expand(lanes, 2, V).contiguous()
    tokens, accepted, _ = B.as_step_verify(target.cuda(), q.expand(lanes, 1, V).contiguous().cuda(), drafted.cuda(), u.cuda(), codes.cuda(), 1.0)
    got = torch.bincount(tokens[:, 0].cpu().long(), minlength=V).double()
    want = torch.softmax(p.double(), 0) * lanes
    assert float(((got - want) ** 2 / want).sum()) < 24.3       # 0.001 of such draws lie above
    share = float(torch.minimum(torch.softmax(p, 0), torch.softmax(q, 0)).sum())
    assert abs(float((accepted > 0).double().mean()) - share) < 4 * math.sqrt(share * (1 - share) / lanes)


def deep_rows(V, dtype, temp, bits, place, margin=4096):
    """(a row of V logits inside a larger buffer of large ones, first and last token that are likely): the tokens of a stretch of several hundred
    have 2^-bits of the likeliest one's probability."""
    buffer = torch.full((V + 2 * margin,), 50.0)
    row = buffer[margin:margin + V]
    row.copy_(torch.linspace(-2.0, 0.0, V) * temp)
    n = V // 3
    row[:n] = row[V - n:] = float(-bits * math.log(2) * temp)
    if place == "front":
        row[V - n:] = -temp
    if place == "end":
        row[:n] = -temp
    likely = (row > -100 * temp).nonzero().flatten()
    return buffer.to(DT[dtype]).cuda()[margin:margin + V], int(likely[0]), int(likely[-1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temp", [1.0, 0.02])
@pytest.mark.parametrize("V", [900, 4099, 50257])
@pytest.mark.parametrize("place", ["front", "end", "both"])
def test_chunks_of_tokens_next_to_nothing(B, dtype, temp, V, place):
    """Chunks whose tokens are so unlikely that some of them count as impossible, with codes that lie at the intervals' very ends."""
    for bits in (930, 945, 949, 951, 953, 955, 957, 960, 965, 970, 975, 979, 981, 985, 990, 999, 1005, 1030):
        row, low, high = deep_rows(V, dtype, temp, bits, place)
        for code in (0.0, 1.0, ONE_BELOW):
            codes = torch.tensor([code], dtype=torch.float64, device="cuda")
            status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
            none = torch.empty(1, 0, dtype=torch.int32, device="cuda")
            u = torch.tensor([[ONE_BELOW]], dtype=torch.float64, device="cuda")
            got = [B.as_step_verify(row.view(1, 1, V), None, none, u[:, :0], codes, temp, lane_status=status)]
            # a likely token is looked up and refused; one is drawn and refused: q has no token but it, or the stretch as well, less likely still
            x = torch.tensor([[(low + high) // 2]], dtype=torch.int32, device="cuda")
            two = row.view(1, 1, V).expand(1, 2, V).contiguous()
            got.append(B.as_step_verify(two, None, x, u, codes, temp))
            for other in (float("-inf"), float(-(bits + 20) * math.log(2) * temp)):
                q = torch.full((1, 1, V), other, device="cuda")
                q[0, 0, int(x)] = 0.0
                got.append(B.as_step_verify(two, q.to(DT[dtype]), x, u, codes, temp))
            assert int(status[0]) == 0
            for tokens, accepted, out in got:
                token = int(tokens[0, 0])
                # (a token less likely than 2^-950 may count as impossible or not)
                assert int(accepted[0]) == 0 and (0 <= token <= low if code == 0.0 else high <= token < V) and 0.0 <= float(out[0]) < 1.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temp", [0.3, 1.0, 40.0])
@pytest.mark.parametrize("mask", ["lowest", -1e30, -1e10, -1e9, -1e5])
@pytest.mark.parametrize("lanes,V", [(40, 17), (20, 1000), (5, 50257), (500, 3000)])
def test_tokens_masked_by_finite_numbers(B, dtype, temp, mask, lanes, V):
    """Single tokens and whole stretches, so that threads see nothing else; the target's masks, the draft's, both."""
    K = 2
    target, draft, drafted, u, codes = inputs(lanes, K, V, dtype, 31)
    low = torch.finfo(DT[dtype]).min if mask == "lowest" else mask
    gen = torch.Generator().manual_seed(4)
    for rows in (target, draft):
        masked = torch.rand(rows.shape, generator=gen) < 0.3
        masked |= torch.rand(rows.shape[0], rows.shape[1], -(-V // 16), generator=gen).lt(0.4).repeat_interleave(16, 2)[:, :, :V]
        masked[torch.rand(rows.shape[:2], generator=gen) < 0.3] = False
        masked[:, :, V // 2] = False
        rows[masked] = low
    some = slice(0, 40)
    check(B, target[some], draft[some], drafted[some], u[some], codes[some], temp, 0, 1.0)
    check(B, target[some], None, drafted[some], u[some], codes[some], temp, 0, 1.0)
    check(B, target[some], draft[some], drafted[some], u[some], codes[some], temp, 0, 0.9)
    # many lanes at a time, a thread block to each, decide as few do
    few = B.as_step_verify(target[some].cuda(), draft[some].cuda(), drafted[some].cuda(), u[some].cuda(), codes[some].cuda(), temp)
    many = B.as_step_verify(target.cuda(), draft.cuda(), drafted.cuda(), u.cuda(), codes.cuda(), temp)
    assert torch.equal(few[0], many[0][some]) and torch.equal(few[1], many[1][some])
