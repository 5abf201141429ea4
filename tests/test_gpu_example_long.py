"""The example that decodes with drafts over bounded caches: a run of windowed attention, weights, eviction, trim and verification
together, against plain code."""
import importlib.util
import math
import os

import pytest

torch = pytest.importorskip("torch")
from tests import test_gpu_verify as V  # noqa: E402
from tests.test_gpu_cache4 import quantise  # noqa: E402

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("decode_long", os.path.join(ROOT, "examples", "decode_long.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain_logits(lm, tokens, window, sinks):
    """float64 logits after every token of one sequence, keys and values quantised as the cache holds them."""
    x = lm.emb[torch.tensor(tokens, device="cuda")].double().cpu()
    n, g = len(tokens), lm.Hq // lm.H
    at = torch.arange(n)
    hidden = at > at.view(-1, 1)
    if window:
        hidden |= (at <= at.view(-1, 1) - window) & (at >= sinks)
    for i in range(lm.layers):
        qkv = (x @ lm.qkv[i].double().cpu()).view(n, lm.Hq + 2 * lm.H, lm.D)
        k, v = (torch.from_numpy(quantise(qkv[:, a:b].float().numpy(), 1.0)[0]).double() for a, b in ((lm.Hq, lm.Hq + lm.H), (lm.Hq + lm.H, lm.Hq + 2 * lm.H)))
        s = torch.einsum("qhd,khd->hqk", qkv[:, :lm.Hq], k.repeat_interleave(g, 1)) / math.sqrt(lm.D)
        s = s.masked_fill(hidden, -math.inf)
        x = x + torch.einsum("hqk,khd->qhd", torch.softmax(s, -1), v.repeat_interleave(g, 1)).reshape(n, -1) @ lm.out[i].double().cpu()
    return x @ lm.head.double().cpu()


def held(st):
    t = st["table"]
    return torch.bincount(t[t >= 0].long(), minlength=st["ref"].numel()).int()


@pytest.mark.parametrize("window,sinks,top_p", [(None, 0, 1.0), (24, 3, 0.9)])
def test_drafted_decode_against_plain_model(ex, window, sinks, top_p):
    lm = ex.LongLM(V=200, seed=3)
    bigram = (lm.emb @ lm.head).contiguous()
    g = torch.Generator().manual_seed(5)
    prompts = [torch.randint(1, lm.V, (n,), generator=g).tolist() for n in (37, 1, 16, 50)]
    N, K, trace = 3, 3, []
    seqs, st = ex.decode(lm, bigram, prompts, N, 0.41, 12, K, window=window, sinks=sinks, top_p=top_p, trace=trace)
    assert torch.equal(held(st), st["ref"])
    done = [len(prompts[i // N]) for i in range(len(seqs))]
    whole = [plain_logits(lm, s, window, sinks) for s in seqs]
    near = 0
    for logits, draft, drafted, u, codes, tokens, accepted, after in trace:
        for lane in range(len(seqs)):
            n = int(accepted[lane])
            # what the model says after the tokens that were accepted is what plain code says.  The calls differ from it by about 1e-6 in a
            # score; a value next to a border between two codes may round to the other one, a step of at most 1/4 of it, in one of
            # some thousand values: most logits agree to 1e-3, few miss 0.05.
            diff = (logits[lane, :n + 1].double().cpu() - whole[lane][done[lane] - 1:done[lane] + n]).abs()
            assert float(diff.max()) < 1.0
            near += int((diff.amax(1) < 0.05).sum())
            # verification, on the logits that it was given
            want = V.verify(logits[lane].float().cpu().numpy(), draft[lane].float().cpu().numpy(), drafted[lane].tolist(), K, u[lane].tolist(), float(codes[lane]), 1.0, 0, top_p)
            if want[3] > 1e-9:
                assert tokens[lane].tolist() == want[0] + [-1] * (K - want[1]) and n == want[1]
            assert seqs[lane][done[lane]:done[lane] + n + 1] == tokens[lane, :n + 1].tolist()
            done[lane] += n + 1
    assert near > 0.9 * sum(done[i] - len(prompts[i // N]) for i in range(len(seqs)))
    # the cache holds all but the last token, less what the window has left behind
    assert st["length"].tolist() == [len(s) - 1 for s in seqs]
    if window:
        P = 16
        first = -(-sinks // P)
        for row, n in zip(st["table"].tolist(), st["length"].tolist()):
            for m in range(len(row)):
                gone = m * P >= n or (first <= m and (m + 1) * P <= n + 1 - window)
                assert (row[m] == -1) == gone


def test_a_cut_prompt(ex):
    """keep below the prompts' lengths: lanes share the cut prompt's pages, lengths and reference counts are right; keep above them
    changes nothing."""
    lm = ex.LongLM(V=200, seed=4)
    bigram = (lm.emb @ lm.head).contiguous()
    g = torch.Generator().manual_seed(6)
    prompts = [torch.randint(1, lm.V, (n,), generator=g).tolist() for n in (90, 20, 133)]
    a, sa = ex.decode(lm, bigram, prompts, 2, 0.2, 6)
    b, sb = ex.decode(lm, bigram, prompts, 2, 0.2, 6, keep=200)
    assert a == b and torch.equal(sa["length"], sb["length"])
    c, sc = ex.decode(lm, bigram, prompts, 2, 0.2, 6, keep=48)
    assert torch.equal(held(sc), sc["ref"])
    for lane, s in enumerate(c):
        n = len(prompts[lane // 2])
        assert int(sc["length"][lane]) == len(s) - n + min(48, n - 1) and all(0 <= t < lm.V for t in s)
        assert (sc["table"][lane, :3].tolist() == sc["table"][lane ^ 1, :3].tolist()) == (min(48, n - 1) >= 48)
