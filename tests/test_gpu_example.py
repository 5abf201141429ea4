"""The example that decodes prompts through pages, the 4-bit cache, attention, logit edits and the step, against plain code."""
import importlib.util
import math
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("decode_prompts", os.path.join(ROOT, "examples", "decode_prompts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain_logits(ex, lm, tokens):
    """float64 logits after every token of one sequence, keys and values quantised as the cache holds them."""
    from test_gpu_cache4 import quantise
    x = lm.emb[torch.tensor(tokens, device="cuda")].double().cpu()
    n, g = len(tokens), lm.Hq // lm.H
    for i in range(lm.layers):
        qkv = (x @ lm.qkv[i].double().cpu()).view(n, lm.Hq + 2 * lm.H, lm.D)
        k, v = (torch.from_numpy(quantise(qkv[:, a:b].float().numpy(), 1.0)[0]).double() for a, b in ((lm.Hq, lm.Hq + lm.H), (lm.Hq + lm.H, lm.Hq + 2 * lm.H)))
        k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
        s = torch.einsum("qhd,khd->hqk", qkv[:, :lm.Hq], k) / math.sqrt(lm.D)
        s = s.masked_fill(torch.ones(n, n).triu(1).bool(), -math.inf)
        x = x + torch.einsum("hqk,khd->qhd", torch.softmax(s, -1), v).reshape(n, -1) @ lm.out[i].double().cpu()
    return x @ lm.head.double().cpu()


def test_decode_against_plain_model(ex, monkeypatch):
    monkeypatch.syspath_prepend(os.path.join(ROOT, "tests"))
    lm = ex.TinyLM(V=300, seed=3)
    lm.head[:, ex.EOS] += 0.02 * lm.head.abs().mean()
    g = torch.Generator().manual_seed(5)
    prompts = [torch.randint(1, lm.V, (n,), generator=g).tolist() for n in (37, 1, 16, 50)]
    words = -(-lm.V // 32)
    even, odd = np.zeros(words * 32, bool), np.zeros(words * 32, bool)
    even[1:lm.V:2] = odd[0:lm.V:2] = True                   # odd and even tokens alternate; EOS follows an odd one
    mask = torch.from_numpy(np.stack([np.packbits(b, bitorder="little").view(np.int32) for b in (even, odd)])).cuda()
    N = 6
    seqs, st = ex.decode(lm, prompts, N, 0.41, 30, mask=mask, keep_logits=True)
    ref = np.zeros(st["ref"].numel(), dtype=np.int64)
    table, length = st["table"].cpu().numpy(), st["length"].cpu().numpy()
    for row, n in zip(table, length):
        for p in row[:-(-int(n) // 16)]:
            ref[p] += 1
    assert np.array_equal(ref, st["ref"].cpu().numpy())     # every page is held by as many lanes as its count says
    checked = 0
    for lane, s in enumerate(seqs):
        p = prompts[lane // N]
        assert s[:len(p)] == p and len(s) > len(p)
        for a, b in zip(s[len(p) - 1:], s[len(p):]):
            assert (a + b) % 2 == 1                         # the grammar
        assert ex.EOS not in s[len(p):-1]
        want = plain_logits(ex, lm, s)
        for step, (logits, alive) in enumerate(st["logits"]):
            at = len(p) - 1 + step
            if at < len(s) - 1 and bool(alive[lane]):
                # one code off by a step of its grid (a sixth of a value) moves a logit by far less than this
                assert (logits[lane].double().cpu() - want[at]).abs().max() < 0.05
                checked += 1
    assert checked > 100


def test_sharing_changes_nothing(ex):
    """The lanes of a prompt decoded together and one by one: the same tokens (codes a lattice apart leave room)."""
    lm = ex.TinyLM(V=200, seed=9, dtype=torch.float32)
    g = torch.Generator().manual_seed(8)
    prompts = [torch.randint(1, lm.V, (70,), generator=g).tolist()]
    together, _ = ex.decode(lm, prompts, 4, 0.2, 6)
    alone, _ = ex.decode(lm, prompts * 4, 1, 0.0, 6)
    assert len(together) == len(alone) == 4 and all(len(s) > 70 for s in together)
    codes_same, _ = ex.decode(lm, prompts, 4, 0.2, 6)
    assert together == codes_same
