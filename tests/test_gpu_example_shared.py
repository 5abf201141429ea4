"""The example's decode with the prompts' pages read once for their lanes, against the same decode without that hint."""
import importlib.util
import os

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


@pytest.mark.parametrize("N,lengths,dtype", [(4, [70], "f32"), (6, [37, 100, 1, 50], "f32"), (40, [130, 65], "f32"), (16, [90, 33], "bf16")])
def test_the_hint_changes_no_logit(ex, monkeypatch, N, lengths, dtype):
    """The same codes decoded lane by lane: attention's N and shared beginnings taken away.  Each step's logits agree while a
    lane's tokens so far are the same (off by about 1e-5 in 32 bits, by less than 0.05 where a stored code falls on the other side of
    a half).  The first two tokens are the same in 32 bits; later ones need not be: a step divides the code's difference by the token's
    probability, so that 1e-6 of a logit is a different token after four or five steps."""
    lm = ex.TinyLM(V=200, seed=9, dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
    g = torch.Generator().manual_seed(8)
    prompts = [torch.randint(1, lm.V, (n,), generator=g).tolist() for n in lengths]
    hints = []
    attend = ex.B.as_cache4_attend

    def watched(*a, **k):
        hints.append((k.get("N", 1), k.get("shared")))
        return attend(*a, **k)

    def alone(*a, **k):
        return attend(*a, **{**k, "N": 1, "shared": None})
    monkeypatch.setattr(ex.B, "as_cache4_attend", watched)
    together, st = ex.decode(lm, prompts, N, 0.2, 8, keep_logits=True)
    assert any(n == N and s is not None and int(s.max()) > 0 for n, s in hints)      # (the hint was there to be taken away)
    monkeypatch.setattr(ex.B, "as_cache4_attend", alone)
    apart, sa = ex.decode(lm, prompts, N, 0.2, 8, keep_logits=True)
    if dtype == "f32":
        assert all(a[:lengths[i // N] + 2] == b[:lengths[i // N] + 2] for i, (a, b) in enumerate(zip(together, apart)))
    compared = 0
    for step, ((x, ax), (y, ay)) in enumerate(zip(st["logits"], sa["logits"])):
        for i in range(len(prompts) * N):
            n = lengths[i // N] + step
            if bool(ax[i]) and bool(ay[i]) and together[i][:n] == apart[i][:n] and len(together[i]) > n - 1:
                # (bf16: each of two layers rounds its activations, of size about 3, to 8 bits)
                assert (x[i].double() - y[i].double()).abs().max() < (0.05 if dtype == "f32" else 0.25)
                compared += 1
    assert compared >= len(prompts) * N
    # other codes decode to other tokens: the comparison above can fail
    assert ex.decode(lm, prompts, N, 0.7, 8)[0] != together
