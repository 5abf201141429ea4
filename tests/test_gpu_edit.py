"""as_logits_edit against the formulas in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import binding
    return binding


def reference(x, seq=None, length=None, prompt=None, rep=1.0, pres=0.0, freq=0.0, bias=None, mask=None, row=None):
    y = x.double().cpu().clone()
    lanes, V = y.shape
    for i in range(lanes):
        if seq is not None:
            n = max(0, min(int(length[i]), seq.shape[1]))
            p = 0 if prompt is None else int(prompt[i])
            count, seen = {}, set()
            for j, t in enumerate(seq[i, :n].tolist()):
                if 0 <= t < V:
                    seen.add(t)
                    if j >= p:
                        count[t] = count.get(t, 0) + 1
            for t in seen:
                v = float(y[i, t])
                y[i, t] = v / rep if v > 0 else v * rep
            for t, c in count.items():
                y[i, t] -= freq * c + pres
        if bias is not None:
            y[i] += (bias if bias.dim() == 1 else bias[i])[:V].double().cpu()
        r = -1 if mask is None else (int(row[i]) if row is not None else (0 if mask.shape[0] == 1 else i))
        if mask is not None and -1 < r < mask.shape[0]:
            w = mask[r].cpu().tolist()
            for t in range(V):
                if not w[t // 32] >> (t % 32) & 1:
                    y[i, t] = -math.inf
    return y


def check(got, want, x, top):
    """Five roundings to 24 bits of values up to `top`, then one to the type's bits: the result lies between the two ends
    of that interval, each rounded to the type."""
    g = got.cpu()
    assert torch.equal(torch.isinf(g), torch.isinf(want)) and torch.equal(torch.isnan(g), torch.isnan(want))
    fine = torch.isfinite(want)
    bound = 5 * 2.0 ** -24 * top
    assert (((want[fine] - bound).to(g.dtype) <= g[fine]) & (g[fine] <= (want[fine] + bound).to(g.dtype))).all()


def masks(rows, V, share, gen):
    words = -(-V // 32)
    bits = torch.rand(rows, words * 32, generator=gen) < share
    w = (bits.view(rows, words, 32).long() << torch.arange(32)).sum(-1)
    return (w - ((w >> 31) << 32)).to(torch.int32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lanes,V,T", [(1, 1, 1), (3, 7, 5), (5, 33, 40), (4, 257, 0), (2, 8192, 100), (3, 8193, 300), (2, 16389, 2000), (7, 1000, 70), (2, 50257, 1000)])
def test_all_edits(B, dtype, lanes, V, T):
    gen = torch.Generator().manual_seed(V + T)
    x = (torch.randn(lanes, V, generator=gen) * 4).to(DT[dtype])
    seq = (torch.rand(lanes, T, generator=gen) ** 2 * V).to(torch.int32)
    length = torch.randint(0, T + 1, (lanes,), generator=gen, dtype=torch.int32)
    length[0] = T
    prompt = (length.float() * torch.rand(lanes, generator=gen)).to(torch.int32)
    bias = torch.randn(V, generator=gen)
    mask, row = masks(3, V, 0.6, gen), torch.randint(-1, 3, (lanes,), generator=gen, dtype=torch.int32)
    status = torch.full((lanes,), 7, dtype=torch.int32, device="cuda")
    c = lambda t: t.cuda()
    got = B.as_logits_edit(c(x), c(seq), c(length), c(prompt), 1.4, 0.3, 0.2, c(bias), c(mask), c(row), lane_status=status)
    check(got, reference(x, seq, length, prompt, 1.4, 0.3, 0.2, bias, mask, row), x, 200.0)
    assert (status == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", ["repetition", "presence", "frequency", "bias", "lane_bias", "mask", "lane_mask", "one_mask", "nothing"])
def test_each_edit_alone_and_in_place(B, dtype, what):
    lanes, V, T = 6, 9001, 64
    gen = torch.Generator().manual_seed(3)
    x = (torch.randn(lanes, V, generator=gen) * 3).to(DT[dtype])
    seq = torch.randint(0, 50, (lanes, T), generator=gen, dtype=torch.int32)
    length = torch.tensor([0, 1, 2, 63, 64, 30], dtype=torch.int32)
    kw, ref = {}, {}
    if what in ("repetition", "presence", "frequency"):
        kw = dict(seq=seq.cuda(), length=length.cuda(), **{what: 1.7})
        ref = dict(seq=seq, length=length, **{{"repetition": "rep", "presence": "pres", "frequency": "freq"}[what]: 1.7})
    elif what.endswith("bias"):
        b = torch.randn(*((lanes, V) if what == "lane_bias" else (V,)), generator=gen)
        kw, ref = dict(bias=b.cuda()), dict(bias=b)
    elif what.endswith("mask"):
        m = masks(lanes if what == "lane_mask" else 1 if what == "one_mask" else 4, V, 0.5, gen)
        r = torch.tensor([0, 1, 2, 3, -1, 0], dtype=torch.int32) if what == "mask" else None
        kw, ref = dict(mask=m.cuda(), mask_row=None if r is None else r.cuda()), dict(mask=m, row=r)
    want = reference(x, **ref)
    y = x.cuda()
    got = B.as_logits_edit(y, **kw)
    assert torch.equal(y.cpu(), x)                       # the input is left alone
    check(got, want, x, 130.0)
    inplace = B.as_logits_edit(y, out=y, **kw)
    assert inplace.data_ptr() == y.data_ptr() and torch.equal(inplace, got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("off_in,off_out,pad_in,pad_out", [(0, 0, 0, 0), (1, 1, 0, 0), (3, 3, 5, 5), (0, 1, 0, 0), (0, 0, 3, 0), (5, 2, 1, 9), (7, 7, 8, 16)])
def test_row_starts_and_pitches(B, dtype, off_in, off_out, pad_in, pad_out):
    lanes, V = 5, 1234
    gen = torch.Generator().manual_seed(9)
    raw_in = (torch.randn(off_in + lanes * (V + pad_in) + 16, generator=gen) * 3).to(DT[dtype]).cuda()
    raw_out = torch.full((off_out + lanes * (V + pad_out) + 16,), 123.0, dtype=DT[dtype], device="cuda")
    x = raw_in[off_in:off_in + lanes * (V + pad_in)].view(lanes, V + pad_in)[:, :V]
    out = raw_out[off_out:off_out + lanes * (V + pad_out)].view(lanes, V + pad_out)[:, :V]
    bias, mask = torch.randn(V, generator=gen), masks(lanes, V, 0.5, gen)
    seq = torch.randint(0, V, (lanes, 300), generator=gen, dtype=torch.int32)
    length = torch.full((lanes,), 300, dtype=torch.int32)
    B.as_logits_edit(x, seq.cuda(), length.cuda(), None, 1.2, 0.5, 0.25, bias.cuda(), mask.cuda(), out=out)
    check(out, reference(x.cpu(), seq, length, None, 1.2, 0.5, 0.25, bias, mask), x, 130.0)
    keep = torch.ones_like(raw_out, dtype=torch.bool)
    keep[off_out:off_out + lanes * (V + pad_out)].view(lanes, V + pad_out)[:, :V] = False
    assert (raw_out[keep] == 123.0).all()                # nothing is written beside the rows


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_at_the_edge(B, dtype):
    """-inf, the type's lowest value, NaN and +inf: masked places are -inf whatever they held, a fully masked row is -inf."""
    V = 70
    lowest = torch.finfo(DT[dtype]).min
    x = torch.linspace(-3, 3, 2 * V).view(2, V).to(DT[dtype])
    x[:, 0], x[:, 1], x[:, 2], x[:, 3], x[:, 5] = float("nan"), float("inf"), float("-inf"), lowest, lowest
    mask = torch.zeros(2, 3, dtype=torch.int32)
    mask[0, 0], mask[0, 2] = ~0b10011 & 0x7FFFFFFF, 1
    seq = torch.tensor([[2, 3, 3, 6], [1, 1, 1, 1]], dtype=torch.int32)
    length = torch.tensor([4, 4], dtype=torch.int32)
    got = B.as_logits_edit(x.cuda(), seq.cuda(), length.cuda(), repetition=2.0, presence=1.0, mask=mask.cuda()).cpu()
    assert (got[1] == float("-inf")).all()
    assert (got[0, [0, 1, 2, 4]] == float("-inf")).all() and got[0, 3] == float("-inf")       # lowest * 2 leaves the type
    assert got[0, 5] == lowest and torch.equal(got[0, 7:31], x[0, 7:31])
    assert (got[0, 31:64] == float("-inf")).all() and got[0, 64] == x[0, 64] and (got[0, 65:] == float("-inf")).all()


def test_status_and_skipped_tokens(B):
    V = 20
    x = torch.zeros(5, V) + 1.0
    seq = torch.tensor([[1, 2, 3], [V, 2, 2], [-1, 4, 4], [5, 5, 5], [6, 6, 6]], dtype=torch.int32)
    length = torch.tensor([3, 3, 2, 9, -2], dtype=torch.int32)
    status = torch.empty(5, dtype=torch.int32, device="cuda")
    mask = torch.full((2, 1), -1, dtype=torch.int32)
    row = torch.tensor([0, 1, -1, 0, 2], dtype=torch.int32)
    got = B.as_logits_edit(x.cuda(), seq.cuda(), length.cuda(), frequency=0.5, mask=mask.cuda(), mask_row=row.cuda(), lane_status=status).cpu()
    assert status.tolist() == [0, B.ERR_INVALID_ARG, B.ERR_INVALID_ARG, B.ERR_INVALID_ARG, B.ERR_INVALID_ARG]
    assert got[1, 2] == 0.0 and got[2, 4] == 0.5 and got[3, 5] == -0.5 and (got[4] == 1.0).all()


def test_other_stream_and_empty(B):
    x = torch.randn(64, 32000, device="cuda", dtype=torch.bfloat16)
    bias = torch.randn(32000, device="cuda")
    want = B.as_logits_edit(x, bias=bias)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = x.clone()
        got = B.as_logits_edit(y, bias=bias)
    s.synchronize()
    assert torch.equal(got, want)
    assert B.as_logits_edit(x[:0]).shape == (0, 32000)


def test_rows_past_32_bits(B):
    """Offsets of the last rows pass 2^31 elements' bytes."""
    lanes, V = 1100, 1 << 19
    x = torch.zeros(lanes, V, device="cuda")
    x[-1, -1], x[-1, 0] = 3.0, 5.0
    seq = torch.tensor([[V - 1, 0]], dtype=torch.int32, device="cuda").expand(lanes, 2).contiguous()
    length = torch.full((lanes,), 2, dtype=torch.int32, device="cuda")
    got = B.as_logits_edit(x, seq, length, frequency=1.0)
    assert got[-1, -1] == 2.0 and got[-1, 0] == 4.0 and got[-1, 1] == 0.0 and got[500, 0] == -1.0
