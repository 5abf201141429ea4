"""The windowed attention, weight, eviction, trim and verification calls captured and replayed, on streams of their own, side by side."""
import pytest

torch = pytest.importorskip("torch")
from tests import test_gpu_cache4 as C  # noqa: E402
from tests import test_gpu_verify as V  # noqa: E402
from tests.test_gpu_stream_argument import busy, overwrite  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import binding
    return binding


def calls(B, T, seed):
    """[(name, function of (stream) -> outputs)] on inputs of one set of lanes."""
    lens, H, D, P, Hq = [700, 333, 1201], 2, 128, 32, 8
    gen = torch.Generator().manual_seed(seed)
    pages, table, _, _ = C.filled(B, lens, H, D, P, seed, None, None)
    n = C.i32(lens)
    q = torch.randn(3, T, Hq, D, generator=gen).bfloat16().cuda()
    lse = torch.empty(3, T, Hq, device="cuda")
    B.as_cache4_attend(pages, q, table, n, 0.1, lse=lse)
    weight = torch.rand(3, H, 1216, generator=gen).cuda()
    target, draft, drafted, u, codes = (x.cuda() for x in V.inputs(9, 3, 5000, "bf16", seed))
    ref = torch.zeros(pages.shape[0], dtype=torch.int32, device="cuda")
    ref[table[table >= 0].long()] = 1
    keep, gone, left = C.i32([650, 333, 700]), C.i32([[0, 64], [0, 0], [32, 600]]), C.i32([300, 200, 700])

    def evict(s):
        mine, out = pages.clone(), torch.empty_like(weight)
        B.as_cache4_evict(mine, weight, table, n, left, 50, weight_out=out, stream=s)
        return mine, out

    def weigh(s):
        w = weight.clone()
        B.as_cache4_weigh(pages, q, lse, table, n, 0.1, w, stream=s)
        return w,

    def trim(s):
        outs = [torch.empty_like(x) for x in (table, n, ref)]
        B.as_pages_trim(keep, table, n, ref, P, gone=gone, table_out=outs[0], length_out=outs[1], ref_out=outs[2], stream=s)
        return tuple(outs)

    return [("window", lambda s: (B.as_cache4_attend(pages, q, table, n, 0.1, window=200, sinks=5, stream=s),)), ("weigh", weigh), ("evict", evict), ("trim", trim),
            ("verify", lambda s: B.as_step_verify(target, draft, drafted, u, codes, 0.9, stream=s)),
            ("verify, nucleus", lambda s: B.as_step_verify(target, draft, drafted, u, codes, 0.9, 0, 0.9, stream=s))]


@pytest.mark.parametrize("T", [1, 60])
def test_captured_and_replayed(B, T):
    for name, call in calls(B, T, 3):
        want = [x.clone() for x in call(None)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(None)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call(None)
        for _ in range(3):
            for x in got:
                x.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), name


@pytest.mark.parametrize("T", [1, 60])
def test_a_stream_of_its_own(B, T):
    """Scratch belongs to the stream that the call launches on."""
    for name, call in calls(B, T, 4):
        want = [x.clone() for x in call(None)]
        torch.cuda.synchronize()
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            keep = busy(stream)
            got = call(stream)
        held = overwrite(1 << 16)
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name
        del keep, held


@pytest.mark.parametrize("T", [1, 60])
def test_two_at_once(B, T):
    """Two sets of lanes on two streams."""
    a, b = calls(B, T, 5), calls(B, T, 6)
    for (name, one), (_, two) in zip(a, b):
        want = [[x.clone() for x in f(None)] for f in (one, two)]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        got = []
        for s, f in zip(streams, (one, two)):
            with torch.cuda.stream(s):
                got.append([f(s) for _ in range(5)])
        torch.cuda.synchronize()
        for w, rounds in zip(want, got):
            assert all(torch.equal(x, y) for r in rounds for x, y in zip(r, w)), name
