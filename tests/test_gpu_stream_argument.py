"""`stream=` of the calls around the step: their scratch stays theirs while the launch stream works."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import binding
    return binding


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def busy(stream):
    """Some milliseconds of work on the stream, so that what is launched behind it has not begun when the call returns."""
    with torch.cuda.stream(stream):
        x = torch.zeros(4096, 4096, device="cuda")
        for _ in range(20):
            x = x @ x
    return x


def overwrite(nbytes):
    """Takes blocks of the current stream's memory of about this size and fills them."""
    held = [torch.full((max(1, nbytes // 4 + d),), 0x5A5A5A5A, dtype=torch.int32, device="cuda") for d in (0, 0, 0, 0, -64, 64)]
    torch.cuda.current_stream().synchronize()
    return held


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("T", [1, 100])
def test_attention(B, T, raw):
    lens, H, D, P = [900, 333, 2000, 120], 4, 64, 64
    g = torch.Generator().manual_seed(T)
    M = 33
    pages = B.cache4_pages(len(lens) * M, H, D, P)
    table = torch.randperm(len(lens) * M, generator=g).to(torch.int32).view(len(lens), M).cuda()
    k, v = (torch.randn(len(lens), 2000, H, D, generator=g).cuda() for _ in range(2))
    B.as_cache4_append(pages, k, v, table, i32(lens))
    q = torch.randn(len(lens), T, 16, D, generator=g).cuda().bfloat16()
    n = i32(lens)
    want = B.as_cache4_attend(pages, q, table, n, 0.1)
    nbytes = B.as_cache4_attend_work_bytes(pages, B.BF16, len(lens), T, 16)
    s = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        keep = busy(s)
        out = torch.zeros_like(q)
        torch.cuda.current_stream().synchronize()
        B.as_cache4_attend(pages, q, table, n, 0.1, out=out, stream=s.cuda_stream if raw else s)
        held = overwrite(nbytes)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(bool((h == 0x5A5A5A5A).all()) for h in held)
        del keep


def test_pages(B):
    P, n_pages = 16, 4000
    lens = [200 + i for i in range(24)]
    M = 20
    table = torch.full((len(lens), M), -1, dtype=torch.int32, device="cuda")
    length, ref = i32([0] * len(lens)), i32([0] * n_pages)
    B.as_pages_grow(i32(lens), table, length, ref, P)
    pool = torch.randint(0, 1 << 30, (2, n_pages, 64), dtype=torch.int32, device="cuda")
    parent, add = i32([i % 24 for i in range(120)]), i32([3] * 120)

    def life(pool, **stream):
        t, n, r = B.as_pages_fork(parent, table, length, ref, P, pool, **outs, **stream)
        B.as_pages_grow(add, t, n, r, P, **stream)
        used = B.as_pages_compact(t, r, pool, **stream)
        return t, n, r, used, pool
    outs = {}
    want = [x.clone() for x in life(pool.clone())]
    s = torch.cuda.Stream()
    for _ in range(3):
        mine = pool.clone()
        torch.cuda.synchronize()
        keep = busy(s)
        got = life(mine, stream=s)
        held = overwrite(B.as_pages_work_bytes(24, 120, n_pages)) + overwrite(B.as_pages_work_bytes(120, 120, n_pages)) + overwrite(4 * n_pages)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(bool((h == 0x5A5A5A5A).all()) for h in held)
        del keep
