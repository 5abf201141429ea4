"""The cache, attention and page calls in the build that checks computed indices, with guard words around outputs and scratch."""
import os
import random

import pytest

torch = pytest.importorskip("torch")
from tests import test_gpu_cache4 as C  # noqa: E402
from tests.test_gpu_pages import Model, same  # noqa: E402

pytestmark = pytest.mark.gpu
GUARD = 256


@pytest.fixture()
def B():
    from paper_2210_15458_b200 import _build, binding
    if not os.path.exists(_build.LIB_CHECKED):
        pytest.fail("checked library missing: run __graft_entry__.build()")
    binding.use_library(_build.LIB_CHECKED)
    binding.as_debug_bounds(reset=True)
    yield binding
    torch.cuda.synchronize()
    record = binding.as_debug_bounds(reset=True)
    binding.use_library(None)
    assert record[0] == 0, "index %d outside [0, %d) at site %d (%d in all)" % (record[2], record[3], record[1], record[0])


class Guarded:
    def __init__(self, shape, dtype):
        n = 1
        for s in shape:
            n *= s
        self.full = torch.full((n + 2 * GUARD,), 7, dtype=dtype, device="cuda")
        self.n, self.view = n, self.full[GUARD:GUARD + n].view(*shape)

    def intact(self):
        return bool((self.full[:GUARD] == 7).all()) and bool((self.full[GUARD + self.n:] == 7).all())


def attend(B, pages, q, table, lens, scale, **kw):
    """(out, lse) between guard words, with scratch of exactly the size that is asked for."""
    lanes, T, Hq, D = q.shape
    out, lse, status = Guarded(q.shape, q.dtype), Guarded((lanes, T, Hq), torch.float32), Guarded((lanes,), torch.int32)
    work = Guarded((B.as_cache4_attend_work_bytes(pages, B.F32 if q.dtype == torch.float32 else B.BF16, lanes, T, Hq, kw.get("N", 1)),), torch.uint8)
    B.as_cache4_attend(pages, q, table, C.i32(lens), scale, out=out.view, lse=lse.view, lane_status=status.view, work=work.view, **kw)
    assert all(x.intact() for x in (out, lse, status, work)) and not status.view.any()
    return out.view, lse.view


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,T,Hq,H,P", C.SHAPES)
def test_attention(B, dtype, D, lens, T, Hq, H, P):
    gen = torch.Generator().manual_seed(T * 7 + Hq)
    gk, gv = (0.2 + 0.3 * torch.rand(H, generator=gen)).cuda(), (0.2 + 0.3 * torch.rand(H, generator=gen)).cuda()
    pages, table, k, v = C.filled(B, lens, H, D, P, 5, gk, gv)
    q = (torch.randn(len(lens), T, Hq + 3, D, generator=gen) * 1.5).to(C.DT[dtype]).cuda()[:, :, 2:2 + Hq]
    out, lse = attend(B, pages, q, table, lens, D ** -0.5, k_scale=gk, v_scale=gv)
    want, wlse, size = C.attention(q.cpu(), k, v, lens, D ** -0.5)
    tol, ltol = C.bounds(dtype, size, max([float(x.abs().max()) for x in v if x.numel()] + [0.0]), want)
    assert ((out.double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,T,Hq,H,D,P,shared,tails", [(3, 1, 4, 2, 128, 16, [0, 48], [5, 1, 17, 1, 2, 40]), (33, 1, 8, 1, 128, 64, [1024, 64], [1 + i % 7 for i in range(66)]),
                                                       (2, 3, 4, 2, 64, 16, [64, 0], [6, 9, 3, 4]), (4, 40, 4, 1, 128, 32, [96], [40, 41, 60, 45]),
                                                       (3, 70, 4, 1, 64, 16, [160], [1, 70, 200]), (64, 1, 4, 2, 64, 128, [1280], [1 + i for i in range(64)])])
def test_shared_beginnings(B, dtype, N, T, Hq, H, D, P, shared, tails):
    lens = [shared[i // N] + t for i, t in enumerate(tails)]
    gen = torch.Generator().manual_seed(T)
    pages, table, k, v = C.filled(B, lens, H, D, P, 12, None, None, shared, N)
    q = (torch.randn(len(lens), T, Hq, D, generator=gen) * 1.5).to(C.DT[dtype]).cuda()
    want, wlse, size = C.attention(q.cpu(), k, v, lens, 0.11)
    tol, ltol = C.bounds(dtype, size, max(float(x.abs().max()) for x in v), want)
    for hint in (C.i32(shared), None):
        out, lse = attend(B, pages, q, table, lens, 0.11, N=N, shared=hint)
        assert ((out.double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_lanes_of_many_lengths(B, dtype):
    gen = torch.Generator().manual_seed(2)
    lens = torch.randint(0, 150, (700,), generator=gen).tolist()
    lens[0] = lens[350] = lens[699] = 0
    pages, table, k, v = C.filled(B, lens, 1, 64, 16, 13, None, None)
    q = torch.randn(700, 1, 2, 64, generator=gen).to(C.DT[dtype]).cuda()
    out, lse = attend(B, pages, q, table, lens, 0.125)
    want, _, size = C.attention(q.cpu(), k, v, lens, 0.125)
    tol, _ = C.bounds(dtype, size, max(float(x.abs().max()) for x in v if x.numel()), want)
    assert ((out.double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,T,H,P", [([1], 1, 1, 16), ([40, 33, 2, 0, 64], 33, 2, 32), ([300], 300, 5, 128), ([1999, 700, 31, 0, 703], 700, 3, 64)])
def test_store_and_load(B, dtype, D, lens, T, H, P):
    gen = torch.Generator().manual_seed(D + T)
    k, v = (torch.randn(len(lens), T, H, D, generator=gen).to(C.DT[dtype]).cuda() for _ in range(2))
    pages, table = C.pool(B, lens, H, D, P)
    held = Guarded(pages.shape, torch.uint8)
    held.view.copy_(pages)
    B.as_cache4_append(held.view, k, v, table, C.i32(lens))
    got = B.as_cache4_load(held.view, table, C.i32(lens), T, dtype=C.DT[dtype])
    torch.cuda.synchronize()
    assert held.intact()
    path = B._path
    B.use_library(None)
    B.as_cache4_append(pages, k, v, table, C.i32(lens))
    want = B.as_cache4_load(pages, table, C.i32(lens), T, dtype=C.DT[dtype])
    B.use_library(path)
    assert torch.equal(pages, held.view) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("seed", range(2))
@pytest.mark.parametrize("n_pages,P,M,lanes", [(7, 4, 3, 2), (40, 16, 6, 5), (300, 3, 20, 37), (20000, 16, 90, 1500)])
def test_a_life_of_the_pool(B, seed, n_pages, P, M, lanes):
    rnd = random.Random(seed * 1000 + n_pages)
    m = Model(n_pages, P, M)
    m.rows, m.lens = [[] for _ in range(lanes)], [0] * lanes
    table = torch.full((lanes, M), -1, dtype=torch.int32, device="cuda")
    length, ref = C.i32([0] * lanes), C.i32([0] * n_pages)
    pool = torch.randint(0, 1 << 30, (2, n_pages, 8), dtype=torch.int32, device="cuda")
    for step in range(4):
        add = [rnd.choice((0, 1, 1, P, rnd.randint(0, M * P // 2))) for _ in m.rows]
        work = Guarded((B.as_pages_work_bytes(len(add), len(add), n_pages) // 4,), torch.int32)
        B.as_pages_grow(C.i32(add), table, length, ref, P, work=work.view)
        m.grow(add)
        n = len(m.rows)
        parent = [rnd.choice((-1, rnd.randrange(n), rnd.randrange(min(n, 3)))) for _ in range(rnd.choice((n, max(1, n // 2), lanes)))]
        fwork = Guarded((B.as_pages_work_bytes(n, len(parent), n_pages) // 4,), torch.int32)
        t, l = Guarded((len(parent), M), torch.int32), Guarded((len(parent),), torch.int32)
        r = Guarded((n_pages,), torch.int32)
        B.as_pages_fork(C.i32(parent), table, length, ref, P, pool, t.view, l.view, r.view, work=fwork.view)
        m.fork(parent)
        cwork = Guarded((B.as_pages_work_bytes(len(parent), len(parent), n_pages) // 4,), torch.int32)
        B.as_pages_compact(t.view, r.view, pool, work=cwork.view)
        m.compact()
        table, length, ref = t.view, l.view, r.view
        same(m, table, length, ref)
        assert all(x.intact() for x in (work, fwork, cwork, t, l, r))
