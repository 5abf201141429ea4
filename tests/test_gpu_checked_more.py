"""The windowed attention, weight, eviction, trim and verification calls in the build that checks computed indices, with guard words around
outputs and scratch."""
import random

import pytest

torch = pytest.importorskip("torch")
from tests import test_gpu_cache4 as C  # noqa: E402
from tests import test_gpu_evict as E  # noqa: E402
from tests import test_gpu_trim as R  # noqa: E402
from tests import test_gpu_verify as V  # noqa: E402
from tests import test_gpu_weigh as G  # noqa: E402
from tests import test_gpu_window as W  # noqa: E402
from tests.test_gpu_checked_cache import B, Guarded  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,T,Hq,H,P,window,sinks", W.SHAPES)
def test_window(B, dtype, D, lens, T, Hq, H, P, window, sinks):  # noqa: F811
    gen = torch.Generator().manual_seed(T * 7 + Hq)
    pages, table, k, v = C.filled(B, lens, H, D, P, 5, None, None)
    q = (torch.randn(len(lens), T, Hq, D, generator=gen) * 1.5).to(C.DT[dtype]).cuda()
    out, lse, status = Guarded(q.shape, q.dtype), Guarded((len(lens), T, Hq), torch.float32), Guarded((len(lens),), torch.int32)
    work = Guarded((B.as_cache4_attend_work_bytes(pages, B.F32 if dtype == "f32" else B.BF16, len(lens), T, Hq),), torch.uint8)
    B.as_cache4_attend(pages, q, table, C.i32(lens), D ** -0.5, out=out.view, lse=lse.view, lane_status=status.view, work=work.view, window=window, sinks=sinks)
    assert all(x.intact() for x in (out, lse, status, work)) and not status.view.any()
    W.check(B, dtype, out.view, lse.view, q, k, v, lens, D ** -0.5, window, sinks)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,T,Hq,H,D,P,shared,tails,window,sinks", W.SHARED)
def test_window_by_groups(B, dtype, N, T, Hq, H, D, P, shared, tails, window, sinks):  # noqa: F811
    W.test_shared_beginnings_by_groups(B, dtype, N, T, Hq, H, D, P, shared, tails, window, sinks)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,T,Hq,H,P,window,sinks", G.SHAPES)
def test_weigh(B, dtype, D, lens, T, Hq, H, P, window, sinks):  # noqa: F811
    gen = torch.Generator().manual_seed(T * 7 + Hq)
    pages, table, k, v = C.filled(B, lens, H, D, P, 5, None, None)
    q = (torch.randn(len(lens), T, Hq, D, generator=gen) * 1.5).to(C.DT[dtype]).cuda()
    lse = torch.empty(len(lens), T, Hq, device="cuda")
    B.as_cache4_attend(pages, q, table, C.i32(lens), D ** -0.5, lse=lse, window=window or None, sinks=sinks)
    want, size = G.weights(q.cpu(), lse.cpu(), k, lens, D ** -0.5, window or 1 << 30, sinks)
    weight, status = Guarded((len(lens), H, max(lens)), torch.float32), Guarded((len(lens),), torch.int32)
    work = Guarded((B.as_cache4_weigh_work_bytes(pages, B.F32 if dtype == "f32" else B.BF16, len(lens), T, Hq),), torch.uint8)
    B.as_cache4_weigh(pages, q, lse, table, C.i32(lens), D ** -0.5, weight.view, window=window or None, sinks=sinks, add=False, lane_status=status.view, work=work.view)
    assert all(x.intact() for x in (weight, status, work)) and not status.view.any()
    top = float(lse[torch.isfinite(lse)].abs().max()) if torch.isfinite(lse).any() else 0.0
    for i, n in enumerate(lens):
        assert ((weight.view[i, :, :n].double().cpu() - want[i]).abs() <= G.tolerance(size, top, T * Hq // H, want[i])).all()


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("lens,keep,first,recent,H,D,P", E.CASES)
def test_evict(B, lens, keep, first, recent, H, D, P, in_place):  # noqa: F811
    pages, table, _, _ = C.filled(B, lens, H, D, P, 1, None, None)
    held = Guarded(pages.shape, torch.uint8)
    held.view.copy_(pages)
    w, out, status = Guarded((len(lens), H, max(lens)), torch.float32), Guarded((len(lens), H, max(lens)), torch.float32), Guarded((len(lens),), torch.int32)
    values = torch.rand(w.view.shape, generator=torch.Generator().manual_seed(keep))
    w.view.copy_(values)
    got = B.as_cache4_evict(held.view, w.view, table, C.i32(lens), C.i32([keep] * len(lens)), recent, first=C.i32([first] * len(lens)),
                            weight_out=None if in_place else out.view, lane_status=status.view)
    assert all(x.intact() for x in (held, w, out, status)) and not status.view.any()
    for i, n in enumerate(lens):
        for h in range(H):
            src, wo = E.model(values[i, h].tolist(), n, keep, first, recent)
            kept = min(n, keep)
            assert torch.equal(E.tokens(held.view, table, i, h, n)[:kept], E.tokens(pages, table, i, h, n)[src[:kept]])
            assert torch.equal(got[i, h].cpu(), torch.tensor(wo))


@pytest.mark.parametrize("seed", range(6))
def test_trim(B, seed):  # noqa: F811
    rng = random.Random(seed)
    lanes, P, M = rng.choice((1, 5, 40, 300)), rng.choice((1, 16, 24, 64)), rng.choice((1, 7, 150))
    table, lens, ref = R.make(rng, lanes, P, M, seed % 2)
    keep, gone = [max(0, n - rng.randint(0, 40)) for n in lens], [(rng.randint(0, n), rng.randint(0, n)) for n in lens]
    outs = [Guarded((lanes, M), torch.int32), Guarded((lanes,), torch.int32), Guarded((len(ref),), torch.int32), Guarded((lanes,), torch.int32)]
    work = Guarded((B.as_pages_work_bytes(lanes, lanes, len(ref)) // 4,), torch.int32)
    B.as_pages_trim(C.i32(keep), C.i32(table), C.i32(lens), C.i32(ref), P, gone=C.i32(gone), table_out=outs[0].view, length_out=outs[1].view, ref_out=outs[2].view,
                    lane_status=outs[3].view, work=work.view)
    assert all(x.intact() for x in outs + [work])
    assert tuple(x.view.tolist() for x in outs) == R.model(table, lens, ref, P, keep, gone)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temp,top_k,top_p", V.CUTS)
@pytest.mark.parametrize("lanes,K,V_", [(5, 3, 1), (7, 2, 2), (40, 4, 33), (33, 1, 1000), (9, 8, 4099), (3, 40, 257), (6, 3, 50257), (700, 2, 513)])
def test_verify(B, dtype, temp, top_k, top_p, lanes, K, V_):  # noqa: F811
    target, draft, drafted, u, codes = V.inputs(lanes, K, V_, dtype, V_ + K)
    work = Guarded(((B.as_step_verify_work_bytes(B.F32 if dtype == "f32" else B.BF16, lanes, K, V_) + 3) // 4,), torch.int32)
    tokens, accepted, out = Guarded((lanes, K + 1), torch.int32), Guarded((lanes,), torch.int32), Guarded((lanes,), torch.float64)
    V.check(B, target, draft, drafted, u, codes, temp, top_k, top_p, work=work.view, tokens=tokens.view, accepted=accepted.view, codes_out=out.view)
    assert all(x.intact() for x in (work, tokens, accepted, out))


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("lanes,H,D,P,top,recent", [(38, 4, 64, 16, 1500, 40), (310, 1, 64, 32, 130, 17), (30, 3, 128, 32, 1500, 33)])
def test_evict_many(B, lanes, H, D, P, top, recent, in_place):  # noqa: F811
    E.test_many_lanes_and_heads(B, lanes, H, D, P, top, recent, "ties", in_place)


@pytest.mark.parametrize("in_place", [True, False])
def test_evict_long(B, in_place):  # noqa: F811
    E.test_middles_beyond_shared_memory(B, [40000, 300], [20000, 100], [7, 3], 90, 1, 64, 64, "ties", in_place)


@pytest.mark.parametrize("place", ["front", "end"])
def test_verify_next_to_nothing(B, place):  # noqa: F811
    V.test_chunks_of_tokens_next_to_nothing(B, "bf16", 1.0, 4099, place)
