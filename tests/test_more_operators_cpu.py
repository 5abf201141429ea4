"""Refusals of the windowed attention, weight, eviction, trim and verification calls: every host-detectable error comes back before
the device is touched."""
import ctypes

import pytest

from tests.test_operators_cpu import CACHE_BAD, P, _cache

torch = pytest.importorskip("torch")
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import _build, binding
    _build.build()
    binding.lib()
    return binding


def _window(B, c, dtype=0, lanes=2, T=1, q=P, q_ld=512, q_heads=4, table=P, max_pages=2, length=P, scale=1.0, N=1, window=4, sinks=0, out=P, work=P, work_bytes=1 << 40):
    return B.lib().as_cache4_attend_window(ctypes.byref(c) if c else None, q, q_ld, dtype, lanes, T, q_heads, table, max_pages, length, scale, N, None, window, sinks,
                                           out, None, None, work, work_bytes, None)


def _weigh(B, c, dtype=0, lanes=2, T=1, q=P, q_ld=512, q_heads=4, lse=P, table=P, max_pages=2, length=P, scale=1.0, window=0, sinks=0, weight=P, weight_ld=32, work=P,
           work_bytes=1 << 40):
    return B.lib().as_cache4_weigh(ctypes.byref(c) if c else None, q, q_ld, dtype, lanes, T, q_heads, lse, table, max_pages, length, scale, window, sinks, 1, None, weight,
                                   weight_ld, None, work, work_bytes, None)


def _evict(B, c, lanes=2, weight=P, weight_ld=32, table=P, max_pages=2, length=P, keep=P, recent=0, out=P):
    return B.lib().as_cache4_evict(ctypes.byref(c) if c else None, weight, weight_ld, lanes, table, max_pages, length, keep, None, recent, None, out, None, None)


@pytest.mark.parametrize("call", [_window, _weigh, _evict])
def test_cache_refusals(B, call):
    for kw, code in CACHE_BAD:
        assert call(B, _cache(B, **kw)) == (B.ERR_INVALID_ARG if code == "inv" else B.ERR_UNSUPPORTED), kw
    assert call(B, None) == B.ERR_INVALID_ARG
    c = _cache(B)
    for kw in (dict(lanes=-1), dict(table=None), dict(length=None), dict(max_pages=0)):
        assert call(B, c, **kw) == B.ERR_INVALID_ARG, kw
    assert call(B, c, max_pages=1 << 27) == B.ERR_UNSUPPORTED
    assert call(B, c, lanes=0, table=None, length=None) == B.OK
    assert B.lib().as_last_error() is not None


@pytest.mark.parametrize("call", [_window, _weigh])
def test_query_refusals(B, call):
    c = _cache(B)
    for kw in (dict(dtype=5), dict(T=0), dict(q_heads=0), dict(q_heads=3), dict(q_ld=255), dict(scale=NAN), dict(scale=INF), dict(scale=1e300), dict(q=None), dict(q=P + 1),
               dict(work=None), dict(work=P + 16), dict(work_bytes=0), dict(sinks=-1), dict(window=-1)):
        assert call(B, c, **kw) == B.ERR_INVALID_ARG, kw
    assert call(B, c, lanes=1 << 16, T=1 << 15) == B.ERR_UNSUPPORTED
    assert call(B, c, lanes=1 << 20, T=512, q_heads=64, q_ld=1 << 20) == B.ERR_UNSUPPORTED
    assert call(B, c, lanes=1 << 14, max_pages=1 << 26) == B.ERR_UNSUPPORTED


def test_more_refusals(B):
    c = _cache(B)
    for kw in (dict(window=0), dict(N=0), dict(lanes=3, N=2), dict(out=None), dict(out=P + 8)):
        assert _window(B, c, **kw) == B.ERR_INVALID_ARG, kw
    for kw in (dict(lse=None), dict(lse=P + 2), dict(weight=None), dict(weight=P + 1), dict(weight_ld=0)):
        assert _weigh(B, c, **kw) == B.ERR_INVALID_ARG, kw
    for kw in (dict(weight=None), dict(weight=P + 2), dict(weight_ld=0), dict(keep=None), dict(recent=-1), dict(out=None), dict(out=P + 1)):
        assert _evict(B, c, **kw) == B.ERR_INVALID_ARG, kw
    wb = lambda **k: B.lib().as_cache4_weigh_work_bytes(ctypes.byref(k.get("c", c)), k.get("dtype", 0), k.get("lanes", 2), k.get("T", 1), k.get("q_heads", 4))
    assert wb() > 0 and wb(c=_cache(B, head_dim=96)) == wb(dtype=3) == wb(lanes=0) == wb(T=0) == wb(q_heads=3) == wb(lanes=1 << 20, T=1 << 20) == 0


def _trim(B, lanes=2, max_pages=2, page_size=16, n_pages=4, table=P, length=P, ref=P, table_out=P, len_out=P, ref_out=P, work=P, work_bytes=1 << 40):
    return B.lib().as_pages_trim(P, None, lanes, max_pages, page_size, n_pages, table, length, ref, table_out, len_out, ref_out, None, work, work_bytes, None)


def test_trim_refusals(B):
    for kw in (dict(lanes=-1), dict(max_pages=0), dict(page_size=0), dict(n_pages=0), dict(table=None), dict(length=None), dict(ref=None), dict(table_out=None), dict(len_out=None),
               dict(ref_out=None), dict(work=None), dict(work=P + 64), dict(work_bytes=16)):
        assert _trim(B, **kw) == B.ERR_INVALID_ARG, kw
    assert _trim(B, max_pages=1 << 27) == B.ERR_UNSUPPORTED and _trim(B, n_pages=(1 << 20) + 1) == B.ERR_UNSUPPORTED


def _verify(B, target=P, target_ld=8, draft=P, draft_ld=8, dtype=0, lanes=2, K=3, V=8, drafted=P, u=P, codes=P, temp=1.0, top_p=1.0, tokens=P, accepted=P, out=P, work=P,
            work_bytes=1 << 40):
    return B.lib().as_step_verify(target, target_ld, draft, draft_ld, dtype, lanes, K, V, drafted, None, u, codes, temp, 0, top_p, tokens, accepted, out, None, work, work_bytes,
                                  None)


def test_verify_refusals(B):
    for kw in (dict(dtype=2), dict(lanes=-1), dict(K=-1), dict(V=0), dict(target_ld=7), dict(draft_ld=7), dict(temp=0.0), dict(temp=INF), dict(temp=NAN), dict(top_p=NAN),
               dict(target=None), dict(target=P + 1), dict(draft=P + 2), dict(drafted=None), dict(u=None), dict(codes=None), dict(tokens=None), dict(accepted=None),
               dict(out=None), dict(work=None), dict(work=P + 8), dict(work_bytes=8)):
        assert _verify(B, **kw) == B.ERR_INVALID_ARG, kw
    big = (1 << 20) + 1
    assert _verify(B, V=big, target_ld=big, draft_ld=big) == B.ERR_UNSUPPORTED
    assert _verify(B, lanes=1 << 20, K=1 << 12) == B.ERR_UNSUPPORTED
    assert _verify(B, lanes=0, target=None) == B.OK
    wb = B.lib().as_step_verify_work_bytes
    assert wb(0, 2, 3, 8) > 0 and wb(2, 2, 3, 8) == wb(0, 0, 3, 8) == wb(0, 2, -1, 8) == wb(0, 2, 3, 0) == wb(0, 1 << 20, 1 << 12, 8) == 0


def test_binding_refusals(B):
    """Shapes and types that the Python side turns away."""
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    pages, table, length = z(4, 2, 1, 18 * 64, dtype=torch.uint8), i(2, 2), i(2)
    q, lse, w = z(2, 1, 4, 64), z(2, 1, 4), z(2, 2, 32)
    bad = [
        lambda: B.as_cache4_attend(pages, q, table, length, 1.0, sinks=3),
        lambda: B.as_cache4_weigh(pages, q, z(2, 1, 3), table, length, 1.0, w),
        lambda: B.as_cache4_weigh(pages, q, lse.double(), table, length, 1.0, w),
        lambda: B.as_cache4_weigh(pages, q, lse, table, length, 1.0, z(2, 3, 32)),
        lambda: B.as_cache4_weigh(pages, q, lse, table, length, 1.0, z(2, 32, 2).transpose(1, 2)),
        lambda: B.as_cache4_weigh(pages, q, lse, table, length, 1.0, w, window=0),
        lambda: B.as_cache4_weigh(pages, q, lse, table, length, 1.0, w, sinks=1),
        lambda: B.as_cache4_evict(pages, w, table, length, i(3)),
        lambda: B.as_cache4_evict(pages, w, table, length, i(2), weight_out=z(2, 2, 33)),
        lambda: B.as_cache4_evict(pages, w, table, length, i(2), ref=i(5)),
        lambda: B.as_pages_trim(i(3), table, length, i(4), 16),
        lambda: B.as_pages_trim(i(2), table, length, i(4), 16, gone=i(2)),
        lambda: B.as_step_verify(z(2, 3, 8), z(2, 2, 8), i(2, 3), z(2, 3, dtype=torch.float64), z(2, dtype=torch.float64)),
        lambda: B.as_step_verify(z(2, 4, 8), z(2, 3, 8).bfloat16(), i(2, 3), z(2, 3, dtype=torch.float64), z(2, dtype=torch.float64)),
        lambda: B.as_step_verify(z(2, 4, 8), z(2, 3, 7), i(2, 3), z(2, 3, dtype=torch.float64), z(2, dtype=torch.float64)),
        lambda: B.as_step_verify(z(2, 4, 8), z(2, 3, 8), i(2, 3), z(2, 3), z(2, dtype=torch.float64)),
        lambda: B.as_step_verify(z(2, 4, 8), z(2, 3, 8), i(2, 3), z(2, 3, dtype=torch.float64), z(3, dtype=torch.float64)),
        lambda: B.as_step_verify(z(2, 4, 16)[:, :, ::2], None, i(2, 3), z(2, 3, dtype=torch.float64), z(2, dtype=torch.float64)),
        lambda: B.as_step_verify(z(2, 4, 8), None, i(2, 3).long(), z(2, 3, dtype=torch.float64), z(2, dtype=torch.float64)),
        lambda: B.as_step_verify(z(2, 4, 8), None, i(2, 3), z(2, 3, dtype=torch.float64), z(2, dtype=torch.float64), V=9),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
