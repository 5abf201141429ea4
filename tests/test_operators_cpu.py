"""Refusals of the logit edit, cache and page calls: every host-detectable error comes back before the device is touched."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import _build, binding
    _build.build()
    binding.lib()
    return binding


BUF = (ctypes.c_char * 8192)()
P = (ctypes.addressof(BUF) + 255) & ~255        # never read: all calls below are refused


def _edit(B, dtype=0, lanes=2, V=4, ld=4, out=None, out_ld=4, logits=P, edits=True, **fields):
    e = B.as_logit_edits()
    e.repetition = 1.0
    for k, v in fields.items():
        setattr(e, k, v)
    return B.lib().as_logits_edit(logits, dtype, lanes, V, ld, ctypes.byref(e) if edits else None, P + 4096 if out is None else out, out_ld, None, None)


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(lanes=-1), dict(V=0), dict(ld=3), dict(out_ld=3), dict(edits=False), dict(repetition=0.0), dict(repetition=float("inf")),
    dict(repetition=float("nan")), dict(presence=float("nan")), dict(frequency=float("inf")), dict(d_bias=P, bias_ld=3), dict(d_bias=P, bias_ld=-1),
    dict(d_mask=P, mask_ld=0, mask_rows=1), dict(d_mask=P, mask_ld=1, mask_rows=0), dict(lanes=3, d_mask=P, mask_ld=1, mask_rows=2),
    dict(logits=None), dict(logits=P + 1), dict(out=P + 4097), dict(d_seq=P, seq_ld=4), dict(d_seq=P, d_len=P, seq_ld=-1), dict(out=P, out_ld=5)])
def test_edit_refusals(B, kw):
    assert _edit(B, **kw) == B.ERR_INVALID_ARG, kw
    assert B.lib().as_last_error()


def test_edit_unsupported_and_empty(B):
    assert _edit(B, V=(1 << 20) + 1, ld=1 << 21, out_ld=1 << 21) == B.ERR_UNSUPPORTED
    assert _edit(B, lanes=0, logits=None) == B.OK


def _cache(B, pages=P, n_pages=4, heads=2, head_dim=64, page_size=16):
    return B.as_cache4(pages, n_pages, heads, head_dim, page_size, None, None)


CACHE_BAD = [(dict(pages=None), "inv"), (dict(pages=P + 8), "inv"), (dict(n_pages=0), "inv"), (dict(heads=0), "inv"),
             (dict(head_dim=96), "uns"), (dict(head_dim=0), "uns"), (dict(page_size=24), "uns"), (dict(page_size=256), "uns")]


def _append(B, c, dtype=0, lanes=2, T=1, k=P, v=P, k_ld=128, v_ld=128, table=P, max_pages=2, length=P):
    return B.lib().as_cache4_append(ctypes.byref(c) if c else None, k, k_ld, v, v_ld, dtype, lanes, T, table, max_pages, length, None, None)


def _load(B, c, dtype=0, lanes=2, T=1, k=P, v=P, table=P, max_pages=2, length=P):
    return B.lib().as_cache4_load(ctypes.byref(c) if c else None, k, v, dtype, lanes, T, table, max_pages, length, None, None)


def _attend(B, c, dtype=0, lanes=2, T=1, q=P, q_ld=512, q_heads=4, table=P, max_pages=2, length=P, scale=1.0, N=1, out=P, work=P, work_bytes=1 << 40):
    return B.lib().as_cache4_attend(ctypes.byref(c) if c else None, q, q_ld, dtype, lanes, T, q_heads, table, max_pages, length, scale, N, None, out,
                                    None, None, work, work_bytes, None)


@pytest.mark.parametrize("call", [_append, _load, _attend])
def test_cache_refusals(B, call):
    for kw, code in CACHE_BAD:
        assert call(B, _cache(B, **kw)) == (B.ERR_INVALID_ARG if code == "inv" else B.ERR_UNSUPPORTED), kw
    assert call(B, None) == B.ERR_INVALID_ARG
    c = _cache(B)
    for kw in (dict(dtype=5), dict(lanes=-1), dict(T=0), dict(table=None), dict(length=None), dict(max_pages=0)):
        assert call(B, c, **kw) == B.ERR_INVALID_ARG, kw
    assert call(B, c, max_pages=1 << 27) == B.ERR_UNSUPPORTED
    assert call(B, c, lanes=1 << 16, T=1 << 15) == B.ERR_UNSUPPORTED
    assert call(B, c, lanes=0, table=None, length=None) == B.OK


def test_cache_call_specific_refusals(B):
    c = _cache(B)
    for kw in (dict(k_ld=127), dict(v_ld=127), dict(k=None), dict(v=None), dict(k=P + 2), dict(dtype=1, v=P + 1)):
        assert _append(B, c, **kw) == B.ERR_INVALID_ARG, kw
    for kw in (dict(k=None), dict(v=None), dict(k=P + 8)):
        assert _load(B, c, **kw) == B.ERR_INVALID_ARG, kw
    for kw in (dict(q_heads=3), dict(q_heads=0), dict(q_ld=255), dict(scale=float("nan")), dict(scale=float("inf")), dict(N=0), dict(N=3),
               dict(q=None), dict(out=None), dict(q=P + 2), dict(out=P + 8), dict(work=None), dict(work_bytes=0), dict(work=P + 16)):
        assert _attend(B, c, **kw) == B.ERR_INVALID_ARG, kw
    assert B.lib().as_cache4_bytes(4, 2, 64, 32) == 4 * 2 * 2 * 18 * 64
    assert B.lib().as_cache4_bytes(0, 2, 64, 32) == 0


def _fork(B, lanes_in=2, lanes_out=3, max_pages=4, page_size=16, n_pages=8, parent=P, table=P, length=P, ref=P, table_out=P + 512, len_out=P + 1024,
          ref_out=P, data=None, planes=1, stride=128, page_bytes=16, work=P, nbytes=1 << 30):
    return B.lib().as_pages_fork(parent, lanes_in, lanes_out, max_pages, page_size, n_pages, table, length, ref, table_out, len_out, ref_out, data, planes,
                                 stride, page_bytes, None, work, nbytes, None)


def test_page_refusals(B):
    for kw in (dict(lanes_in=-1), dict(lanes_out=-1), dict(max_pages=0), dict(page_size=0), dict(n_pages=0), dict(parent=None), dict(table=None),
               dict(length=None), dict(ref=None), dict(table_out=None), dict(len_out=None), dict(ref_out=None), dict(table_out=P), dict(len_out=P),
               dict(work=None), dict(work=P + 4), dict(nbytes=8), dict(data=P, planes=-1), dict(data=P, page_bytes=8), dict(data=P, page_bytes=24),
               dict(data=P + 4), dict(data=P, stride=40), dict(data=P, planes=2, stride=112)):
        assert _fork(B, **kw) == B.ERR_INVALID_ARG, kw
    assert _fork(B, n_pages=(1 << 20) + 1) == B.ERR_UNSUPPORTED
    assert _fork(B, max_pages=1 << 28) == B.ERR_UNSUPPORTED
    L = B.lib()
    grow = lambda add=P, lanes=2, max_pages=4, page_size=16, n_pages=8, table=P, length=P, ref=P, work=P, nbytes=1 << 30: L.as_pages_grow(
        add, lanes, max_pages, page_size, n_pages, table, length, ref, None, work, nbytes, None)
    for kw in (dict(add=None), dict(lanes=-1), dict(max_pages=0), dict(page_size=0), dict(n_pages=0), dict(table=None), dict(length=None),
               dict(ref=None), dict(work=None), dict(nbytes=0)):
        assert grow(**kw) == B.ERR_INVALID_ARG, kw
    assert grow(lanes=0, add=None) == B.OK
    compact = lambda lanes=2, max_pages=4, n_pages=8, table=P, ref=P, table_out=P, ref_out=P, used=P, data=None, planes=1, stride=128, page_bytes=16, \
        work=P, nbytes=1 << 30: L.as_pages_compact(lanes, max_pages, n_pages, table, ref, table_out, ref_out, used, data, planes, stride, page_bytes,
                                                   work, nbytes, None)
    for kw in (dict(lanes=-1), dict(max_pages=0), dict(n_pages=0), dict(table=None), dict(ref=None), dict(table_out=None), dict(ref_out=None),
               dict(used=None), dict(work=None), dict(nbytes=0), dict(data=P, page_bytes=0)):
        assert compact(**kw) == B.ERR_INVALID_ARG, kw
    assert L.as_pages_work_bytes(-1, 1, 1) == 0 and L.as_pages_work_bytes(1, 1, 1) % 256 == 0


def test_binding_checks_layouts(B):
    import torch
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        B.as_logits_edit(x, seq=torch.zeros(2, 3, dtype=torch.int32))
    with pytest.raises(ValueError):
        B.as_logits_edit(x, seq=torch.zeros(2, 3, dtype=torch.int64), length=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        B.as_logits_edit(x, bias=torch.zeros(7))
    with pytest.raises(ValueError):
        B.as_logits_edit(x, mask=torch.zeros(2, 0, dtype=torch.int32))
    with pytest.raises(ValueError):
        B.as_logits_edit(x, out=torch.zeros(2, 7))
    pages = B.cache4_pages(3, 2, 64, 32, device="cpu")
    assert pages.shape == (3, 2, 2, 18 * 64) and B.cache4_pages(3, 2, 64, 32, planes=5, device="cpu").shape[0] == 5
    table, length = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    k = torch.zeros(1, 4, 2, 64)
    with pytest.raises(ValueError):
        B.as_cache4_append(pages[0], k, k, table, length)
    with pytest.raises(ValueError):
        B.as_cache4_append(pages, k[..., :32], k[..., :32], table, length)
    with pytest.raises(ValueError):
        B.as_cache4_append(pages, k.transpose(1, 2), k.transpose(1, 2), table, length)
    with pytest.raises(ValueError):
        B.as_cache4_append(pages, k, k, table, length, k_scale=torch.ones(3))
    with pytest.raises(ValueError):
        B.as_cache4_attend(pages, k, table[0], length, 1.0)
    with pytest.raises(ValueError):
        B.as_pages_fork(torch.zeros(2, dtype=torch.int32), table, length, torch.zeros(4, dtype=torch.int32), 16, pool=torch.zeros(2, 5, 4))


def test_scratch_sizes_of_shapes_that_are_refused():
    """Sizes whose products leave 32 bits end neither the process nor in a size: 0, as for every shape that the call refuses."""
    import subprocess
    import sys
    code = """
import ctypes
from paper_2210_15458_b200 import binding as B
L = B.lib()
c = lambda **k: ctypes.byref(B.as_cache4(**dict(dict(d_pages=256, n_pages=4, heads=1, head_dim=64, page_size=16), **k)))
f = L.as_cache4_attend_work_bytes
for args in ((1, 65536, 65536, 1), (1, 1 << 30, 4, 1), (1, 1 << 16, 1 << 15, 1), (65536, 65536, 1, 65536), (0, 65536, 1, 65536), (1 << 16, 1 << 15, 1, 1), (3, 1, 1, 2),
             (2, 1, 1, 0), (2, 0, 1, 1), (-1, 1, 1, 1), (2, 1, 0, 1), (2147483647, 1, 2, 2147483647), (0, 1, 1, 1)):
    for dtype in (0, 1):
        assert f(c(), dtype, *args) == 0, args
assert f(c(heads=2), 1, 2, 1, 3, 1) == 0 and f(c(head_dim=96), 1, 2, 1, 2, 1) == 0 and f(c(heads=0), 1, 2, 1, 2, 1) == 0 and f(c(), 7, 2, 1, 2, 1) == 0
assert f(None, 1, 2, 1, 2, 1) == 0
assert f(c(), 1, 2, 1, 2, 1) % 256 == 0 and f(c(), 1, 2, 1, 2, 2) > f(c(), 1, 2, 1, 2, 1) > 0
print("fine")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT)
    assert r.returncode == 0 and r.stdout.strip() == "fine", (r.returncode, r.stderr[-500:])


def test_every_unit_that_keeps_a_record_of_indices_checks_some():
    """A translation unit with a reader of out-of-range indices has indices that are checked, in its own file or its headers."""
    import re
    from paper_2210_15458_b200 import _build
    for name in _build.SOURCES:
        files = [f for f in _build._depends(os.path.join(_build.CSRC, name)) if not f.endswith("as_bounds.cuh")]
        text = "".join(open(f).read() for f in files)
        assert "ASX_BOUNDS_READER(" in text
        sites = re.findall(r"ASX_AT\(", text)
        assert len(sites) >= 3, (name, len(sites))


def test_a_scale_that_is_infinite_in_32_bits_is_refused(B):
    c = _cache(B)
    for scale in (1e39, -1e300, 3.5e38):
        assert _attend(B, c, scale=scale) == B.ERR_INVALID_ARG, scale
        assert b"scale" in B.lib().as_last_error(), scale
