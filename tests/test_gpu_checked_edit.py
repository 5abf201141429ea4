"""Logit edits in the build that checks every shared-memory index, with guard words around the output."""
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture()
def B():
    from paper_2210_15458_b200 import _build, binding
    if not os.path.exists(_build.LIB_CHECKED):
        pytest.skip("checked build not there")
    binding.use_library(_build.LIB_CHECKED)
    yield binding
    binding.use_library(None)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lanes,V,T,off", [(1, 1, 3, 0), (3, 7, 9, 1), (2, 2047, 100, 3), (2, 2049, 100, 0), (3, 8200, 500, 5), (300, 8193, 60, 2)])
def test_no_index_leaves_its_array(B, dtype, lanes, V, T, off):
    g = torch.Generator().manual_seed(V)
    raw = torch.full((off + lanes * V + 64,), 7.0, dtype=dtype, device="cuda")
    x = torch.randn(off + lanes * V, generator=g).to(dtype).cuda()[off:].view(lanes, V)
    seq = torch.randint(-1, V + 1, (lanes, T), generator=g, dtype=torch.int32).cuda()
    length = torch.randint(0, T + 1, (lanes,), generator=g, dtype=torch.int32).cuda()
    bias = torch.randn(V, generator=g).cuda()
    mask = torch.randint(-2**31, 2**31 - 1, (1, -(-V // 32)), generator=g, dtype=torch.int64).to(torch.int32).cuda()
    B.as_debug_bounds(reset=True)
    out = raw[off:off + lanes * V].view(lanes, V)
    B.as_logits_edit(x, seq, length, None, 1.3, 0.2, 0.1, bias, mask, out=out)
    checked = out.clone()
    torch.cuda.synchronize()
    assert B.as_debug_bounds(reset=True)[0] == 0
    assert (raw[:off] == 7).all() and (raw[off + lanes * V:] == 7).all()
    B.use_library(None)
    assert torch.equal(B.as_logits_edit(x, seq, length, None, 1.3, 0.2, 0.1, bias, mask), checked)
