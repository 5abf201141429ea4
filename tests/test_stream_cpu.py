"""Which stream the binding's own allocations belong to, without a device: the library is a stand-in that accepts every call."""
import contextlib

import pytest

torch = pytest.importorskip("torch")
from torch.utils._python_dispatch import TorchDispatchMode  # noqa: E402


class Library:
    """Every call succeeds and every size is 4096 bytes."""

    def __getattr__(self, name):
        return lambda *a: 4096 if name.endswith("_bytes") else 0


class Allocations(TorchDispatchMode):
    """Records, for every allocation, the stream that is current in `at`."""

    def __init__(self, at):
        super().__init__()
        self.at, self.seen = at, []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        if func._schema.name.split("::")[1] in ("empty", "new_empty", "empty_like", "empty_strided", "new_empty_strided"):
            self.seen.append(self.at[-1])
        return func(*args, **(kwargs or {}))


@pytest.fixture()
def B(monkeypatch):
    from paper_2210_15458_b200 import binding
    monkeypatch.setattr(binding, "_lib", Library())
    monkeypatch.setattr(binding, "lib", lambda: binding._lib)
    current = [None]

    @contextlib.contextmanager
    def stream(s):
        current.append(s)
        yield
        current.pop()
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda raw, device=None: ("external", raw))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: ("default",))
    monkeypatch.setattr(binding, "_current_stream", lambda: 96)
    return binding, current


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def calls(B):
    x, seq, lens = torch.zeros(2, 40), i32(2, 4), i32(2)
    pages, table = B.cache4_pages(3, 2, 64, 16, device="cpu"), i32(2, 2)
    k = torch.zeros(2, 1, 2, 64)
    ref = i32(3)
    return {"edit": (1, lambda **s: B.as_logits_edit(x, seq, lens, **s)),
            "load": (2, lambda **s: B.as_cache4_load(pages, table, lens, 1, **s)),
            "attend": (2, lambda **s: B.as_cache4_attend(pages, k, table, lens, 1.0, **s)),
            "fork": (4, lambda **s: B.as_pages_fork(i32(2), table, lens, ref, 16, **s)),
            "grow": (1, lambda **s: B.as_pages_grow(lens, table, lens, ref, 16, **s)),
            "compact": (2, lambda **s: B.as_pages_compact(table, ref, **s))}


@pytest.mark.parametrize("name", ["edit", "load", "attend", "fork", "grow", "compact"])
def test_scratch_and_outputs_belong_to_the_stream_of_the_launch(B, name):
    """Outputs and scratch that a call allocates come from the launch stream's memory: the block of a scratch tensor that is
    dropped on return may only go to later work of the same stream."""
    binding, current = B
    n, call = calls(binding)[name]
    for given, want in ((7 << 4, ("external", 7 << 4)), (0, ("default",)), (type("S", (), {"cuda_stream": 48})(), ("external", 48))):
        with Allocations(current) as a:
            call(stream=given)
        assert a.seen == [want] * n
    for same in (None, 96):                             # the current stream, named or not: nothing to switch
        with Allocations(current) as a:
            call(stream=same)
        assert a.seen == [None] * n


def test_the_current_stream_by_public_names_alone(monkeypatch):
    """A torch without the two unlisted look-ups: the public one gives the same handle."""
    import importlib
    from paper_2210_15458_b200 import binding
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    monkeypatch.delattr(torch._C, "_cuda_getDevice")
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: type("S", (), {"cuda_stream": 4242})())
    spec = importlib.util.spec_from_file_location("paper_2210_15458_b200.binding_again", binding.__file__)
    again = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(again)
    assert again._stream(None) == 4242 and again._current_stream() == 4242
