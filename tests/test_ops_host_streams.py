"""Where the wrappers' buffers come from when a stream is given, host side: stand-ins for tensors and streams, nothing is launched."""
import contextlib

import pytest
import torch

from paper_2607_19058_gb300 import _build
from paper_2607_19058_gb300 import skewadam as S


@pytest.fixture(scope="module", autouse=True)
def lib():
    _build.build()
    return S.load()


class FakeTensor:
    """What the wrappers ask a CUDA tensor for."""

    def __init__(self, shape, dtype=torch.bfloat16, index=0):
        self.shape, self.dtype, self.device, self.is_cuda = torch.Size(shape), dtype, torch.device("cuda", index), True

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x10000

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)


@pytest.fixture
def world(monkeypatch):
    """A list of what happens: ("empty" or "zeros" or "bind", the stream that is current or bound on)."""
    seen, current = [], ["current"]

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    def fake(name, real):
        def make(shape, dtype=None, device=None, **kw):
            seen.append((name, current[-1]))
            return real(shape, dtype=dtype)
        return make

    monkeypatch.setattr(S, "_on", on)
    monkeypatch.setattr(S, "_raw_stream", lambda: lambda index: current[-1])
    monkeypatch.setattr(torch, "empty", fake("empty", torch.empty))
    monkeypatch.setattr(torch, "zeros", fake("zeros", torch.zeros))
    monkeypatch.setattr(S, "skew_clip_bind", lambda h, ws, n, stream: seen.append(("bind", stream)))
    return seen


def test_clip_takes_its_buffers_on_the_stream_given(world):
    """The stream that fills and reads them: another one's zero-fill could come after the norm, and a block of another one's
    pool may still be written to by what is queued there."""
    S.GradClip([FakeTensor((100,))], stream=7)
    assert [name for name, _ in world][-1] == "bind" and {stream for _, stream in world} == {7}
    world.clear()
    S.GradClip([FakeTensor((100,))])
    assert [name for name, _ in world][-1] == "bind" and {stream for _, stream in world} == {"current"}
