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

    made, recorded = 0, []

    def __init__(self, shape, dtype=torch.bfloat16, index=0):
        self.shape, self.dtype, self.device, self.is_cuda = torch.Size(shape), dtype, torch.device("cuda", index), True
        FakeTensor.made += 1
        self.at = FakeTensor.made << 20

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at

    def __getitem__(self, part):
        return self

    def record_stream(self, stream):
        FakeTensor.recorded.append((self.at, stream.cuda_stream))

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

    def fake(name):
        def make(shape, dtype=None, device=None):
            seen.append((name, current[-1]))
            device = torch.device(device)
            return FakeTensor((shape,) if isinstance(shape, int) else shape, dtype, device.index or 0)
        return make

    monkeypatch.setattr(S, "_on", on)
    monkeypatch.setattr(S, "_raw_stream", lambda: lambda index: current[-1])
    monkeypatch.setattr(torch, "empty", fake("empty"))
    monkeypatch.setattr(torch, "zeros", fake("zeros"))
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


def _objects(monkeypatch):
    """One of each class, that launch into a list."""
    launched = []
    launch = lambda *a: launched.append(a) or 0  # noqa: E731
    emb, router = S.Embedding(10, 8), S.Router(8, 2)
    for o in (emb, router):
        o._new = lambda shape, strides, dtype, device: FakeTensor(shape, dtype, device.index)
    emb._lookup = emb._grad = router._forward = router._grad = launch
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    clip = S.GradClip([FakeTensor((100,))])
    clip._norm = clip._apply = launch
    return launched, clip, emb, router


def _calls(clip, emb, router):
    """Each class's calls on stand-ins for tensors of device 0."""
    ids, table, dy = FakeTensor((5,), torch.int64), FakeTensor((10, 8)), FakeTensor((5, 8))
    x, chosen, dw = FakeTensor((5, 8)), FakeTensor((5, 2), torch.int32), FakeTensor((5, 2), torch.float32)
    return [lambda: clip.norm(1.0), lambda: clip.clip(1.0), lambda: emb.lookup(table, ids), lambda: emb.grad(ids, dy),
            lambda: router.route(x), lambda: router.grad(x, chosen, dw), lambda: S.GradClip([FakeTensor((100,))])]


def test_tensors_of_another_device_are_refused(world, monkeypatch):
    """Their stream may be the default one, whose handle is the current device's too: a launch would run there on the others' pointers."""
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
    current = [0]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    launched, *objects = _objects(monkeypatch)
    calls = _calls(*objects)
    for k, call in enumerate(calls):
        call()
        assert len(launched) == min(k + 1, 6)
    current[0] = 1
    for o in (launched, world):
        o.clear()
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()
    assert not launched and not world


def test_a_workspace_for_each_device(world, monkeypatch):
    """A graph may hold each of them, so none is dropped for another device's; and they grow with the tokens alone."""
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
    current = [0]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    launched, _, emb, router = _objects(monkeypatch)
    world.clear()
    at = {0: set(), 1: set()}
    for k in range(20):
        current[0] = d = k % 2
        emb.grad(FakeTensor((5,), torch.int64, d), FakeTensor((5, 8), index=d))
        at[d].add(launched[-1][7])
        router.route(FakeTensor((5, 8), index=d))
        at[d].add(launched[-1][8])
    assert sorted(name for name, _ in world) == ["empty"] * 2 + ["zeros"] * 2
    assert len(at[0]) == len(at[1]) == 2 and not at[0] & at[1]


class FakeStream:
    def __init__(self, handle, stream_id=3):
        self.cuda_stream, self.stream_id = handle, stream_id


def test_memory_that_other_streams_use_is_not_given_away(world, monkeypatch):
    """Each block that an object keeps is recorded, once, on every stream of torch's that uses it beside its own."""
    now = [FakeStream(100)]
    monkeypatch.setattr(S, "_raw_stream", lambda: lambda index: now[0].cuda_stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[0])

    @contextlib.contextmanager
    def on(stream):
        before, now[0] = now[0], stream if hasattr(stream, "cuda_stream") else FakeStream(stream, stream)
        yield
        now[0] = before

    monkeypatch.setattr(S, "_on", on)
    launched, clip, emb, router = _objects(monkeypatch)
    ids, dy, x = FakeTensor((5,), torch.int64), FakeTensor((5, 8)), FakeTensor((5, 8))
    both = lambda s=None: (clip.norm(1.0, stream=s), clip.clip(1.0, stream=s), emb.grad(ids, dy, stream=s), router.route(x, stream=s))  # noqa: E731
    both()
    FakeTensor.recorded.clear()
    own = {clip.workspace.at, clip.result.at, launched[-2][7], launched[-1][8]}
    assert len(own) == 4
    for _ in range(3):
        both()
        both(FakeStream(200))
        now[0] = FakeStream(300)
        both()
        now[0] = FakeStream(0, 0)   # the default stream
        both()
        both(400)                   # a raw handle: not torch's to ask later
        now[0] = FakeStream(100)
    assert sorted(FakeTensor.recorded) == sorted((at, h) for at in own for h in (200, 300, 0))
    emb.grad(FakeTensor((5000,), torch.int64), FakeTensor((5000, 8)))  # a larger workspace: a new block
    emb.grad(ids, dy, stream=FakeStream(200))
    assert FakeTensor.recorded[-1] == (launched[-1][7], 200) and launched[-1][7] not in own


def test_the_step_takes_its_buffers_on_the_stream_given(world, monkeypatch):
    monkeypatch.setattr(S, "skew_bind", lambda h, state, n, ws, m, stream: world.append(("bind", stream)))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: FakeStream("current"))
    params = [(FakeTensor((16, 8)), FakeTensor((16, 8)), S.TIER_BACKBONE)]
    for stream, want in ((7, 7), (None, "current")):
        world.clear()
        S.SkewAdam(params, S.hparams(), stream=stream)
        assert world == [("empty", want), ("empty", want), ("bind", want)]


def test_the_step_refuses_tensors_of_another_device(world, monkeypatch):
    stepped, current = [], [0]
    monkeypatch.setattr(S, "skew_bind", lambda *a: None)
    monkeypatch.setattr(S, "skew_step", lambda *a: stepped.append(a))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: FakeStream(5))
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    params = [(FakeTensor((16, 8)), FakeTensor((16, 8)), S.TIER_BACKBONE)]
    opt = S.SkewAdam(params, S.hparams())
    opt.step(1, 1e-3, 5)
    assert len(stepped) == 1
    current[0] = 1
    world.clear()
    with pytest.raises(ValueError, match="current device"):
        opt.step(2, 1e-3, 5)
    with pytest.raises(ValueError, match="current device"):
        S.SkewAdam(params, S.hparams())
    assert len(stepped) == 1 and not world
