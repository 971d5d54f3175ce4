"""The operators on a stream of their own while much work is still queued on the current one."""
import math

import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


def _queue(busy, passes=200):
    """Some tens of milliseconds of ordinary work on the current stream."""
    for _ in range(passes):
        busy.mul_(1.0)


@pytest.mark.parametrize("raw", [False, True])
def test_clip_beside_a_backlog(raw):
    """What is queued on the current stream, a write to a block that has been given back among it, touches neither the table nor the result."""
    g = torch.randn(300000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()
    want = float(g.double().norm())
    busy = torch.ones(1 << 28, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    _queue(busy)
    for n in (512, 1 << 16, 1 << 17, 1 << 18, 1 << 20):  # blocks of the sizes that a clip takes
        torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
    clip = S.GradClip([g], stream=side.cuda_stream if raw else side)
    clip.norm(1.0, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    norm, gamma = clip.result.tolist()
    assert abs(norm - want) <= 1e-5 * want and math.isclose(gamma, 1.0 / want, rel_tol=1e-5)
    with torch.cuda.stream(side):
        clip.norm(1.0)
    torch.cuda.synchronize()
    assert clip.result.tolist() == [norm, gamma]


def test_a_dropped_object_keeps_its_memory_until_its_work_is_done():
    """Work queued on another stream than the one that a workspace was allocated on still counts in it: new tensors of the
    first stream lie elsewhere. (They are allocated and not written.)"""
    T, E, V, d = 5000, 40, 300, 96
    x, ids = torch.randn((T, E), device="cuda"), torch.randint(0, V, (T,), device="cuda")
    dy = torch.randn((T, d), device="cuda").bfloat16()
    busy = torch.ones(1 << 28, device="cuda")
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    assert side.stream_id != side.cuda_stream and torch.cuda.ExternalStream(other.cuda_stream).stream_id == other.cuda_stream
    clip, emb, router = S.GradClip([dy]), S.Embedding(V, d), S.Router(E, 3)
    call = lambda s=None: (clip.norm(1.0, stream=s), emb.grad(ids, dy, stream=s), router.route(x, stream=s))  # noqa: E731
    call()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        _queue(busy)
    call(side)
    call(other.cuda_stream)
    blocks = [clip.workspace, clip.result, *(next(iter(o._workspaces.values())).tensor for o in (emb, router))]
    sizes, at = [b.untyped_storage().nbytes() for b in blocks], {b.data_ptr() for b in blocks}
    other.synchronize()
    del clip, emb, router, call, blocks
    new = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
    assert not at & {t.data_ptr() for t in new}
    torch.cuda.synchronize()


def test_the_default_streams_handle():
    """0 is the default stream's handle: given for each object and call, and for the optimizer."""
    g = torch.randn(5000, device="cuda").bfloat16().view(50, 100)
    clip = S.GradClip([g], stream=0)
    norm = clip.norm(1.0, stream=0)
    want = float(g.double().norm())
    assert abs(float(norm[0]) - want) <= 1e-5 * want
    ids = torch.arange(50, device="cuda")
    assert torch.equal(S.Embedding(50, 100).lookup(g, ids, stream=0), g)
    chosen, _, counts = S.Router(4, 1).route(torch.zeros((30, 4), device="cuda"), stream=0)
    assert counts.tolist() == [30, 0, 0, 0] and int(chosen.abs().max()) == 0
    w = [torch.ones_like(g) for _ in range(2)]
    for t, stream in zip(w, (0, None)):
        opt = S.SkewAdam([(t, g, S.TIER_BACKBONE)], S.hparams(), stream=stream)
        opt.step(1, 1e-2, 3, stream=stream)
        opt.sync_status(stream=stream)
    assert torch.equal(*w) and not torch.equal(w[0], torch.ones_like(g))
