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
