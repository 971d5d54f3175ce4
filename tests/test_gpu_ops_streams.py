"""The operators on streams other than the current one, and a workspace that grows while a graph holds the old one."""
import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


def _inputs(T, V=300, d=96, E=40):
    g = torch.Generator(device="cuda").manual_seed(T)
    ids = torch.randint(-1, V, (T,), device="cuda", generator=g)
    dy = torch.randn((T, d), device="cuda", generator=g).bfloat16()
    return ids, dy, torch.randn((T, E), device="cuda", generator=g)


@pytest.mark.parametrize("raw", [False, True])
def test_a_stream_given(raw):
    """What a call returns belongs to the stream it ran on: blocks of a dropped result are not handed to other work before that
    stream has passed them."""
    emb, router = S.Embedding(300, 96), S.Router(40, 3, score="sigmoid")
    table = torch.randn((300, 96), device="cuda").bfloat16()
    ids, dy, x = _inputs(5000)
    bias = torch.randn(40, device="cuda") * 0.1
    want = [emb.lookup(table, ids), emb.grad(ids, dy), *router.route(x, bias)]
    want.append(router.grad(x, want[2], want[3]))
    side = torch.cuda.Stream()
    s = side.cuda_stream if raw else side
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        got = [emb.lookup(table, ids, stream=s), emb.grad(ids, dy, stream=s), *router.route(x, bias, stream=s)]
        got.append(router.grad(x, got[2], got[3], stream=s))
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    clip = S.GradClip([dy], stream=s)
    norm = clip.norm(1.0, stream=s)
    side.synchronize()
    assert abs(float(norm[0]) - float(dy.double().norm())) <= 1e-5 * float(norm[0])


def test_a_graph_keeps_its_workspace():
    emb = S.Embedding(300, 96)
    ids, dy, _ = _inputs(500)
    want = emb.grad(ids, dy)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = emb.grad(ids, dy)
    for T in (5000, 9000, 60000):                       # the workspace grows twice or more
        i, y, _ = _inputs(T)
        emb.grad(i, y)
    junk = [torch.full((1 << 20,), -1, dtype=torch.int32, device="cuda") for _ in range(8)]  # over what would have been freed
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(junk) == 8


def test_a_routers_first_call_is_not_captured():
    """Its counters are zeroed once: in a graph they would be zeroed only when that runs."""
    _, _, x = _inputs(100)
    router = S.Router(40, 3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = x + 1
        with pytest.raises(S.SkewError) as e:
            router.route(x)
    assert e.value.code == S.SKEW_ESTATE
    graph.replay()
    chosen, _, counts = router.route(x)
    assert int(counts.sum()) == 300 and torch.equal(torch.bincount(chosen.reshape(-1).long(), minlength=40), counts.long())
    assert torch.equal(y, x + 1)
