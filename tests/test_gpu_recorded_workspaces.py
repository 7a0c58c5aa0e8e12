"""Calls of RolloutStage that are recorded: replays stay right, and write into nobody's memory, whatever is called on the recording stream afterwards; two graphs recorded
on one stream may run side by side."""
import pytest
import torch

from nat_testlib import DEV

pytestmark = pytest.mark.gpu


def rand(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def attention(g, size):
    n = 4000 * size
    q, k, v = rand(g, 24, 8, 64), rand(g, n, 2, 64), rand(g, n, 2, 64)
    cu_q, cu_k = (torch.tensor([0, x], dtype=torch.int32, device=DEV) for x in (24, n))
    return q, lambda stage: stage.attention(q, k, v, cu_q, cu_k)


def backward(g, size):
    n = 800 * size
    q, k, v, do = rand(g, n, 8, 64), rand(g, n, 1, 64), rand(g, n, 1, 64), rand(g, n, 8, 64)
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)

    def call(stage):
        out, lse = stage.attention(q, k, v, cu)
        return (out, lse, *stage.attention_backward(do, q, k, v, out, lse, cu))
    return do, call


def decode(g, size):
    from paper_2603_06619_amd.rollout import PagedCache, RolloutStage
    pages = 40 * size
    cache = PagedCache.empty(pages, 2, 64, 64, False, DEV)
    k = rand(g, pages * 64, 2, 64)
    RolloutStage(DEV).write_cache(cache, k, k.flip(0), torch.arange(pages * 64, device=DEV))
    q, table = rand(g, 1, 8, 64), torch.randperm(pages, device=DEV).to(torch.int32).view(1, pages)
    lens = torch.tensor([pages * 64 - 5], dtype=torch.int32, device=DEV)
    return q, lambda stage: stage.decode(q, cache, table, lens)


def sample(g, size):
    z = 2 * rand(g, 4 * size, 60007, dtype=torch.float32)
    w = torch.randint(-2 ** 31, 2 ** 31, (4 * size,), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    kw = dict(top_k=torch.full((4 * size,), 30, dtype=torch.int32, device=DEV), top_p=torch.full((4 * size,), 0.9, device=DEV))
    return z, lambda stage: tuple(stage.sample(z, w, **kw).values())


KINDS = [attention, backward, decode, sample]


def record(stage, side, call):
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(stage)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = call(stage)
    torch.cuda.synchronize()
    return graph, out


@pytest.mark.parametrize("kind", KINDS)
def test_a_larger_call_after_recording(kind):
    from paper_2603_06619_amd.rollout import RolloutStage
    stage, fresh, side = RolloutStage(DEV), RolloutStage(DEV), torch.cuda.Stream()
    g = torch.Generator(device=DEV).manual_seed(1)
    x, call = kind(g, 1)
    _, larger = kind(g, 3)
    graph, out = record(stage, side, call)
    sizes = sorted({t.numel() for t in stage._ws.values()})
    assert sizes                                                   # the warm-up had a workspace
    with torch.cuda.stream(side):
        larger(stage)
        theirs = [torch.full((n // 4,), 123456789, dtype=torch.int32, device=DEV) for n in sizes for _ in range(3)]      # where replaced workspaces lay
    torch.cuda.synchronize()
    for _ in range(3):
        x.copy_(torch.randn(x.shape, device=DEV))
        want = call(fresh)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
        assert all(bool((t == 123456789).all()) for t in theirs)


@pytest.mark.parametrize("kind", KINDS)
def test_two_graphs_of_one_stream_side_by_side(kind):
    from paper_2603_06619_amd.rollout import RolloutStage
    stage, fresh, side, other = RolloutStage(DEV), RolloutStage(DEV), torch.cuda.Stream(), torch.cuda.Stream()
    g = torch.Generator(device=DEV).manual_seed(2)
    cases = [kind(g, 1), kind(g, 1)]
    graphs = [record(stage, side, call) for _, call in cases]
    wants = [call(fresh) for _, call in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (graph, _) in zip((side, other), graphs):
            with torch.cuda.stream(s):
                graph.replay()
        eager = cases[0][1](stage)
        torch.cuda.synchronize()
        for (_, out), want in zip(graphs, wants):
            for a, b in zip(out, want):
                assert torch.equal(a, b)
        for a, b in zip(eager, wants[0]):
            assert torch.equal(a, b)


def test_a_larger_loss_call_after_recording():
    """Log-probs of the loss stage, whose workspace a larger call replaces."""
    from paper_2603_06619_amd.stage import LossStage
    stage, fresh, side = LossStage(DEV), LossStage(DEV), torch.cuda.Stream()
    g = torch.Generator(device=DEV).manual_seed(3)
    W = rand(g, 5000, 256) * 0.1
    hidden, ids = rand(g, 300, 256), torch.randint(0, 5000, (300,), generator=g, device=DEV).to(torch.int32)
    more, more_ids = rand(g, 3000, 256), torch.randint(0, 5000, (3000,), generator=g, device=DEV).to(torch.int32)
    graph, out = record(stage, side, lambda s: s.logp(hidden, W, ids, 300)["logp"])
    size = stage._ws["loss"].numel()
    with torch.cuda.stream(side):
        stage.logp(more, W, more_ids, 3000)
        assert stage._ws["loss"].numel() > size
        theirs = [torch.full((size // 4,), 123456789, dtype=torch.int32, device=DEV) for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(3):
        hidden.copy_(torch.randn(hidden.shape, device=DEV))
        want = fresh.logp(hidden, W, ids, 300)["logp"]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(bool((t == 123456789).all()) for t in theirs)
