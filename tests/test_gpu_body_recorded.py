"""Calls of the embedding, of norms and rotation and of page tables that are recorded: every replay, with other inputs and the program's own work between, gives what an eager call
gives, bit for bit; two graphs recorded on one stream may run side by side; calls on several streams at once."""
import pytest
import torch

from nat_testlib import DEV

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def ints(g, low, high, *shape):
    return torch.randint(low, high, shape, generator=g, device=DEV, dtype=torch.int64).to(torch.int32)


def heads(g, n):
    D, new = 64, lambda *s: torch.randn(s, generator=g, device=DEV).bfloat16()
    t = dict(q=new(n, 6, D), k=new(n, 2, D), dq_out=new(n, 6, D), dk_out=new(n, 2, D), q_weight=new(D), k_weight=new(D), position_ids=ints(g, 0, 9000, n))
    freq = 1e4 ** (-torch.arange(D // 2, dtype=torch.float64, device=DEV) / 32)

    def call(stage):
        kw = dict(q=t["q"], k=t["k"], position_ids=t["position_ids"], inv_freq=freq, q_weight=t["q_weight"], k_weight=t["k_weight"])
        return *stage.norm_rotate(**kw), *stage.norm_rotate_backward(t["dq_out"], t["dk_out"], **kw)
    return t, call


def embedding(g, n):
    V, H = 3000, 72
    t = dict(E=torch.randn((V, H), generator=g, device=DEV), dout=torch.randn((n, H), generator=g, device=DEV).bfloat16(), ids=ints(g, -2, V + 2, n))
    t["ids"][::3] = 7

    def call(stage):
        out = stage.embed(t["ids"], t["E"], 0.5)
        total = stage.embed_backward(t["dout"], t["ids"], V)
        return out, total, stage.embed_backward(out, t["ids"], V, 2.0, dE=total.clone(), accumulate=True)
    return t, call


def pages(g, n):
    page, width = 16, 40
    n_pages = 12 * n
    table = torch.randperm(n * width, generator=g, device=DEV).to(torch.int32).view(n, width) % n_pages
    t = dict(lens=ints(g, 0, 300, n), new=ints(g, 0, 200, n), keep=ints(g, 0, 400, n), free=torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32),
             counts=torch.tensor([7 * n, 0], dtype=torch.int32, device=DEV), table=table)

    def call(stage):
        table, free = t["table"].clone(), t["free"].clone()
        lens, counts = stage.release(table, t["lens"], t["keep"], free, t["counts"], page)
        return (*stage.reserve(table, lens, t["new"], free, counts, page, 200 * n).values(), lens, counts, table, free)
    return t, call


KINDS = [heads, embedding, pages]


def record(stage, side, call):
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(stage)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = call(stage)
    torch.cuda.synchronize()
    return graph, out


def refill(t, other):
    for name, x in t.items():
        x.copy_(other[name])


@pytest.mark.parametrize("size", [50, 9000])
@pytest.mark.parametrize("kind", KINDS)
def test_replays(kind, size):
    from paper_2603_06619_amd.rollout import RolloutStage
    if kind is pages:
        size //= 50                               # sequences: 1 and 180
    stage, fresh, side = RolloutStage(DEV), RolloutStage(DEV), torch.cuda.Stream()
    t, call = kind(gen(1), size)
    _, larger = kind(gen(2), 3 * size)
    graph, out = record(stage, side, call)
    with torch.cuda.stream(side):
        larger(stage)                             # takes and replaces the stream's workspaces
        sizes = sorted({w.numel() for w in stage._ws.values()})
        theirs = [torch.full((b // 4,), 123456789, dtype=torch.int32, device=DEV) for b in sizes for _ in range(3)]
    torch.cuda.synchronize()
    for rep in range(4):
        refill(t, kind(gen(10 + rep), size)[0])
        want = call(fresh)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), rep
        assert all(bool((x == 123456789).all()) for x in theirs)


@pytest.mark.parametrize("kind", KINDS)
def test_two_graphs_and_an_eager_call_side_by_side(kind):
    from paper_2603_06619_amd.rollout import RolloutStage
    size = 60 if kind is pages else 9000
    stage, fresh, side, other = RolloutStage(DEV), RolloutStage(DEV), torch.cuda.Stream(), torch.cuda.Stream()
    cases = [kind(gen(20 + i), size) for i in range(3)]
    want = [call(fresh) for _, call in cases]
    graphs = [record(stage, side, call) for _, call in cases[:2]]
    torch.cuda.synchronize()
    for _ in range(4):
        with torch.cuda.stream(side):
            graphs[0][0].replay()
        with torch.cuda.stream(other):
            graphs[1][0].replay()
        mine = cases[2][1](stage)
        torch.cuda.synchronize()
        for got, ref in zip((graphs[0][1], graphs[1][1], mine), want):
            assert all(torch.equal(a, b) for a, b in zip(got, ref))


@pytest.mark.parametrize("kind", KINDS, ids=lambda f: f.__name__)
def test_tensors_of_another_device_are_refused(kind, monkeypatch):
    """A kernel is launched on the current device, which tensors elsewhere may not be reached from (the device is named here only)."""
    from paper_2603_06619_amd.rollout import RolloutStage
    stage = RolloutStage(DEV)
    _, call = kind(gen(3), 20)
    call(stage)
    here = torch.cuda.current_device()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: here + 1)
    with pytest.raises(ValueError, match="current device"):
        call(stage)
