"""nat_sample where several workgroups share a row (few rows of a large vocabulary): as the oracle draws, with the limits of test_gpu_sample.py, and the same
tokens as one workgroup per row draws."""
import math

import numpy as np
import pytest
import torch

from nat_testlib import DEV
from test_gpu_sample import K, M, P, T, check, draw, stage, words_of  # noqa: F401 (stage is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V,sigma", [(1, 45057, 2.0), (9, 50257, 1.0), (4, 65543, 6.0), (3, 100003, 0.3), (100, 81929, 2.0)])
def test_draws(stage, dtype, n, V, sigma):  # noqa: F811
    rng = np.random.default_rng(V)
    z = torch.from_numpy((rng.standard_normal((n, V), dtype=np.float32) * np.float32(sigma))).to(dtype).to(DEV)
    w = words_of(rng, n)
    pick = lambda x: rng.choice(x, n)
    for kw in (dict(), dict(temperature=pick(T), top_k=pick(K), top_p=pick(P), min_p=pick(M)), dict(top_k=pick([1000, 3000, 20000]), top_p=pick([0.5, 1.0]))):
        check(z, w, draw(stage, z, w, **kw), **kw)
        if n > 9:
            break


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_equal_logits_masks_and_not_finite(stage, dtype):  # noqa: F811
    inf, nan, V, n = math.inf, math.nan, 45003, 12
    rng = np.random.default_rng(1)
    z = rng.integers(-3, 3, (n, V)).astype(np.float32)            # lists of thousands of equal logits, longer than a workgroup keeps
    z[0] = 0.0
    z[1] = -inf
    z[2] = nan
    z[3, : V - 1] = -inf
    z[4, 5] = nan
    z[5, 77] = z[5, 40000] = inf
    z[6] = np.where(rng.random(V) < 0.5, -0.0, 0.0)
    z[7] = np.finfo(np.float32).min
    z[7, 40000:40100] = 1.0
    z[8] = np.finfo(np.float32).min
    z[9, :] = -inf
    z[9, 123] = -1e30
    z = torch.from_numpy(z).to(dtype).to(DEV)
    w = words_of(rng, n)
    pick = lambda x: rng.choice(x, n)
    for kw in (dict(), dict(top_k=pick([1, 2, 777, 4500, 45002])), dict(top_p=pick([0.0, 0.2, 0.77, 0.99])),
               dict(top_k=pick([3, 3000]), top_p=pick([0.3, 0.9]), min_p=pick([0.0, 0.2])), dict(temperature=pick(T), top_k=pick(K), top_p=pick(P))):
        check(z, w, draw(stage, z, w, **kw), **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_row_alone_and_among_many(stage, dtype):  # noqa: F811
    """300 rows take one workgroup each; the first of them alone, at other places in memory, many: the same tokens and weights, whose sums are whole numbers."""
    V, n = 70001, 300
    g = torch.Generator(device=DEV).manual_seed(4)
    z = (2 * torch.randn((n, V), generator=g, device=DEV)).to(dtype)
    rng = np.random.default_rng(5)
    w = words_of(rng, n)
    kw = dict(temperature=rng.choice([1.0, 0.7], n), top_k=rng.choice([0, 0, 40, 1500], n), top_p=rng.choice([0.9, 0.99, 1.0], n), min_p=rng.choice([0.0, 0.01], n))
    many = draw(stage, z, w, **kw)
    for lead, rows in ((0, 1), (3, 7), (7, 4), (1, 2)):
        whole = torch.full((rows, V + 11), 1000.0, dtype=dtype, device=DEV)
        part = whole[:, lead:lead + V]
        part.copy_(z[:rows])
        few = draw(stage, part, w[:rows], **{k: x[:rows] for k, x in kw.items()})
        for name in ("ids", "logq"):
            assert np.array_equal(few[name], many[name][:rows]), (lead, rows, name)
        assert np.all(np.abs(few["logp"] - many["logp"][:rows]) <= 2e-6 * (1 + np.abs(many["logp"][:rows])))


def test_graph_and_streams(stage):  # noqa: F811
    """Recorded once and replayed on new logits, with other calls between; and on two streams at once, whose workspaces are their own."""
    V, n = 60007, 5
    g = torch.Generator(device=DEV).manual_seed(6)
    new = lambda: 2 * torch.randn((n, V), generator=g, device=DEV)
    w = torch.randint(-2 ** 31, 2 ** 31, (n,), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    kw = dict(top_k=torch.full((n,), 30, dtype=torch.int32, device=DEV), top_p=torch.full((n,), 0.9, device=DEV))
    z, other = new(), new()
    want_other = stage.sample(other, w, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        stage.sample(z, w, **kw)                             # the workspace of this stream
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = stage.sample(z, w, **kw)
    for _ in range(4):
        z.copy_(new())
        want = stage.sample(z, w, **kw)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph.replay()
        beside = stage.sample(other, w, **kw)
        torch.cuda.synchronize()
        for name in want:
            assert torch.equal(out[name], want[name]) and torch.equal(beside[name], want_other[name])
