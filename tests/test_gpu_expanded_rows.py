"""Inputs expanded along their rows give, bit for bit, what the same values in rows of their own give; the memory behind the one stored row has no influence."""
import pytest
import torch

from nat_testlib import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def stage():
    from paper_2603_06619_amd.rollout import RolloutStage
    return RolloutStage(DEV)


def one_row(g, n, *shape, dtype=torch.bfloat16):
    """A row expanded to n, in front of memory that holds NaN."""
    whole = torch.full((n, *shape), float("nan"), dtype=dtype, device=DEV)
    whole[0] = torch.randn(shape, generator=g, device=DEV, dtype=dtype)
    return whole[:1].expand(n, *shape)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name", ["q", "k", "v", "dout"])
def test_attention(stage, D, name):
    g = torch.Generator(device=DEV).manual_seed(D)
    n, hq, hkv = 150, 6, 2
    c = {x: torch.randn((n, hkv if x in "kv" else hq, D), generator=g, device=DEV, dtype=torch.bfloat16) for x in ("q", "k", "v", "dout")}
    cu = torch.tensor([0, 100, n], dtype=torch.int32, device=DEV)

    def run(c):
        out, lse = stage.attention(c["q"], c["k"], c["v"], cu)
        return (out, lse, *stage.attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, cu))
    c[name] = one_row(g, n, *c[name].shape[1:])
    got = run(c)
    want = run({x: t.contiguous() for x, t in c.items()})
    for a, b in zip(got, want):
        assert torch.equal(a, b) and bool(torch.isfinite(a.float()).all()) and a.stride() == b.stride()


def test_gradient_of_a_sum(stage):
    """dout as autograd hands it on from a sum over rows and elements: one number for all."""
    g = torch.Generator(device=DEV).manual_seed(3)
    q, k, v = (torch.randn((70, h, 64), generator=g, device=DEV, dtype=torch.bfloat16) for h in (4, 2, 2))
    cu = torch.tensor([0, 70], dtype=torch.int32, device=DEV)
    out, lse = stage.attention(q, k, v, cu)
    dout = torch.ones((), dtype=torch.bfloat16, device=DEV).expand(out.shape)
    for a, b in zip(stage.attention_backward(dout, q, k, v, out, lse, cu), stage.attention_backward(dout.contiguous(), q, k, v, out, lse, cu)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("fp8", [True, False])
def test_cache_and_decoding(stage, fp8):
    from paper_2603_06619_amd.rollout import PagedCache
    g = torch.Generator(device=DEV).manual_seed(5)
    k, v = one_row(g, 40, 2, 64), one_row(g, 40, 2, 64)
    caches = []
    for kk, vv in ((k, v), (k.contiguous(), v.contiguous())):
        cache = PagedCache.empty(5, 2, 16, 64, fp8, DEV)
        for x in (cache.k, cache.v, cache.k_exp, cache.v_exp):
            if x is not None:
                x.view(torch.uint8).fill_(0x11)
        stage.write_cache(cache, kk, vv, torch.arange(40, device=DEV))
        caches.append(cache)
    for x in ("k", "v", "k_exp", "v_exp") if fp8 else ("k", "v"):
        assert torch.equal(*(getattr(c, x).view(torch.uint8) for c in caches)), x
    q = one_row(g, 3, 4, 64)                                # one query for several sequences
    table = torch.tensor([[0, 1, 2], [2, 1, 0], [1, 0, 3]], dtype=torch.int32, device=DEV)
    lens = torch.tensor([40, 20, 33], dtype=torch.int32, device=DEV)
    for a, b in zip(stage.decode(q, caches[0], table, lens), stage.decode(q.contiguous(), caches[0], table, lens)):
        assert torch.equal(a, b) and bool(torch.isfinite(a.float()).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V", [(8, 5003), (5, 50257)])    # one workgroup per row, and several
def test_a_group_drawn_from_one_prompt(stage, dtype, n, V):
    g = torch.Generator(device=DEV).manual_seed(V)
    z = one_row(g, n, V, dtype=dtype)
    w = torch.randint(-2 ** 31, 2 ** 31, (n,), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    p = torch.full((n,), 0.9, device=DEV)
    got, want = stage.sample(z, w, top_p=p), stage.sample(z.contiguous(), w, top_p=p)
    for name in want:
        assert torch.equal(got[name], want[name]), name
    assert bool((got["ids"] >= 0).all()) and len(set(got["ids"].tolist())) > 1
