"""More (row, head) pairs than one launch has room for: 2^32 work-items are 2^28 of them at 16 lanes each."""
import pytest
import torch

from nat_testlib import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rows():
    """65552 rows of 4096 heads of 128 elements, 64 GiB, of which the first and last 16 have values and a place in a cache of one page."""
    n, heads, D = 65552, 4096, 128
    x = torch.empty((n, heads, D), dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    for part in (x[:16], x[-16:]):
        part.copy_(torch.randn(part.shape, generator=g, device=DEV))
    yield x
    del x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("fp8", [False, True])
def test_write(rows, fp8):
    from paper_2603_06619_amd.rollout import PagedCache, RolloutStage
    stage = RolloutStage(DEV)
    n, heads, D = rows.shape
    slots = torch.full((n,), -1, dtype=torch.int64, device=DEV)
    slots[:8], slots[-8:] = torch.arange(8, device=DEV), torch.arange(8, 16, device=DEV)
    new = lambda: PagedCache.empty(1, heads, 16, D, fp8, DEV)
    cache, small = new(), new()
    for c in (cache, small):
        for t in (c.k, c.v, c.k_exp, c.v_exp):
            if t is not None:
                t.view(torch.uint8).zero_()
    stage.write_cache(cache, rows, rows, slots)
    both = torch.cat((rows[:8], rows[-8:]))
    stage.write_cache(small, both, both, torch.arange(16, device=DEV))
    for name in ("k", "v", "k_exp", "v_exp") if fp8 else ("k", "v"):
        assert torch.equal(getattr(cache, name).view(torch.uint8), getattr(small, name).view(torch.uint8)), name


@pytest.mark.parametrize("fp8", [False, True])
def test_read(rows, fp8):
    """A sequence of the last 16 rows; those before it belong to none."""
    import paper_2603_06619_amd as nat
    from paper_2603_06619_amd.rollout import PagedCache, RolloutStage
    n, heads, D = rows.shape
    cache = PagedCache.empty(1, heads, 16, D, fp8, DEV)
    RolloutStage(DEV).write_cache(cache, rows[-16:], rows[-16:], torch.arange(16, device=DEV))
    cu = torch.tensor([0, 16], dtype=torch.int32, device=DEV)
    want, _ = RolloutStage(DEV).read_cache(cache, torch.zeros((1, 1), dtype=torch.int32, device=DEV), cu, 16)
    k = torch.empty_like(rows)
    k[-40:] = 7.0
    nat.nat_kv_read(cache, torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.tensor([n - 16, n], dtype=torch.int32, device=DEV), k, k)
    assert torch.equal(k[-16:], want) and bool((k[-40:-16] == 7.0).all())
