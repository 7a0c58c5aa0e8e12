"""More rows than one launch has room for (2^32 work-items are 2^23 rows of one workgroup each)."""
import pytest
import torch

from nat_testlib import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("filtered", [False, True])
def test_rows(filtered):
    from paper_2603_06619_amd.rollout import RolloutStage
    stage, n, V = RolloutStage(DEV), 2 ** 23 + 41, 8
    g = torch.Generator(device=DEV).manual_seed(1)
    z = torch.randn((n, V), generator=g, device=DEV)
    w = torch.randint(-2 ** 31, 2 ** 31, (n,), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    kw = dict(temperature=torch.rand(n, generator=g, device=DEV) + 0.5, top_k=torch.randint(1, 9, (n,), generator=g, device=DEV).to(torch.int32),
              top_p=torch.rand(n, generator=g, device=DEV), min_p=torch.rand(n, generator=g, device=DEV) / 2) if filtered else {}
    got = stage.sample(z, w, **kw)
    assert bool(((got["ids"] >= 0) & (got["ids"] < V)).all())
    for at in (slice(0, 50), slice(2 ** 22 - 20, 2 ** 22 + 20), slice(2 ** 23 - 40, n)):
        want = stage.sample(z[at], w[at], **{name: x[at] for name, x in kw.items()})
        for name in want:
            assert torch.equal(got[name][at], want[name]), (name, at)
    assert float((got["logp"] - z.log_softmax(1).gather(1, got["ids"].long()[:, None])[:, 0]).abs().max()) <= 1e-5
