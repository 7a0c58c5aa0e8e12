"""The embedding's gradient where its zeros are more than 512 MB and its pairs are sorted in tiles: zeros behind the workgroups that rank them."""
import numpy as np
import pytest
import torch

from nat_testlib import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n", [1025, 8192, 8193, 12289, 20483, 32767, 32768, 32769])
def test_large_gradients(n, accumulate, dtype):
    """Sums of a row's k pairs in fp32: k + 1 roundings of the magnitudes, one more with what was there before."""
    from paper_2603_06619_amd.rollout import RolloutStage
    V, H = 131101, 1032
    assert V * H * 4 > 512 << 20
    g = torch.Generator(device=DEV).manual_seed(n)
    rng = np.random.default_rng(n)
    ids = rng.integers(0, V, n)
    ids[::5], ids[1::7], ids[[0, n // 2, n - 1]] = V // 3, rng.integers(0, 40, len(ids[1::7])), V - 1       # a fifth in one row, others often, the last one
    ids[[2, n - 2]], ids[n // 3] = (-1, V), -2 ** 31                                                    # padding
    at = torch.from_numpy(ids.astype(np.int32)).to(DEV)
    dout = torch.randn((n, H), generator=g, device=DEV).to(dtype)
    into = torch.full((V, H), 0.25 if accumulate else float("nan"), device=DEV)
    got = RolloutStage(DEV).embed_backward(dout, at, V, dE=into, accumulate=accumulate)
    ok = (at >= 0) & (at < V)
    used, place = at[ok].unique(return_inverse=True)
    total = lambda x: torch.zeros((used.numel(), x.shape[1]), dtype=torch.float64, device=DEV).index_add_(0, place, x)
    rows, old = dout[ok].double(), 0.25 if accumulate else 0.0
    limit = (total(torch.ones_like(rows[:, :1])) + 2) * 2.0 ** -24 * (total(rows.abs()) + old)
    assert bool(((got[used.long()].double() - total(rows) - old).abs() <= limit).all())
    got[used.long()] = old
    assert bool((got == old).all())
