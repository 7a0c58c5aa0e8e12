"""Norms of heads whose squares leave fp32's range, up to the largest finite elements, and with an eps at either end of its range."""
import numpy as np
import pytest
import torch

from nat_testlib import DEV
from oracle import heads as ohead

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def stage():
    from paper_2603_06619_amd.rollout import RolloutStage
    return RolloutStage(DEV)


def host(t):
    return None if t is None else t.double().cpu().numpy()


def close(got, want, limit):
    got = host(got)
    assert np.isfinite(got).all() and np.all(np.abs(got - want) <= limit), float((np.abs(got - want) / np.maximum(limit, 1e-300)).max())


def rotation(n, R):
    return dict(position_ids=torch.arange(n, dtype=torch.int32, device=DEV) * 37, inv_freq=1e4 ** (-2.0 * torch.arange(R // 2, dtype=torch.float64, device=DEV) / R))


def check(stage, c, grads, eps):
    """Each element within the oracle's limits, which are relative to the numbers that it is made of.  Results and what is held on the way are in fp32's normal range, but for r = 1 / sqrt(mean x^2),
    which of elements near 2^128 is 2^-128 with a step of 2^-149: 4 F of the 72 F, of which the formulas take 65."""
    dtype, angle = c["q"].dtype, (host(c["position_ids"]), host(c["inv_freq"]))
    got, back = stage.norm_rotate(**c, eps=eps), stage.norm_rotate_backward(*grads, **c, eps=eps)
    for i, name in enumerate("qk"):
        x, w = host(c[name]), host(c[name + "_weight"])
        close(got[i], *ohead.norm_rotate(x, w, *angle, eps=eps, half=HALF[dtype]))
        ref = ohead.norm_rotate_backward(host(grads[i]), x, w, *angle, eps=eps, half=HALF[dtype], chain=64)
        close(back[i], ref["dx"], ref["e_dx"])
        close(back[2 + i], ref["dw"], ref["e_dw"])


def case(seed, rows, n, D, dtype, grad=1e20):
    """rows(random numbers in [1/2, 1), their signs) of 3 query heads and 2 key heads; gradients whose quotients by the largest elements are normal numbers."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    new = lambda h: rows(0.5 + 0.5 * torch.rand((n, h, D), generator=g, device=DEV), torch.randint(2, (n, h, D), generator=g, device=DEV) * 2 - 1).to(dtype)
    weight = lambda: (1 + 0.3 * torch.rand(D, generator=g, device=DEV)).to(dtype)
    c = dict(q=new(3), k=new(2), q_weight=weight(), k_weight=weight(), **rotation(n, D))
    return c, [(grad * torch.randn(x.shape, generator=g, device=DEV)).to(dtype) for x in (c["q"], c["k"])]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size", [1.7e18, 2.4e18, 1e30, 1e37, 3.1e37, 4.4e37, 1e38, 3e38])
def test_equal_sizes(stage, size, D, dtype):
    c, grads = case(1, lambda x, sign: size * sign, 5, D, dtype)
    check(stage, c, grads, 1e-6)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_large_elements_among_small_ones(stage, D, dtype):
    """One to all elements of a head near the largest number, the others far below it."""
    def rows(x, sign):
        many = torch.tensor([1, 2, D // 2, D - 1, D], device=DEV)
        large = (torch.arange(D, device=DEV) * 29 + 3) % D < many[:, None, None]
        return x * sign * torch.where(large, 3.3e38, 1e8)
    c, grads = case(2, rows, 5, D, dtype)
    check(stage, c, grads, 1e-6)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_other_heads_do_not_see_it(stage, dtype):
    c, grads = case(3, lambda x, sign: x * sign, 4, 64, dtype, grad=1.0)
    want, back = stage.norm_rotate(**c), stage.norm_rotate_backward(*grads, **c)
    c["q"][1, 0], c["k"][2, 1], grads[0][1, 0], grads[1][2, 1] = 3e38, -3e38, 0, 0
    got, mine = stage.norm_rotate(**c), stage.norm_rotate_backward(*grads, **c)
    for i, at in ((0, (1, 0)), (1, (2, 1))):
        keep = torch.ones(c["qk"[i]].shape[:2], dtype=torch.bool, device=DEV)
        keep[at] = False
        assert torch.equal(got[i][keep], want[i][keep]) and torch.equal(mine[i][keep], back[i][keep])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("eps", [1e30, 1.5e38])
def test_large_eps(stage, D, eps):
    """As large as the mean square, which passes the range as a sum."""
    c, grads = case(4, lambda x, sign: 2.4e18 * x.add(0.5) * sign, 5, D, torch.float32)
    assert bool(torch.isinf(c["q"].square().sum(-1)).any())
    check(stage, c, grads, eps)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size", [1e15, 1e17, 1e18, 1e30])
def test_largest_eps(stage, D, size):
    """A sum with the mean square, of which neither passes the range alone."""
    c, grads = case(6, lambda x, sign: size * x * sign, 5, D, torch.float32)
    check(stage, c, grads, float(np.finfo(np.float32).max))


@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1.2e-38])
def test_small_eps(stage, eps):
    """Beside it the squares are everything; a row of zeros stays zeros."""
    eps = float(np.float32(eps))
    c, grads = case(5, lambda x, sign: 1e-3 * x * sign, 5, 64, torch.float32, grad=1.0)
    check(stage, c, grads, eps)
    c["q"][3], c["k"][1] = 0, 0
    q, k = stage.norm_rotate(**c, eps=eps)
    assert bool((q[3] == 0).all()) and bool((k[1] == 0).all()) and bool(q.isfinite().all()) and bool(k.isfinite().all())
