"""Infinities and NaN that rows do see: results are what the formulas give, at the mask's edge (where masked ones are taken out by hand) as in whole tiles, and everything
that they do not enter keeps its bits.  Places `at`: the first tile of keys, its last row, later tiles' edges and insides."""
import numpy as np
import pytest
import torch

from nat_testlib import DEV
from oracle import attention as oattn
from test_gpu_attention import host, make, run, stage  # noqa: F401 (stage is a fixture)

pytestmark = pytest.mark.gpu
AT = [1, 63, 70, 128, 150, 199]


def clone(c):
    return {n: x.clone() for n, x in c.items()}


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", AT)
def test_a_key_of_minus_infinity(stage, D, at):  # noqa: F811
    """All its scores are -inf, so its probabilities and dS are 0: as with a very low finite element, but that dq's own element is 0 times infinity."""
    n = 200
    c = make(21, [n, 30], [n, 30], 4, 2, D)
    c["q"][:, :, 1] = c["q"][:, :, 1].abs() + 0.1
    low, bad = clone(c), clone(c)
    low["k"][at, :, 1], bad["k"][at, :, 1] = -1e30, -float("inf")
    want, got = run(stage, low), run(stage, bad)
    ref = oattn.attention(host(low["q"]), host(low["k"]), host(low["v"]), host(c["cu_q"]), host(c["cu_k"]), dout=host(c["dout"]))
    for name in ("out", "dq", "dk", "dv"):                         # rows of few keys among them: the limit of test_gpu_attention's long rows
        assert np.linalg.norm(host(want[name]) - ref[name]) <= 1.5e-2 * np.linalg.norm(ref[name]), name
    for name in ("out", "lse", "dk", "dv"):
        assert torch.equal(got[name], want[name]), name
    assert bool(got["dq"][at:n, :, 1].isnan().all())
    got["dq"][at:n, :, 1] = want["dq"][at:n, :, 1]
    assert torch.equal(got["dq"], want["dq"])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", AT)
def test_a_query_that_is_not_a_number(stage, D, at):  # noqa: F811
    """Its probabilities are NaN: its own row, and the gradients of all keys that it sees, whole; nothing else."""
    n = 200
    c = make(22, [n, 30], [n, 30], 4, 2, D)
    want = run(stage, c)
    c["q"][at, :, 3] = float("nan")
    got = run(stage, c)
    for name, seen in (("out", slice(at, at + 1)), ("dq", slice(at, at + 1)), ("dk", slice(0, at + 1)), ("dv", slice(0, at + 1))):
        assert bool(got[name][seen].isnan().all()), name
        got[name][seen] = want[name][seen]
        assert torch.equal(got[name], want[name]), name


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", AT)
def test_an_infinite_gradient(stage, D, at):  # noqa: F811
    """dv of the keys that its row sees has its sign, dS of them is not finite; nothing else changes."""
    n = 200
    for value in (float("inf"), -float("inf")):
        c = make(23, [n, 30], [n, 30], 4, 2, D)
        want = run(stage, c)
        c["dout"][at, :, 5] = value
        got = run(stage, c)
        assert bool((got["dv"][:at + 1, :, 5] == value).all())
        assert not bool(torch.isfinite(got["dq"][at]).any()) and not bool(torch.isfinite(got["dk"][:at + 1]).any())
        got["dv"][:at + 1, :, 5] = want["dv"][:at + 1, :, 5]
        got["dq"][at], got["dk"][:at + 1] = want["dq"][at], want["dk"][:at + 1]
        for name in want:
            assert torch.equal(got[name], want[name]), name


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", [0] + AT)
def test_an_infinite_value(stage, D, at):  # noqa: F811
    """Every row that sees it has its sign in that element; nothing else changes."""
    n = 200
    for value in (float("inf"), -float("inf")):
        c = make(24, [n, 30], [n, 30], 4, 2, D)
        want = run(stage, c, backward=False)
        c["v"][at, :, 9] = value
        got = run(stage, c, backward=False)
        assert bool((got["out"][at:n, :, 9] == value).all())
        got["out"][at:n, :, 9] = want["out"][at:n, :, 9]
        assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])


@pytest.mark.parametrize("D", [64, 128])
def test_an_infinite_value_among_shared_keys(stage, D):  # noqa: F811
    """Rows whose keys several workgroups share: seen by all rows, by some, in a part of its own."""
    for at in (0, 1400, 2985, 2999):
        c = make(25, [20], [3000], 4, 2, D)
        want = run(stage, c, backward=False)
        c["v"][at, :, 9] = float("inf")
        got = run(stage, c, backward=False)
        first = max(at - 2980, 0)
        assert bool((got["out"][first:, :, 9] == float("inf")).all())
        got["out"][first:, :, 9] = want["out"][first:, :, 9]
        assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
