"""nat_embed and nat_embed_bwd against oracle/embedding.py."""
import numpy as np
import pytest
import torch

from nat_testlib import DEV
from oracle import embedding as oemb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def stage():
    from paper_2603_06619_amd.rollout import RolloutStage
    return RolloutStage(DEV)


def ids_of(seed, n, V, kind):
    rng = np.random.default_rng(seed)
    if kind == "text":                        # a few tokens make up much of it
        ids = np.minimum(np.exp(rng.uniform(0, np.log(V + 0.5), n)).astype(np.int64), V) - 1
        ids = rng.permutation(V)[ids]
    elif kind == "one":
        ids = np.full(n, V - 1)
    elif kind == "two":
        ids = np.where(np.arange(n) < n // 2, V - 1, 0)
    else:
        ids = rng.integers(0, V, n)
    if n > 10:
        ids[[3, n - 2]] = [-1, V]             # no tokens
        ids[n // 2] = -2 ** 31
    return ids.astype(np.int32)


def normal(seed, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V,H", [(1, 1, 8), (2, 5, 16), (7, 100, 24), (300, 777, 64), (65, 3001, 1032), (1000, 512, 4096), (3, 11, 5120)])
def test_forward(stage, dtype, n, V, H):
    ids, E = ids_of(n, n, V, "any"), normal(V, V, H, dtype=dtype)
    at = torch.from_numpy(ids).to(DEV)
    got = stage.embed(at, E)
    want = oemb.embed(ids, E.double().cpu().numpy())
    assert got.dtype == dtype and np.array_equal(got.double().cpu().numpy(), want)            # nothing is rounded at a scale of 1
    for scale in (H ** 0.5, -0.3):
        got = stage.embed(at, E, scale).double().cpu().numpy()
        ref = oemb.embed(ids, E.double().cpu().numpy(), float(np.float32(scale)))
        half = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8 + 2.0 ** -23               # bf16: after the product's rounding
        assert np.all(np.abs(got - ref) <= half * np.abs(ref))


def test_forward_strides_and_rows_left_alone(stage):
    import paper_2603_06619_amd as nat
    ids, E = ids_of(1, 50, 90, "any"), normal(2, 90, 40, dtype=torch.bfloat16)
    at = torch.from_numpy(ids).to(DEV)
    whole = torch.full((53, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    nat.nat_embed(at, E, 1.0, whole[:50, 8:48])
    assert torch.equal(whole[:50, 8:48], stage.embed(at, E))
    whole[:50, 8:48] = 7
    assert bool((whole == 7).all())
    assert stage.embed(at[:0], E).shape == (0, 40)


def test_forward_beyond_32_bit_offsets(stage):
    V, H = 700_000, 4096                                                                     # 5.7 GB
    E = torch.zeros((V, H), dtype=torch.bfloat16, device=DEV)
    for i in (0, 262143, 262144, 524288, V - 1):
        E[i] = normal(i + 1, H, dtype=torch.bfloat16)
    ids = torch.tensor([V - 1, 0, 524288, 262144, 262143], dtype=torch.int32, device=DEV)
    assert torch.equal(stage.embed(ids, E), E[ids.long()])


def check(stage, ids, dout, V, scale=1.0):
    at = torch.from_numpy(ids).to(DEV)
    got = stage.embed_backward(dout, at, V, scale)
    want, limit = oemb.embed_backward(dout.double().cpu().numpy(), ids, V, float(np.float32(scale)))
    assert got.shape == want.shape and got.dtype == torch.float32
    assert np.all(np.abs(got.double().cpu().numpy() - want) <= limit)
    return at, got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["text", "one", "two", "any"])
@pytest.mark.parametrize("n,V,H", [(1, 1, 8), (2, 3, 8), (9, 2, 16), (64, 1000, 24), (257, 63, 64), (1023, 64, 40), (3000, 32000, 64), (700, 300, 2056)])
def test_gradient(stage, dtype, kind, n, V, H):
    dout = normal(n + V, n, H, dtype=dtype)
    check(stage, ids_of(n, n, V, kind), dout, V)


@pytest.mark.parametrize("n", [8191, 8192, 8193, 12288, 40000, 270000])
@pytest.mark.parametrize("kind,V", [("text", 152064), ("any", 511), ("one", 512), ("two", 300000)])
def test_gradient_of_many_rows(stage, n, kind, V):
    """Across the sizes at which the sort takes one workgroup, several, and a scan of their counts."""
    dout = normal(n, n, 8, dtype=torch.bfloat16)
    check(stage, ids_of(n, n, V, kind), dout, V, 0.7)


def test_gradient_adds_and_repeats(stage):
    n, V, H = 5000, 400, 136
    ids, dout, old = ids_of(5, n, V, "text"), normal(6, n, H, dtype=torch.bfloat16), normal(7, V, H)
    at, got = check(stage, ids, dout, V, 2.0)
    total = stage.embed_backward(dout, at, V, 2.0, dE=old.clone(), accumulate=True)
    assert torch.equal(total, old + got)                      # one addition each
    unused = torch.ones(V, dtype=torch.bool)
    unused[ids[(ids >= 0) & (ids < V)]] = False
    assert torch.equal(total[unused.to(DEV)], old[unused.to(DEV)])
    for _ in range(3):
        assert torch.equal(stage.embed_backward(dout, at, V, 2.0), got)
    into = torch.full((V, H), float("nan"), device=DEV)       # what was there does not matter
    assert torch.equal(stage.embed_backward(dout, at, V, 2.0, dE=into), got)


def test_gradient_of_strided_shared_and_no_rows(stage):
    n, V, H = 600, 77, 48
    ids, dout = ids_of(8, n, V, "any"), normal(9, n, H, dtype=torch.bfloat16)
    at, got = check(stage, ids, dout, V)
    wide = torch.full((n, 64), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 8:56] = dout
    assert torch.equal(stage.embed_backward(wide[:, 8:56], at, V), got)
    one = dout[:1].expand(n, H)                               # the same gradient for all rows
    assert torch.equal(stage.embed_backward(one, at, V), stage.embed_backward(one.contiguous(), at, V))
    none = stage.embed_backward(dout[:0], at[:0], V)
    assert none.shape == (V, H) and bool((none == 0).all())
    kept = normal(10, V, H)
    assert torch.equal(stage.embed_backward(dout[:0], at[:0], V, dE=kept.clone(), accumulate=True), kept)
    outside = torch.full((n,), V, dtype=torch.int32, device=DEV)
    assert bool((stage.embed_backward(dout, outside, V) == 0).all())


def test_gradient_beyond_32_bit_offsets(stage):
    V, H, n = 600_000, 4096, 40                               # 9.8 GB
    ids = torch.tensor([V - 1, 0, 524288, 262144, 262143, 524288, V - 1, 131072] * 5, dtype=torch.int32, device=DEV)
    dout = normal(11, n, H, dtype=torch.bfloat16)
    got = stage.embed_backward(dout, ids, V)
    for i in ids.unique().tolist():
        rows = dout[ids == i].double()
        limit = rows.shape[0] * 2.0 ** -24 * rows.abs().sum(0)
        assert bool(((got[i].double() - rows.sum(0)).abs() <= limit).all())
        got[i] = 0
    assert int(torch.count_nonzero(got)) == 0


def test_gradient_against_differences(stage):
    """The loss is linear in E: a difference over a step of 1 is the gradient but for the roundings of two fp32 sums of 200 x 32 terms."""
    n, V, H = 200, 50, 32
    ids, dout, E, u = ids_of(12, n, V, "text"), normal(13, n, H), normal(14, V, H), normal(15, V, H)
    at = torch.from_numpy(ids).to(DEV)
    f = lambda x: float((stage.embed(at, x, 1.5).double() * dout.double()).sum())
    want = float((stage.embed_backward(dout, at, V, 1.5).double() * u.double()).sum())
    size = float((stage.embed(at, u.abs() + E.abs(), 1.5).double() * dout.double().abs()).sum())
    assert abs(f(E + u) - f(E) - want) <= 2.0 ** -20 * size


def test_other_streams_side_by_side(stage):
    n, V, H = 9000, 5000, 64
    cases = [(torch.from_numpy(ids_of(20 + i, n, V, "text")).to(DEV), normal(30 + i, n, H, dtype=torch.bfloat16)) for i in range(3)]
    want = [stage.embed_backward(d, i, V) for i, d in cases]
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in cases]
    got = [None] * 3
    for _ in range(4):
        for j, (i, d) in enumerate(cases):
            with torch.cuda.stream(sides[j]):
                got[j] = stage.embed_backward(d, i, V)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("n", [4097, 8192, 12289, 16384, 32767, 32768, 32769, 65536, 65537])
def test_gradient_where_the_sort_changes(stage, n):
    """Ids of a small vocabulary, equal ones in every tile; and a run that is longer than 64 pieces of 64 rows."""
    dout = normal(n, n, 16)
    check(stage, ids_of(n, n, 37, "any"), dout, 37)
    ids = ids_of(n, n, 5000, "text")
    ids[n // 7: n // 7 + min(n // 2, 20000)] = 4999
    check(stage, ids, dout, 5000, -1.5)


@pytest.mark.parametrize("V,H", [(70000, 1024), (60000, 1160), (30011, 2248), (66000, 1032)])
@pytest.mark.parametrize("kind", ["text", "one", "any"])
def test_gradient_of_a_large_vocabulary(stage, V, H, kind):
    """Above 256 MB: rows that begin and end inside the pieces in which zeros are written; every second id, runs longer than a wavefront."""
    n = 3000
    ids = ids_of(V, n, V, kind)
    ids[100:900:2] = np.arange(400) * 2 + V - 800            # (up to the last but one)
    ids[1200:1500] = V // 2
    at, dout = torch.from_numpy(ids).to(DEV), normal(V, n, H, dtype=torch.bfloat16)
    got = stage.embed_backward(dout, at, V, dE=torch.full((V, H), float("nan"), device=DEV))
    ok = (at >= 0) & (at < V)
    want = torch.zeros((V, H), dtype=torch.float64, device=DEV).index_add_(0, at[ok].long(), dout[ok].double())
    size = torch.zeros((V, H), dtype=torch.float64, device=DEV).index_add_(0, at[ok].long(), dout[ok].double().abs())
    count = torch.zeros(V, dtype=torch.float64, device=DEV).index_add_(0, at[ok].long(), torch.ones(int(ok.sum()), dtype=torch.float64, device=DEV))
    assert bool(((got.double() - want).abs() <= (count[:, None] + 1) * 2.0 ** -24 * size).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [255, 256, 1024, 1025])
def test_gradient_of_few_rows(stage, n, dtype):
    """Around the sizes at which there is no sort: runs over all 64s of the pairs, from the first pair and to the last; on top of what was there."""
    V, H = 999, 520
    ids = ids_of(n, n, V, "any")
    ids[::7] = 5
    ids[[0, n - 1]] = V - 1
    dout, old = normal(n, n, H, dtype=dtype), normal(n + 1, V, H)
    at, got = check(stage, ids, dout, V, -1.5)
    assert torch.equal(stage.embed_backward(dout, at, V, -1.5, dE=old.clone(), accumulate=True), old + got)
    check(stage, np.full(n, 7, np.int32), dout, 8)


@pytest.mark.parametrize("n,V,H", [(300, 30011, 2248), (300, 300000, 8), (1024, 30011, 2248), (300, 140001, 1032), (2500, 140001, 1032), (40000, 140001, 1032)])
def test_gradient_where_the_zeros_change(stage, n, V, H):
    """Zeros beside the sums, beside the sort, and in a launch of their own."""
    ids = ids_of(n, n, V, "any")
    ids[20:30] = V - 1
    ids[40:240:2] = np.arange(100) * 2 + V // 2
    at, dout = torch.from_numpy(ids).to(DEV), normal(V, n, H, dtype=torch.bfloat16)
    got = stage.embed_backward(dout, at, V, dE=torch.full((V, H), float("nan"), device=DEV))
    ok = (at >= 0) & (at < V)
    used, place = at[ok].unique(return_inverse=True)
    total = lambda x: torch.zeros((used.numel(), x.shape[1]), dtype=torch.float64, device=DEV).index_add_(0, place, x)
    rows = dout[ok].double()
    limit = (total(torch.ones_like(rows[:, :1])) + 1) * 2.0 ** -24 * total(rows.abs())
    assert bool(((got[used.long()].double() - total(rows)).abs() <= limit).all())
    got[used.long()] = 0
    assert bool((got == 0).all())
