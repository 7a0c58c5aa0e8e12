"""nat_sample: tokens bit for bit as the oracle draws them, log-probabilities to 2e-6 (1 + |log p|): a soft-max sum of fp32
exponentials (relative error below 1e-6) and one rounding."""
import math

import numpy as np
import pytest
import torch

from nat_testlib import DEV
from oracle import sampling as osamp

pytestmark = pytest.mark.gpu

T, K, P, M = [0.0, 0.3, 0.7, 1.0, 1.0, 1.5, 30.0], [0, 0, 1, 2, 7, 50, 100000], [0.0, 0.05, 0.5, 0.9, 0.999, 1.0, 1.0], [0.0, 0.0, 0.01, 0.3, 1.0]


@pytest.fixture(scope="module")
def stage():
    from paper_2603_06619_amd.rollout import RolloutStage
    return RolloutStage(DEV)


def draw(stage, z, words, temperature=None, top_k=None, top_p=None, min_p=None):
    dev = lambda x, dt: None if x is None else torch.as_tensor(np.asarray(x, dt)).to(DEV)
    w = torch.from_numpy(np.asarray(words, np.uint32).view(np.int32).copy()).to(DEV)
    r = stage.sample(z, w, dev(temperature, np.float32), dev(top_k, np.int32), dev(top_p, np.float32), dev(min_p, np.float32))
    torch.cuda.synchronize()
    return {n: x.cpu().numpy() for n, x in r.items()}


def check(z, words, r, temperature=None, top_k=None, top_p=None, min_p=None):
    host = z.float().cpu().numpy()
    for i in range(len(words)):
        at = lambda x, off: off if x is None else np.asarray(x)[i].item()
        ids, logp, logq = osamp.sample(host[i], int(words[i]), at(None if temperature is None else np.float32(temperature), 1.0), at(top_k, 0),
                                       at(None if top_p is None else np.float32(top_p), 1.0), at(None if min_p is None else np.float32(min_p), 0.0))
        assert r["ids"][i] == ids, (i, r["ids"][i], ids)
        for got, want in ((r["logp"][i], logp), (r["logq"][i], logq)):
            assert (math.isnan(got) and math.isnan(want)) or abs(got - want) <= 2e-6 * (1 + abs(want)), (i, got, want)


def words_of(rng, n):
    w = rng.integers(0, 2 ** 32, n, dtype=np.uint64).astype(np.uint32)
    w[:2] = [0, 2 ** 32 - 1][:min(2, n)]
    return w


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,sigma", [(1, 1.0), (2, 1.0), (7, 3.0), (63, 1.0), (1000, 2.0), (4097, 0.5), (8191, 6.0), (20011, 2.0), (33001, 2.0)])
def test_draws(stage, dtype, V, sigma):
    rng = np.random.default_rng(V)
    n = 40 if V < 10000 else 12
    z = torch.from_numpy((rng.standard_normal((n, V)) * sigma).astype(np.float32)).to(dtype).to(DEV)
    w = words_of(rng, n)
    check(z, w, draw(stage, z, w))
    pick = lambda x: rng.choice(x, n)
    for kw in (dict(temperature=pick(T)), dict(top_k=pick(K)), dict(top_p=pick(P)), dict(min_p=pick(M)), dict(top_k=pick(K), top_p=pick(P)),
               dict(temperature=pick(T), top_k=pick(K), top_p=pick(P), min_p=pick(M))):
        check(z, w, draw(stage, z, w, **kw), **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_equal_logits_masks_and_not_finite(stage, dtype):
    inf, nan, V = math.inf, math.nan, 9000
    rng = np.random.default_rng(1)
    n = 48
    z = rng.integers(-3, 3, (n, V)).astype(np.float32)            # a handful of values: ties at every cut
    z[0] = 0.0
    z[1] = -inf
    z[2] = nan
    z[3, : V - 1] = -inf
    z[4, 5] = nan
    z[5, 77] = z[5, 8000] = inf
    z[6] = np.where(rng.random(V) < 0.5, -0.0, 0.0)
    z[7] = np.finfo(np.float32).min                               # a mask by the type's lowest value
    z[7, 4000:4100] = 1.0
    z[8] = np.finfo(np.float32).min
    z[9, :] = -inf
    z[9, 123] = -1e30
    z = torch.from_numpy(z).to(dtype).to(DEV)
    w = words_of(rng, n)
    pick = lambda x: rng.choice(x, n)
    for kw in (dict(), dict(top_k=pick([1, 2, 777, 4500, 8999])), dict(top_p=pick([0.0, 0.2, 0.77, 0.99])),
               dict(top_k=pick([3, 3000]), top_p=pick([0.3, 0.9]), min_p=pick([0.0, 0.2])), dict(temperature=pick(T), top_k=pick(K), top_p=pick(P))):
        check(z, w, draw(stage, z, w, **kw), **kw)


def test_settings_out_of_range(stage):
    rng = np.random.default_rng(2)
    n, V = 8, 500
    z = torch.from_numpy(rng.standard_normal((n, V)).astype(np.float32)).to(DEV)
    w = words_of(rng, n)
    plain = draw(stage, z, w)
    off = draw(stage, z, w, [1.0] * n, [0, -1, V, V + 1, 2 ** 31 - 1, 0, 0, 0], [1.0, 2.0, math.inf, math.nan, 1.0, 1.0, 1.0, 1.0],
               [0.0, -1.0, math.nan, -math.inf, 0.0, 0.0, 0.0, 0.0])
    greedy = draw(stage, z, w, [0.0, -1.0, math.nan, -math.inf, 0.0, 0.0, 0.0, 0.0])
    first = draw(stage, z, w, None, None, [-1.0, 0.0, -math.inf] + [0.0] * 5)
    one = draw(stage, z, w, None, None, None, [5.0, 1.0, math.inf] + [1.0] * 5)
    for name in plain:
        assert np.array_equal(plain[name], off[name])
    top = z.cpu().numpy().argmax(1)
    for r in (greedy, first, one):
        assert np.array_equal(r["ids"], top) and np.all(r["logq"] == 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_at_any_alignment_and_stride(stage, dtype):
    rng = np.random.default_rng(3)
    V = 5003
    z = torch.from_numpy(rng.standard_normal((9, V)).astype(np.float32)).to(dtype).to(DEV)
    w = words_of(rng, 9)
    kw = dict(top_k=[0, 40] * 4 + [9], top_p=[0.9] * 9)
    ref = draw(stage, z, w, **kw)
    for pad, lead in ((1, 0), (5, 3), (8, 1), (13, 7)):
        whole = torch.full((9, V + pad + lead), 1000.0, dtype=dtype, device=DEV)
        part = whole[:, lead:lead + V]
        part.copy_(z)
        r = draw(stage, part, w, **kw)
        for name in ref:
            assert np.array_equal(ref[name], r[name]), (pad, lead, name)


def test_real_vocabularies_in_places(stage):
    """Rows of 151936 and 152064 logits."""
    for V, dtype in ((151936, torch.bfloat16), (152064, torch.float32)):
        g = torch.Generator(device=DEV).manual_seed(V)
        z = 2 * torch.randn((6, V), generator=g, device=DEV)
        z[:, ::5000] += 9
        z[1, 1000:] = -math.inf
        z = z.to(dtype)
        w = words_of(np.random.default_rng(V), 6)
        for kw in (dict(), dict(temperature=[1.0, 0.7, 1.0, 0.0, 1.2, 0.9], top_k=[0, 50, 1000, 5, 1, 0], top_p=[0.95, 1.0, 0.5, 0.9, 0.9, 0.3],
                                min_p=[0.0, 0.05, 0.0, 0.0, 0.0, 0.01])):
            check(z, w, draw(stage, z, w, **kw), **kw)


def test_the_largest_vocabulary_and_rows_beyond_32_bit_offsets(stage):
    V, stride = 1 << 20, (1 << 31) + 3
    base = torch.full((stride + V,), -1.0, dtype=torch.bfloat16, device=DEV)
    z = base.as_strided((2, V), (stride, 1))
    z[1, 777777] = 3.0
    w = np.array([2 ** 32 - 1, 2 ** 31], np.uint32)
    r = draw(stage, z, w, None, [0, 2], None, None)
    assert r["ids"][0] == V - 1 and r["ids"][1] == 777777
    assert abs(r["logp"][0] + math.log(V)) < 1e-4


def test_behaviour_log_probs_are_what_the_loss_stage_takes(stage):
    """logp of a drawn token = nat_logp_fwd of that token from the same hidden rows (1e-4: the logits are held in fp32 here)."""
    from paper_2603_06619_amd.stage import LossStage
    g = torch.Generator(device=DEV).manual_seed(9)
    n, H, V = 50, 128, 4099
    hidden = torch.randn((n, H), generator=g, device=DEV, dtype=torch.bfloat16)
    W = (torch.randn((V, H), generator=g, device=DEV) * 0.2).bfloat16()
    z = hidden.float() @ W.float().t()
    w = torch.randint(-2 ** 31, 2 ** 31, (n,), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    r = stage.sample(z, w)
    lp = LossStage(DEV).logp(hidden, W, r["ids"], n)["logp"][:n]
    assert float((lp - r["logp"]).abs().max()) <= 1e-4
    assert torch.equal(r["logp"].isnan(), r["logq"].isnan()) and float((r["logp"] - r["logq"]).abs().max()) <= 1e-5


def test_another_stream_and_runs(stage):
    g = torch.Generator(device=DEV).manual_seed(10)
    z = torch.randn((64, 30011), generator=g, device=DEV)
    w = torch.randint(-2 ** 31, 2 ** 31, (64,), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    p = torch.full((64,), 0.9, device=DEV)
    a = stage.sample(z, w, top_p=p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = stage.sample(z, w, top_p=p)
    side.synchronize()
    for n in a:
        assert torch.equal(a[n], b[n])
