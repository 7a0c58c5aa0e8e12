"""Pins of the oracle of attention, cache format and sampling: autograd, finite differences, closed forms, torch's own 8-bit type."""
import math

import numpy as np
import pytest
import torch

from oracle import attention as oattn
from oracle import kv_cache as okv
from oracle import sampling as osamp


def _case(seed, lens_q, lens_k, hq, hkv, D):
    rng = np.random.default_rng(seed)
    n_q, n_k = sum(lens_q), sum(lens_k)
    return dict(q=rng.standard_normal((n_q, hq, D)), k=rng.standard_normal((n_k, hkv, D)), v=rng.standard_normal((n_k, hkv, D)),
                dout=rng.standard_normal((n_q, hq, D)), cu_q=np.cumsum([0] + lens_q), cu_k=np.cumsum([0] + lens_k))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", [([5, 1, 7], [5, 1, 7]), ([3, 2], [9, 6]), ([6, 4], [3, 4]), ([2, 0, 3], [0, 4, 3])])
def test_attention_and_gradients_against_autograd(lens, causal):
    c = _case(1, *lens, 4, 2, 8)
    got = oattn.attention(c["q"], c["k"], c["v"], c["cu_q"], c["cu_k"], causal, dout=c["dout"])
    q, k, v = (torch.from_numpy(c[n]).requires_grad_() for n in ("q", "k", "v"))
    outs = []
    for b in range(len(c["cu_q"]) - 1):
        i, j = slice(c["cu_q"][b], c["cu_q"][b + 1]), slice(c["cu_k"][b], c["cu_k"][b + 1])
        n, m = i.stop - i.start, j.stop - j.start
        s = torch.einsum("ihd,jhd->hij", q[i], k[j].repeat_interleave(2, 1)) / math.sqrt(8)
        seen = torch.ones(n, m, dtype=torch.bool) if not causal else torch.arange(m) <= torch.arange(n)[:, None] + (m - n)
        s = s.masked_fill(~seen, -1e30)
        p = torch.softmax(s, -1) * seen if m else s
        outs.append(torch.einsum("hij,jhd->ihd", p, v[j].repeat_interleave(2, 1)))
    out = torch.cat(outs)
    (out * torch.from_numpy(c["dout"])).sum().backward()
    assert np.allclose(got["out"], out.detach().numpy(), atol=1e-12)
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        assert np.allclose(got[name], x.grad.numpy(), atol=1e-11), name


def test_gradients_against_differences():
    c = _case(2, [4, 3], [6, 3], 2, 1, 8)
    g = oattn.attention(c["q"], c["k"], c["v"], c["cu_q"], c["cu_k"], dout=c["dout"])
    f = lambda q, k, v: (oattn.attention(q, k, v, c["cu_q"], c["cu_k"])["out"] * c["dout"]).sum()
    rng = np.random.default_rng(3)
    for name in ("q", "k", "v"):
        for _ in range(4):
            u = rng.standard_normal(c[name].shape)
            at = lambda t: f(*[c[n] + (t * u if n == name else 0) for n in ("q", "k", "v")])
            assert abs((at(1e-5) - at(-1e-5)) / 2e-5 - (g["d" + name] * u).sum()) < 1e-7


def test_rows_without_keys_and_masked_infinities():
    c = _case(4, [5], [2], 2, 2, 8)
    g = oattn.attention(c["q"], c["k"], c["v"], c["cu_q"], c["cu_k"], dout=c["dout"])
    assert np.all(g["out"][:3] == 0) and np.all(np.isneginf(g["lse"][:, :3])) and np.all(g["dq"][:3] == 0)
    # the last key's value is seen by the last query alone
    c["v"][1, 0, 3] = np.inf
    bad = oattn.attention(c["q"], c["k"], c["v"], c["cu_q"], c["cu_k"])["out"]
    assert np.array_equal(bad[:4], g["out"][:4]) and np.isnan(bad[4, 0, 3])


def test_decode_is_attention_over_the_pages_tokens():
    rng = np.random.default_rng(5)
    k, v = rng.standard_normal((2, 7, 2, 16, 8))
    table = np.array([[4, 2, 0], [1, 5, -1], [3, 6, 6]])
    q = rng.standard_normal((3, 4, 8))
    got = oattn.decode(q, k, v, table, [37, 16, 0])
    rows = lambda c, b, n: np.concatenate([c[p].transpose(1, 0, 2) for p in table[b]])[:n]
    for b, n in ((0, 37), (1, 16)):
        ref = oattn.attention(q[b:b + 1], rows(k, b, n), rows(v, b, n), [0, 1], [0, n])
        assert np.allclose(got["out"][b], ref["out"][0]) and np.allclose(got["lse"][b], ref["lse"][:, 0])
    assert np.all(got["out"][2] == 0) and np.all(np.isneginf(got["lse"][2]))
    # a page that does not exist counts for nothing
    assert np.allclose(oattn.decode(q, k, v, table, [37, 48, 0])["out"][1], oattn.decode(q, k, v, table, [37, 32, 0])["out"][1])


def test_fp8_codes_against_torch():
    codes = np.arange(256).astype(np.uint8)
    ref = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    got = okv.decode_fp8(codes)
    assert np.array_equal(np.isnan(ref), np.isnan(got)) and np.array_equal(ref[~np.isnan(ref)], got[~np.isnan(got)])
    rng = np.random.default_rng(6)
    x = (rng.standard_normal((200, 64)) * np.exp(rng.standard_normal((200, 1)) * 8)).astype(np.float32)
    q, e = okv.quantise_rows(x)
    scale = 2.0 ** (e.astype(np.float64) - 127)
    y = torch.from_numpy(x.astype(np.float64) / scale[:, None]).float()
    assert np.array_equal(y.to(torch.float8_e4m3fn).view(torch.uint8).numpy(), q)
    top = np.abs(x).max(1)
    assert np.all(top <= 448 * scale) and np.all(top > 224 * scale)
    assert np.all(np.abs(okv.row_values(q, e) - x) <= np.maximum(np.abs(x) * 2.0 ** -4, scale[:, None] * 2.0 ** -10))


def test_fp8_rows_of_zeros_and_not_finite():
    x = np.array([[0.0, -0.0, 0.0], [np.inf, 1.0, -3.0], [np.nan, -np.inf, 0.0], [448.0, 1.0, 2.0], [450.0, 0.0, 0.0]])
    q, e = okv.quantise_rows(x)
    assert list(e) == [1, 127 - 7, 1, 127, 128]
    assert list(q[0]) == [0, 128, 0] and q[1][0] == 127 and q[2][0] == 127 and q[2][1] == 255
    assert okv.row_values(q, e)[1][2] == -3.0 and okv.row_values(q, e)[3][0] == 448.0


def test_draws_cover_the_distribution():
    """Words spread evenly over their range draw every token as often as its probability says, to one draw."""
    z = np.array([0.3, -1.0, 2.0, 2.0, -np.inf, 1.1], np.float32)
    n = 4096
    for kw, p in ((dict(), np.exp(z.astype(np.float64))), (dict(temperature=0.5), np.exp(2 * z.astype(np.float64))),
                  (dict(top_k=3), np.exp(z.astype(np.float64)) * [0, 0, 1, 1, 0, 1]), (dict(top_k=1), np.array([0, 0, 1.0, 0, 0, 0])),
                  (dict(top_p=0.3), np.array([0, 0, 1.0, 0, 0, 0])), (dict(min_p=0.2), np.exp(z.astype(np.float64)) * [0, 0, 1, 1, 0, 1])):
        p = p / p.sum()
        got = [osamp.sample(z, i << 20, **kw) for i in range(n)]
        counts = np.bincount([g[0] for g in got], minlength=6)
        assert np.all(np.abs(counts - n * p) <= 1.0 + 1e-6), (kw, counts, n * p)
        for tok, logp, logq in got[::97]:
            assert abs(logq - math.log(p[tok])) < 1e-6
            assert abs(logp - (z[tok] - np.log(np.exp(z.astype(np.float64)).sum()))) < 1e-12


def test_nucleus_is_the_smallest_prefix():
    rng = np.random.default_rng(8)
    z = rng.standard_normal(50).astype(np.float32)
    a, _ = osamp.weights(z, 1.0)
    order = np.argsort(-z, kind="stable")
    for p in (1e-9, 0.1, 0.5, 0.9, 0.999, 1.0 - 2 ** -24):
        kept, _ = osamp.filtered(z, top_p=p)
        n = sum(w > 0 for w in kept)
        run = np.cumsum([a[i] for i in order])
        assert set(np.nonzero(kept)[0]) == set(order[:n])
        assert run[n - 1] / run[-1] >= np.float32(p) - 1e-9 and (n == 1 or run[n - 2] / run[-1] < p)


def test_rows_without_logits_and_greedy():
    inf = np.inf
    assert osamp.sample(np.array([-inf, np.nan, -inf], np.float32), 5)[0] == -1
    assert osamp.sample(np.array([1.0, 3.0, 3.0, np.nan], np.float32), 2 ** 32 - 1, temperature=0.0)[0] == 1
    assert osamp.sample(np.array([1.0, inf, 3.0, inf], np.float32), 2 ** 32 - 1) == (3, -math.log(2), -math.log(2))
    assert osamp.sample(np.array([-0.0, 0.0], np.float32), 0, top_k=1)[0] == 0
