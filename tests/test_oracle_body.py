"""Pins of the oracle of norms and rotation, the embedding, page tables and the 4-bit format: autograd, differences, closed forms, counting."""
import numpy as np
import pytest
import torch

from oracle import embedding as oemb
from oracle import heads as ohead
from oracle import kv_cache as okv
from oracle import pages as opage


def _case(seed, n=5, heads=3, D=64, R=64):
    rng = np.random.default_rng(seed)
    return dict(x=rng.standard_normal((n, heads, D)) * 2, w=1 + 0.3 * rng.standard_normal(D), positions=rng.integers(0, 5000, n),
                inv_freq=1e4 ** (-2.0 * np.arange(R // 2) / R)), rng


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [64, 32, 16])
def test_norm_and_rotation_against_autograd(R, interleaved):
    c, rng = _case(1, R=R)
    dout = rng.standard_normal(c["x"].shape)
    x, w = (torch.from_numpy(c[n]).requires_grad_() for n in ("x", "w"))
    n = torch.nn.functional.rms_norm(x, (64,), w, 1e-6)
    angle = torch.from_numpy(c["positions"]).double()[:, None] * torch.from_numpy(c["inv_freq"])
    pairs = n[..., :R].unflatten(-1, (-1, 2)) if interleaved else n[..., :R].unflatten(-1, (2, -1)).transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(angle), angle)[:, None]
    pairs = torch.view_as_real(z)
    y = torch.cat(((pairs if interleaved else pairs.transpose(-1, -2)).flatten(-2), n[..., R:]), -1)
    got, _ = ohead.norm_rotate(**c, interleaved=interleaved)
    assert np.allclose(got, y.detach().numpy(), atol=1e-10)
    y.backward(torch.from_numpy(dout))
    back = ohead.norm_rotate_backward(dout, c["x"], c["w"], c["positions"], c["inv_freq"], interleaved=interleaved)
    assert np.allclose(back["dx"], x.grad.numpy(), atol=1e-10) and np.allclose(back["dw"], w.grad.numpy(), atol=1e-9)


def test_rotation_alone_and_norm_alone():
    c, rng = _case(2)
    y, _ = ohead.norm_rotate(c["x"], None, c["positions"], c["inv_freq"])
    assert np.allclose(np.square(y).sum(-1), np.square(c["x"]).sum(-1))                     # lengths stay
    # scores depend on the distance of positions alone
    dot = lambda p, q: (ohead.norm_rotate(c["x"][:1], None, [p], c["inv_freq"])[0] * ohead.norm_rotate(c["x"][1:2], None, [q], c["inv_freq"])[0]).sum(-1)
    assert np.allclose(dot(100, 40), dot(1060, 1000))
    n, _ = ohead.norm_rotate(c["x"], np.ones(64), eps=1e-30)
    assert np.allclose(np.square(n).mean(-1), 1.0)
    back = ohead.norm_rotate_backward(y, c["x"], None, c["positions"], c["inv_freq"])
    assert np.allclose(back["dx"], c["x"])                                                   # the rotation back


def test_gradients_of_norm_and_rotation_against_differences():
    c, rng = _case(3)
    dout = rng.standard_normal(c["x"].shape)
    back = ohead.norm_rotate_backward(dout, c["x"], c["w"], c["positions"], c["inv_freq"])
    f = lambda x, w: (ohead.norm_rotate(x, w, c["positions"], c["inv_freq"])[0] * dout).sum()
    for _ in range(4):
        u, v = rng.standard_normal(c["x"].shape), rng.standard_normal(64)
        assert abs((f(c["x"] + 1e-5 * u, c["w"]) - f(c["x"] - 1e-5 * u, c["w"])) / 2e-5 - (back["dx"] * u).sum()) < 1e-6
        assert abs((f(c["x"], c["w"] + 1e-5 * v) - f(c["x"], c["w"] - 1e-5 * v)) / 2e-5 - (back["dw"] * v).sum()) < 1e-6


def test_embedding_and_its_gradient():
    rng = np.random.default_rng(4)
    E, ids = rng.standard_normal((11, 8)), np.array([3, 3, 0, -1, 10, 3, 11, 7])
    ok = (ids >= 0) & (ids < 11)
    out = oemb.embed(ids, E, 2.0)
    onehot = np.where(ok[:, None], np.eye(11)[np.where(ok, ids, 0)], 0.0)
    assert np.allclose(out, 2.0 * onehot @ E)
    dout = rng.standard_normal((8, 8))
    assert np.allclose(oemb.embed_backward(dout, ids, 11, 2.0)[0], 2.0 * onehot.T @ dout)
    old = rng.standard_normal((11, 8))
    assert np.allclose(oemb.embed_backward(dout, ids, 11, 2.0, old)[0], old + 2.0 * onehot.T @ dout)


def test_pages_by_hand():
    table, free = [[5, -1], [7, 8], [-1, -1]], [1, 2, 3, 4, 0, 0, 0, 0, 0]
    r = opage.reserve(table, [16, 20, 0], [1, 2, 40], free, [4, 9], 16, 50)
    assert table == [[5, 4], [7, 8], [-1, -1]]                       # the third wants three places of a table of two
    assert r["counts"] == [3, 1] and r["seq_lens"] == [17, 22, 0] and r["start"] == [16, 20, -1] and r["cu_new"] == [0, 1, 3, 43]
    assert r["slots"][:4] == [4 * 16, 8 * 16 + 4, 8 * 16 + 5, -1] and r["position_ids"][:4] == [16, 20, 21, 0] and r["slots"][43:] == [-1] * 7
    lens, counts = opage.release(table, [17, 22, 0], [0, 16, 5], free, [3, 0], 16)
    assert lens == [0, 16, 0] and counts == [6, 0] and free[:6] == [1, 2, 3, 5, 4, 8]


def test_pages_are_given_once_and_come_back():
    rng = np.random.default_rng(5)
    n_pages, width, page, n = 40, 6, 16, 9
    free, table, lens, counts = list(rng.permutation(n_pages)), [[-1] * width for _ in range(n)], [0] * n, [n_pages, 0]
    for _ in range(60):
        new = [int(x) for x in rng.integers(0, 40, n)]
        r = opage.reserve(table, lens, new, free, counts, page, sum(new))
        lens, counts = r["seq_lens"], r["counts"]
        used = [table[i][p] for i in range(n) for p in range(opage.pages_of(lens[i], page))]
        assert len(set(used) | set(free[:counts[0]])) == n_pages == len(used) + counts[0]
        live = [s for s in r["slots"] if s >= 0]
        assert len(set(live)) == len(live)
        keep = [int(x) for x in rng.integers(0, 97, n)]
        lens, counts = opage.release(table, lens, keep, free, counts, page)
    lens, counts = opage.release(table, lens, [0] * n, free, counts, page)
    assert counts[0] == n_pages and sorted(free) == list(range(n_pages))


def test_4_bit_groups():
    x = np.zeros((1, 64))
    x[0, :16] = [0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -0.2, 5.01, 0.26, -6]        # halfway: the even code
    codes, e = okv.quantise_groups(x)
    v = okv.group_values(codes, e)
    assert list(e[0]) == [127, 2] and list(v[0, :16]) == [0, 0, 1, 1, 2, 2, 4, 4, 6, 0, -1, -1, 0, 6, 0.5, -6]
    assert np.signbit(v[0, [9, 12]]).all() and (codes[0, 16:] == 0).all()
    rng = np.random.default_rng(6)
    y = rng.standard_normal((200, 128)) * np.exp(5 * rng.standard_normal((200, 1)))
    codes, e = okv.quantise_groups(y)
    v = okv.group_values(codes, e).reshape(200, 4, 32)
    g, s = y.reshape(200, 4, 32), 2.0 ** (e.astype(float) - 127)
    top = np.abs(g).max(-1)
    assert np.all(top <= 6 * s) and np.all(top > 3 * s) and np.all(np.abs(v - g) <= np.maximum(np.abs(g) / 4, s[..., None] / 4) + 1e-300)
    again = okv.quantise_groups(v.reshape(200, 128))
    assert np.array_equal(okv.group_values(*again), v.reshape(200, 128))                      # values of the format stay
    for bad in (np.inf, -np.inf, np.nan):
        x[0, 3] = bad
        codes, e = okv.quantise_groups(x)
        assert list(e[0]) == [255, 2] and np.isnan(okv.group_values(codes, e)[0, :32]).all() and np.all(okv.group_values(codes, e)[0, 32:] == 0)
    big = np.full((1, 32), 3.3895313892515355e38)
    codes, e = okv.quantise_groups(big)
    assert e[0, 0] == 252 and np.all(okv.group_values(codes, e) == 6 * 2.0 ** 125)
