"""Host-only: tensors whose rows are one and the same in memory (expanded along dimension 0).  The library reads a row stride of 0 as "rows back to back", so
the binding gives such inputs rows of their own and refuses such outputs before anything is called."""
import pytest
import torch

import paper_2603_06619_amd as nat
from paper_2603_06619_amd import binding, rollout


class OnDevice(torch.Tensor):
    """A host tensor that passes for one on a device: what is tested here never gets as far as the real library."""
    is_cuda = property(lambda self: True)


def device(*shape, dtype=torch.bfloat16, g=None):
    return (torch.randn(shape, generator=g).to(dtype) if g else torch.zeros(shape, dtype=dtype)).as_subclass(OnDevice)


@pytest.fixture
def calls(monkeypatch):
    """What the library would have been called with, by name.  Tensors live as long as the call, so their memory is read in it: `reads` maps a call's name to a
    function of its arguments."""
    class Library:
        made, reads = {}, {}

        def __getattr__(self, name):
            if name.startswith("nat_") and name.endswith("_bytes"):
                return lambda *a: 0

            def call(*a):
                self.made[name] = self.reads[name](*a) if name in self.reads else a
                return 0
            return call
    lib = Library()
    Library.made, Library.reads = {}, {}
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    monkeypatch.setattr(binding, "_stream", lambda: None)
    return lib


def memory(at, rows, stride, row):
    """`rows` rows of `row` two-byte elements, `stride` elements apart, as the library would read them."""
    import ctypes
    stride = stride or row
    raw = (ctypes.c_uint16 * (stride * (rows - 1) + row)).from_address(at)
    return torch.tensor(list(raw), dtype=torch.int32).as_strided((rows, row), (stride, 1)).clone()


def bits(t):
    return t.as_subclass(torch.Tensor).contiguous().flatten(1).view(torch.int16).to(torch.int32) & 0xffff


def test_row_strides():
    rows = binding._rows
    for t in (device(1, 4, 64).expand(5, 4, 64), device(5, 1, 64)[:1].expand(7, 1, 64), device(1, 1, 1).expand(5, 4, 64), device(1, 1, 64).expand(5, 4, 64)):
        assert rows(t, "x", is_input=True) == binding._SHARED
        with pytest.raises(ValueError):
            rows(t, "x")
    for kw in (dict(), dict(is_input=True)):
        with pytest.raises(ValueError):
            rows(device(9 * 64).as_strided((3, 2, 64), (64, 64, 1)), "x", **kw)
        for t, want in ((device(5, 4, 64), 0), (device(1, 4, 64), 0), (device(0, 4, 64), 0), (device(1, 4, 64).expand(1, 4, 64), 0), (device(5, 6, 64)[:, :4], 384),
                        (device(1, 6, 64)[:, :4], 0)):
            assert rows(t, "x", **kw) == want


def test_inputs_get_rows_of_their_own(calls):
    """Every input of every call in turn, expanded: the library reads the same rows n times, the other inputs where they are."""
    g = torch.Generator().manual_seed(1)
    n, D = 4, 64
    full = lambda h: device(n, h, D, g=g)
    wide = lambda h: device(1, h, D, g=g).expand(n, h, D)
    cu, lse, ws = device(2, dtype=torch.int32), device(8 * n, dtype=torch.float32), device(4096, dtype=torch.uint8)
    heads = lambda x: 2 if x in ("k", "v", "dk", "dv") else 8
    width = lambda x: heads(x) * D

    def attn(params, names, pointers):
        p = params._obj
        return {x: memory(at, n, getattr(p, x + "_stride"), width(x)) for x, at in zip(names, pointers) if x in ("q", "k", "v", "out", "dout")}
    calls.reads["nat_attn_fwd_split"] = lambda p, *a: attn(p, ("q", "k", "v"), a)
    calls.reads["nat_attn_bwd"] = lambda p, *a: attn(p, ("q", "k", "v", "out", "lse", "dout"), a)
    for name in ("q", "k", "v", "out", "dout"):
        t = {x: (wide if x == name else full)(heads(x)) for x in ("q", "k", "v", "out", "dout")}
        if name in ("q", "k", "v"):
            nat.nat_attn_fwd(t["q"], t["k"], t["v"], cu, cu, True, 0.125, full(8), lse, ws)
            for x, got in calls.made.pop("nat_attn_fwd_split").items():
                assert torch.equal(got, bits(t[x])), (name, x)
        nat.nat_attn_bwd(t["q"], t["k"], t["v"], t["out"], lse, t["dout"], cu, cu, True, 0.125, full(8), full(2), full(2), ws)
        made = calls.made.pop("nat_attn_bwd")
        assert set(made) == set(t)
        for x, got in made.items():
            assert torch.equal(got, bits(t[x])), (name, x)
    cache = nat.KvCache(device(3, 2, 16, D), device(3, 2, 16, D))
    calls.reads["nat_kv_write"] = lambda c, k, ks, v, vs, *a: (memory(k, n, ks, 2 * D), memory(v, n, vs, 2 * D))
    for k, v in ((wide(2), full(2)), (full(2), wide(2)), (wide(2), wide(2)), (device(n, 3, D, g=g)[:, 1:], full(2))):
        nat.nat_kv_write(cache, k, v, device(n, dtype=torch.int64))
        assert all(torch.equal(a, bits(b)) for a, b in zip(calls.made.pop("nat_kv_write"), (k, v)))
    calls.reads["nat_attn_decode"] = lambda c, q, qs, *a: memory(q, n, qs, 8 * D)
    q = wide(8)
    nat.nat_attn_decode(cache, q, device(n, 3, dtype=torch.int32), device(n, dtype=torch.int32), 0.125, full(8), lse, ws)
    assert torch.equal(calls.made.pop("nat_attn_decode"), bits(q))
    calls.reads["nat_sample"] = lambda z, row, rows, V, *a: memory(z, rows, row, V)
    word = device(n, dtype=torch.int32)
    for z in (device(1, 100, g=g).expand(n, 100), device(1, 1, g=g).expand(n, 1), device(n, 120, g=g)[:, 7:107], device(n, 100, g=g)):
        nat.nat_sample(z, word, None, None, None, None, word)
        assert torch.equal(calls.made.pop("nat_sample"), bits(z))


def test_outputs_and_overlapping_rows_are_refused(calls):
    n, D = 4, 64
    full, wide = (lambda h: device(n, h, D)), (lambda h: device(1, h, D).expand(n, h, D))
    cu, lse, ws = device(2, dtype=torch.int32), device(8 * n, dtype=torch.float32), device(4096, dtype=torch.uint8)
    q, k = full(8), full(2)
    cache = nat.KvCache(device(3, 2, 16, D), device(3, 2, 16, D))
    table, lens, word = device(n, 3, dtype=torch.int32), device(n, dtype=torch.int32), device(n, dtype=torch.int32)
    windows = device(20 * D).as_strided((n, 8, D), (D, D, 1))
    with pytest.raises(ValueError):
        nat.nat_attn_fwd(q, k, k, cu, cu, True, 0.125, wide(8), lse, ws)
    for outs in ((wide(8), full(2), full(2)), (full(8), wide(2), full(2)), (full(8), full(2), wide(2))):
        with pytest.raises(ValueError):
            nat.nat_attn_bwd(q, k, k, q, lse, q, cu, cu, True, 0.125, *outs, ws)
    for outs in ((wide(2), full(2)), (full(2), wide(2))):
        with pytest.raises(ValueError):
            nat.nat_kv_read(cache, table[:1], cu, *outs)
    with pytest.raises(ValueError):
        nat.nat_attn_decode(cache, q, table, lens, 0.125, wide(8), lse, ws)
    for call in (lambda: nat.nat_attn_fwd(windows, k, k, cu, cu, True, 0.125, q, lse, ws), lambda: nat.nat_attn_decode(cache, windows, table, lens, 0.125, q, lse, ws),
                 lambda: nat.nat_sample(device(400).as_strided((n, 100), (99, 1)), word, None, None, None, None, word)):
        with pytest.raises(ValueError):
            call()
    assert not calls.made


def test_stage_results_have_rows_of_their_own(monkeypatch):
    """What RolloutStage allocates for expanded inputs."""
    seen = {}
    for name in ("nat_attn_fwd", "nat_attn_bwd", "nat_attn_decode"):
        monkeypatch.setattr(binding, name, lambda *a, name=name: seen.__setitem__(name, a))
    monkeypatch.setattr(rollout.RolloutStage, "_buf", lambda self, key, nbytes: None)
    stage = rollout.RolloutStage("cpu")
    q, k, cu = torch.zeros(1, 8, 64).expand(4, 8, 64), torch.zeros(1, 2, 64).expand(4, 2, 64), torch.tensor([0, 4], dtype=torch.int32)
    out, lse = stage.attention(q, k, k, cu)
    grads = stage.attention_backward(out, q, k, k, out, lse, cu)
    cache = nat.KvCache(device(3, 2, 16, 64), device(3, 2, 16, 64))
    other, _ = stage.decode(q, cache, torch.zeros((4, 3), dtype=torch.int32), torch.ones(4, dtype=torch.int32))
    for x, like in ((out, q), (other, q), (grads[0], q), (grads[1], k), (grads[2], k)):
        assert x.shape == like.shape and x.is_contiguous()
    assert set(seen) == {"nat_attn_fwd", "nat_attn_bwd", "nat_attn_decode"}
