"""Host-only: the argument checks of the operators beside the loss stage, through the C ABI.  Every call fails, or has nothing to do,
before anything is launched; pointers named `fake` are never dereferenced."""
import ctypes
import os

import pytest

OK, INVALID, SHAPE, WORKSPACE, DTYPE = 0, 1, 2, 3, 4
fake = 4096


@pytest.fixture(scope="module")
def nat():
    import paper_2603_06619_amd as nat
    if not os.path.exists(nat.library_path()):
        from paper_2603_06619_amd import build
        build.build()
    return nat


def attn(nat, entry="nat_attn_fwd", ptr=None, ws=(fake, 1 << 40), **kw):
    from paper_2603_06619_amd import binding
    p = dict(n_seqs=3, n_q_heads=8, n_kv_heads=2, head_dim=64, dtype=nat.DTYPE_BF16, causal=1, scale=0.125, n_q=100, n_k=120)
    p.update(kw)
    c = binding._CAttnParams()
    for name, value in p.items():
        setattr(c, name, value)
    at = dict(q=fake, k=fake, v=fake, out=fake, lse=fake, dout=fake, cu_q=fake, cu_k=fake, dq=fake, dk=fake, dv=fake)
    at.update(ptr or {})
    lib = nat.load_library()
    if entry == "nat_attn_fwd":
        return lib.nat_attn_fwd(ctypes.byref(c), at["q"], at["k"], at["v"], at["cu_q"], at["cu_k"], at["out"], at["lse"], None)
    return lib.nat_attn_bwd(ctypes.byref(c), at["q"], at["k"], at["v"], at["out"], at["lse"], at["dout"], at["cu_q"], at["cu_k"], at["dq"], at["dk"],
                            at["dv"], ws[0], ws[1], None)


@pytest.mark.parametrize("entry", ["nat_attn_fwd", "nat_attn_bwd"])
def test_attention_refusals(nat, entry):
    call = lambda **kw: attn(nat, entry, **kw)
    assert nat.load_library().nat_attn_fwd(None, fake, fake, fake, fake, fake, fake, fake, None) == INVALID
    assert call(dtype=nat.DTYPE_F32) == DTYPE and call(dtype=7) == DTYPE
    for kw in (dict(n_seqs=-1), dict(n_q=-1), dict(n_k=-1), dict(n_q=1 << 31), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(causal=2), dict(causal=-1)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(head_dim=96), dict(head_dim=0), dict(head_dim=256), dict(n_kv_heads=3), dict(n_kv_heads=0), dict(n_q_heads=0), dict(n_q_heads=-8),
               dict(n_q_heads=8192, n_kv_heads=1), dict(q_stride=504), dict(q_stride=516), dict(k_stride=120), dict(v_stride=132), dict(out_stride=8),
               dict(q_stride=1 << 31), dict(n_q=(1 << 31) - 1, n_kv_heads=1), dict(n_k=(1 << 31) - 1, n_seqs=(1 << 31) - 1)):
        assert call(**kw) == SHAPE, kw
    for name in ("q", "k", "v", "cu_q", "cu_k", "out", "lse"):
        assert call(ptr={name: None}) == INVALID, name
    for name in ("q", "k", "v", "out"):
        assert call(ptr={name: fake + 8}) == INVALID, name
    assert call(n_seqs=0) == OK
    if entry == "nat_attn_fwd":
        assert call(n_q=0) == OK


def test_attention_backward_refusals(nat):
    call = lambda **kw: attn(nat, "nat_attn_bwd", **kw)
    for name in ("dout", "dq", "dk", "dv"):
        assert call(ptr={name: None}) == INVALID and call(ptr={name: fake + 4}) == INVALID, name
    for kw in (dict(dout_stride=504), dict(dq_stride=513), dict(dk_stride=64), dict(dv_stride=130)):
        assert call(**kw) == SHAPE, kw
    need = nat.attn_bwd_workspace_bytes(100, 8)
    assert need >= 100 * 8 * 4 and need % 256 == 0
    assert call(ws=(None, 1 << 30)) == WORKSPACE and call(ws=(fake, need - 1)) == WORKSPACE and call(ws=(fake + 16, need)) == INVALID
    assert nat.attn_bwd_workspace_bytes(0, 8) == 0 and nat.attn_bwd_workspace_bytes(-4, 8) == 0 and nat.attn_bwd_workspace_bytes(8, 0) == 0
    assert nat.attn_bwd_workspace_bytes((1 << 31) - 1, 4096) == ((1 << 31) - 1) * 4096 * 4 // 256 * 256 + (256 if ((1 << 31) - 1) * 4096 * 4 % 256 else 0)
    assert call(n_q=0, n_k=0, ptr=dict(q=None, k=None, v=None, out=None, lse=None, dout=None, dq=None, dk=None, dv=None), ws=(None, 0)) == OK


def cache(nat, **kw):
    from paper_2603_06619_amd import binding
    c = binding._CKvCache(fake, fake, fake, fake, 10, 2, 64, 128, nat.KV_FP8)
    for name, value in kw.items():
        setattr(c, name, value)
    return ctypes.byref(c)


def cache_calls(nat):
    lib = nat.load_library()
    return (lambda c: lib.nat_kv_write(c, fake, 0, fake, 0, fake, 5, None), lambda c: lib.nat_kv_read(c, fake, 4, fake, 2, 50, fake, 0, fake, 0, None),
            lambda c: lib.nat_attn_decode(c, fake, 0, 2, 8, fake, 4, fake, 0.1, fake, 0, fake, fake, 1 << 30, None))


def test_cache_refusals(nat):
    for call in cache_calls(nat):
        assert call(None) == INVALID
        for kw in (dict(n_pages=0), dict(n_pages=-1), dict(d_k=None), dict(d_v=None), dict(d_k=fake + 8), dict(d_k_exp=None), dict(d_v_exp=None),
                   dict(d_v_exp=fake + 1)):
            assert call(cache(nat, **kw)) == INVALID, kw
        for kw in (dict(page_size=0), dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(page_size=-16), dict(head_dim=80),
                   dict(n_kv_heads=0), dict(n_kv_heads=-2), dict(n_kv_heads=5000)):
            assert call(cache(nat, **kw)) == SHAPE, kw
        assert call(cache(nat, format=2)) == DTYPE


def test_write_and_read_refusals(nat):
    lib, c = nat.load_library(), cache(nat)
    write = lambda k=fake, ks=0, v=fake, vs=0, slots=fake, n=5: lib.nat_kv_write(c, k, ks, v, vs, slots, n, None)
    assert write(k=None) == write(v=None) == write(slots=None) == write(k=fake + 2) == write(n=-1) == INVALID
    assert write(ks=248) == write(vs=260) == write(n=1 << 31) == SHAPE
    assert write(n=0, k=None, v=None, slots=None) == OK
    read = lambda table=fake, width=4, cu=fake, seqs=2, n=50, k=fake, ks=0, v=fake, vs=0: lib.nat_kv_read(c, table, width, cu, seqs, n, k, ks, v, vs, None)
    assert read(table=None) == read(cu=None) == read(k=None) == read(v=None) == read(v=fake + 8) == read(width=-1) == read(seqs=-1) == read(n=-1) == INVALID
    assert read(ks=8) == read(vs=257) == read(n=1 << 31) == SHAPE
    assert read(n=0) == read(seqs=0) == OK


def test_decode_refusals(nat):
    lib, c = nat.load_library(), cache(nat)

    def call(q=fake, qs=0, n=2, hq=8, table=fake, width=4, lens=fake, scale=0.1, out=fake, os=0, lse=fake, ws=fake, ws_bytes=1 << 30):
        return lib.nat_attn_decode(c, q, qs, n, hq, table, width, lens, scale, out, os, lse, ws, ws_bytes, None)
    assert call(q=None) == call(table=None) == call(lens=None) == call(out=None) == call(lse=None) == call(q=fake + 8) == call(out=fake + 2) == INVALID
    assert call(n=-1) == call(width=-1) == call(scale=0.0) == call(scale=float("nan")) == call(scale=float("inf")) == INVALID
    assert call(hq=7) == call(hq=0) == call(hq=-2) == call(qs=1000) == call(os=1028) == call(width=1 << 30) == call(hq=8192) == SHAPE
    assert call(n=0) == OK
    need = nat.attn_decode_workspace_bytes(2, 8, 2, 128, 1000 * 64)
    assert need > 0 and need % 256 == 0 and nat.attn_decode_workspace_bytes(2, 8, 2, 128, 64) == 0
    assert call(width=1000, ws=None) == call(width=1000, ws_bytes=need - 1) == WORKSPACE and call(width=1000, ws=fake + 64) == INVALID
    for bad in ((-1, 8, 2, 128, 64), (2, 7, 2, 128, 64), (2, 8, 2, 96, 64), (2, 8, 2, 128, -1), (2, 8, 0, 128, 64), (2, 8, 2, 128, 1 << 40)):
        assert nat.attn_decode_workspace_bytes(*bad) == 0, bad
    # the workspace grows with neither less memory for more sequences nor without bound for long tables
    assert nat.attn_decode_workspace_bytes(1, 28, 4, 128, 1 << 20) < 64 << 20


def test_sample_refusals(nat):
    lib = nat.load_library()

    def call(logits=fake, stride=0, n=3, V=1000, dtype=1, word=fake, ids=fake, ws=fake, ws_bytes=1 << 30):
        return lib.nat_sample(logits, stride, n, V, dtype, word, None, None, None, None, ids, None, None, ws, ws_bytes, None)
    assert call(dtype=5) == DTYPE
    assert call(n=-1) == call(logits=None) == call(word=None) == call(ids=None) == call(logits=fake + 1) == call(logits=fake + 2, dtype=0) == INVALID
    assert call(V=0) == call(V=-3) == call(V=(1 << 20) + 1) == call(stride=999) == call(stride=-1) == SHAPE
    assert call(n=0, logits=None, word=None, ids=None) == OK
    need = nat.sample_workspace_bytes(3, 150000, nat.DTYPE_BF16)
    assert need > 0 and need % 256 == 0 and nat.sample_workspace_bytes(1000, 150000, nat.DTYPE_BF16) == 0
    assert call(V=150000, ws=None) == call(V=150000, ws_bytes=need - 1) == WORKSPACE and call(V=150000, ws=fake + 128) == INVALID
    assert nat.sample_workspace_bytes(0, 10, 0) == nat.sample_workspace_bytes(5, 0, 0) == nat.sample_workspace_bytes(5, 10, 3) == 0


def test_binding_refuses_what_the_library_cannot_see(nat):
    import torch
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(TypeError):                     # host tensors
        nat.nat_attn_fwd(q, q, q, cu, cu, True, 1.0, q, torch.zeros((2, 4)))
    with pytest.raises(TypeError):
        nat.nat_sample(torch.zeros((2, 8)), cu, None, None, None, None, cu)
    with pytest.raises(TypeError):
        nat.KvCache(q.view(1, 2, 4, 64), q.view(1, 2, 4, 64))
    with pytest.raises(TypeError):
        nat.KvCache(q, q)


def test_kernel_classes_are_named(nat):
    lib = nat.load_library()
    names = [lib.nat_profile_class_name(i).decode() for i in range(lib.nat_profile_num_classes())]
    assert {"attn_fwd", "attn_bwd", "kv_cache", "attn_decode", "sample"} <= set(names) and len(set(names)) == len(names)
