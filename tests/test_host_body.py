"""Host-only: the argument checks of the embedding, of norms and rotation, of the page tables and of the 4-bit cache, through the C ABI and the binding.  Every call
fails before anything is launched, or has nothing to do; pointers named `fake` are never dereferenced."""
import ctypes

import pytest

from test_host_operators import DTYPE, INVALID, OK, SHAPE, WORKSPACE, cache, fake, nat  # noqa: F401 (nat is a fixture)

BIG = 1 << 40


def qk(nat, back=False, ptr=None, ws=(fake, BIG), accumulate=0, **kw):  # noqa: F811
    from paper_2603_06619_amd import binding
    c = binding._CQkParams()
    p = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, dtype=nat.DTYPE_BF16, rotary_dim=64, interleaved=0, eps=1e-6, n_rows=10)
    p.update(kw)
    for name, value in p.items():
        setattr(c, name, value)
    at = dict.fromkeys(("q", "k", "qw", "kw", "pos", "freq", "qo", "ko", "dq", "dk", "dqw", "dkw"), fake)
    at.update(ptr or {})
    lib, head = nat.load_library(), ("q", "k", "qw", "kw", "pos", "freq", "qo", "ko")
    if back:
        return lib.nat_qk_norm_rope_bwd(ctypes.byref(c), *(at[n] for n in head + ("dq", "dk", "dqw", "dkw")), accumulate, *ws, None)
    return lib.nat_qk_norm_rope(ctypes.byref(c), *(at[n] for n in head), None)


@pytest.mark.parametrize("back", [False, True])
def test_norm_and_rotation_refusals(nat, back):  # noqa: F811
    call = lambda **kw: qk(nat, back, **kw)
    lib = nat.load_library()
    assert lib.nat_qk_norm_rope(None, *[fake] * 8, None) == INVALID
    assert call(dtype=2) == call(dtype=-1) == DTYPE
    for kw in (dict(n_rows=-1), dict(n_rows=1 << 31), dict(eps=0.0), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(interleaved=2),
               dict(interleaved=-1)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(head_dim=96), dict(head_dim=0), dict(head_dim=256), dict(n_q_heads=0), dict(n_kv_heads=0), dict(n_q_heads=4097), dict(n_kv_heads=-1),
               dict(rotary_dim=8), dict(rotary_dim=24), dict(rotary_dim=80), dict(rotary_dim=-16), dict(q_stride=504), dict(q_stride=516), dict(k_stride=120),
               dict(q_out_stride=520 + 4), dict(k_out_stride=8), dict(q_stride=1 << 31), dict(dtype=0, k_stride=130)):
        assert call(**kw) == SHAPE, kw
    for name in ("q", "k", "qo", "ko", "pos", "freq") + (("dq", "dk", "dqw", "dkw", "qw", "kw") if back else ()):
        assert call(ptr={name: None}) == INVALID, name
    for name in ("q", "k", "qw", "kw", "qo", "ko") + (("dq", "dk") if back else ()):
        assert call(ptr={name: fake + 8}) == INVALID, name
    assert call(ptr=dict(freq=fake + 4)) == INVALID and call(rotary_dim=0) == INVALID              # positions without a rotation
    ends = ("dq", "dk") if back else ("qo", "ko")                                                  # in the inputs' place, with other rows
    apart = dict.fromkeys(("q", "k", "qo", "ko", "dq", "dk"), fake)
    apart.update(dict(zip(ends, (2 * fake, 2 * fake))))
    for stride, end, start in (("q_out_stride", ends[0], "qo" if back else "q"), ("k_out_stride", ends[1], "ko" if back else "k")):
        assert call(ptr={**apart, end: apart[start]}, **{stride: 1024}) == INVALID, stride
    none = dict.fromkeys(("q", "k", "pos", "freq", "qo", "ko", "dq", "dk"))
    assert call(n_rows=0, ptr=none) == OK if not back else call(n_rows=0, ptr=none, accumulate=1, ws=(None, 0)) == OK


def test_norm_and_rotation_workspace(nat):  # noqa: F811
    need = nat.qk_norm_rope_bwd_workspace_bytes(10, 64)
    assert need > 0 and need % 256 == 0
    assert qk(nat, True, ws=(None, BIG)) == qk(nat, True, ws=(fake, need - 1)) == WORKSPACE and qk(nat, True, ws=(fake + 16, need)) == INVALID
    assert nat.qk_norm_rope_bwd_workspace_bytes(0, 64) == nat.qk_norm_rope_bwd_workspace_bytes(-1, 64) == nat.qk_norm_rope_bwd_workspace_bytes(5, 96) == 0
    assert nat.qk_norm_rope_bwd_workspace_bytes((1 << 31) - 1, 128) <= 64 << 20


def test_embedding_refusals(nat):  # noqa: F811
    lib = nat.load_library()

    def call(ids=fake, n=5, E=fake, V=100, H=64, dtype=1, scale=1.0, out=fake, stride=0):
        return lib.nat_embed(ids, n, E, V, H, dtype, scale, out, stride, None)
    assert call(dtype=2) == DTYPE
    assert call(ids=None) == call(E=None) == call(out=None) == call(E=fake + 8) == call(out=fake + 4) == call(n=-1) == call(n=1 << 31) == INVALID
    assert call(scale=float("nan")) == call(scale=float("inf")) == INVALID
    assert call(V=0) == call(V=-5) == call(H=0) == call(H=(1 << 30) + 8) == call(H=12) == call(H=2, dtype=0) == call(stride=56) == call(stride=68) == call(stride=-64) == SHAPE
    assert call(n=0, ids=None, E=None, out=None) == OK


def test_embedding_gradient_refusals(nat):  # noqa: F811
    lib = nat.load_library()

    def call(ids=fake, n=5, dout=fake, stride=0, V=100, H=64, dtype=1, scale=1.0, dE=fake, acc=0, ws=fake, ws_bytes=BIG):
        return lib.nat_embed_bwd(ids, n, dout, stride, V, H, dtype, scale, dE, acc, ws, ws_bytes, None)
    assert call(dtype=2) == DTYPE
    assert call(ids=None) == call(dout=None) == call(dE=None) == call(dout=fake + 8) == call(dE=fake + 4) == call(n=-1) == INVALID
    assert call(scale=float("nan")) == call(ws=fake + 16) == INVALID
    assert call(V=0) == call(H=0) == call(H=12) == call(stride=56) == call(stride=68) == call(V=(1 << 30) + 1) == call(n=1 << 29) == SHAPE
    need = nat.embed_bwd_workspace_bytes(5, 100, 64)
    assert need > 0 and need % 256 == 0
    assert call(ws=None) == call(ws_bytes=need - 1) == WORKSPACE
    assert nat.embed_bwd_workspace_bytes(0, 100, 64) == nat.embed_bwd_workspace_bytes(5, 0, 64) == nat.embed_bwd_workspace_bytes(5, 100, 0) == 0
    assert call(n=0, ids=None, dout=None, acc=1, ws=None, ws_bytes=0) == OK
    # the sums need room for fewer than 2^24 workgroups
    assert call(n=(1 << 29) - 1, H=1 << 16, dtype=0) == SHAPE


def test_page_refusals(nat):  # noqa: F811
    lib = nat.load_library()

    def reserve(table=fake, width=4, n=3, page=16, lens=fake, new=fake, free=fake, pages=9, counts=fake, cap=10, counts_out=fake, lens_out=fake,
                start=fake, cu=fake, slots=fake, pos=fake, ws=fake, ws_bytes=BIG):
        return lib.nat_kv_reserve(table, width, n, page, lens, new, free, pages, counts, cap, counts_out, lens_out, start, cu, slots, pos, ws, ws_bytes, None)

    def release(table=fake, width=4, n=3, page=16, lens=fake, new=fake, free=fake, pages=9, counts=fake, counts_out=fake, lens_out=fake, ws=fake,
                ws_bytes=BIG):
        return lib.nat_kv_release(table, width, n, page, lens, new, free, pages, counts, counts_out, lens_out, ws, ws_bytes, None)
    for call in (reserve, release):
        for name in ("table", "lens", "new", "free", "counts", "counts_out", "lens_out"):
            assert call(**{name: None}) == INVALID, name
        assert call(n=-1) == call(width=-1) == call(pages=-1) == call(ws=fake + 16) == INVALID
        assert call(page=8) == call(page=48) == call(page=512) == call(page=0) == call(n=(1 << 24) + 1) == call(width=1 << 27) == SHAPE
        assert call(ws=None) == call(ws_bytes=255) == WORKSPACE
    for name in ("start", "cu", "slots"):
        assert reserve(**{name: None}) == INVALID, name
    assert reserve(cap=-1) == reserve(cap=1 << 31) == INVALID
    assert nat.kv_reserve_workspace_bytes(0) == nat.kv_release_workspace_bytes(-3) == nat.kv_reserve_workspace_bytes((1 << 24) + 1) == 0
    assert nat.kv_reserve_workspace_bytes(65) == 512 and nat.kv_release_workspace_bytes(64) == 512


def test_4_bit_cache_refusals(nat):  # noqa: F811
    lib = nat.load_library()
    write = lambda c: lib.nat_kv_write(c, fake, 0, fake, 0, fake, 5, None)
    read = lambda c: lib.nat_kv_read(c, fake, 4, fake, 2, 50, fake, 0, fake, 0, None)
    decode = lambda c: lib.nat_attn_decode(c, fake, 0, 2, 8, fake, 4, fake, 0.1, fake, 0, fake, fake, 1 << 30, None)
    for call in (write, read, decode):
        for kw in (dict(d_k_exp=None), dict(d_v_exp=None), dict(d_k_exp=fake + 4), dict(d_k=None)):
            assert call(cache(nat, format=nat.KV_FP4, **kw)) == INVALID, kw
        assert call(cache(nat, format=nat.KV_FP4, head_dim=96)) == SHAPE
        assert call(cache(nat, format=3)) == call(cache(nat, format=5)) == call(cache(nat, format=-1)) == DTYPE


def test_binding_refuses_what_the_library_cannot_see(nat):  # noqa: F811
    import torch
    from paper_2603_06619_amd.rollout import PagedCache, RolloutStage
    q, i32 = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):                     # host tensors
        nat.nat_qk_norm_rope(q, q, None, None, None, None, 1e-6, False, q, q)
    with pytest.raises(TypeError):
        nat.nat_qk_norm_rope(q.half(), q.half(), None, None, None, None, 1e-6, False, q, q)
    with pytest.raises(TypeError):
        nat.nat_embed(i32, q[0], 1.0, q[0])
    with pytest.raises(TypeError):
        nat.nat_embed_bwd(i32, q[0], 1.0, torch.zeros((3, 64)), False, None)
    with pytest.raises(TypeError):
        nat.nat_kv_reserve(i32.view(2, 2), i32[:2], i32[:2], i32, i32[:2], 16, 0, i32[:2], i32[:2], i32[:2], i32[:3], i32[:0].long(), None, None)
    with pytest.raises(TypeError):
        nat.KvCache(q.view(1, 2, 4, 64).view(torch.uint8), q.view(1, 2, 4, 64).view(torch.uint8))
    with pytest.raises(ValueError):
        PagedCache.empty(1, 1, 16, 64, fp8=True, fp4=True, device="cpu")
    with pytest.raises(ValueError):
        RolloutStage("cpu").embed_backward(q[0], i32, 3, accumulate=True)


def test_kernel_classes_are_named(nat):  # noqa: F811
    lib = nat.load_library()
    names = [lib.nat_profile_class_name(i).decode() for i in range(lib.nat_profile_num_classes())]
    assert {"qk_norm_rope", "embed", "pages"} <= set(names) and len(set(names)) == len(names)
