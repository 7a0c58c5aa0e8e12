"""Workspace of attention's backward pass with shared rows: its size, and what it is for counts out of range."""
import pytest

import paper_2603_06619_amd as nat


def test_full_workspace():
    full, least = nat.attn_bwd_workspace_full_bytes, nat.attn_bwd_workspace_bytes
    for n, hq, hkv, D in ((1024, 32, 8, 128), (8192, 4, 4, 64), (2048, 2, 1, 128)):
        slab = n * hkv * D * 8
        size = full(n, n, 1, hq, hkv, D, True)
        assert size > least(n, hq) and (size - least(n, hq)) % slab == 0 and (size - least(n, hq)) // slab in range(2, 9)
    assert full(32768, 32768, 8, 32, 8, 128, True) == least(32768, 32)              # keys enough
    assert full(64, 64, 1, 8, 8, 64, True) == least(64, 8)                          # too few rows to share
    assert full(0, 10, 1, 8, 8, 64, True) == 0


@pytest.mark.parametrize("kw", [dict(hq=3, hkv=2), dict(hkv=0), dict(hq=-4, hkv=-4), dict(D=96), dict(n_q=1 << 40), dict(n_k=1 << 40), dict(n_seqs=-1), dict(n_k=-5)])
def test_counts_out_of_range(kw):
    a = dict(n_q=1000, n_k=1000, n_seqs=1, hq=8, hkv=1, D=64)
    a.update(kw)
    size = nat.attn_bwd_workspace_full_bytes(a["n_q"], a["n_k"], a["n_seqs"], a["hq"], a["hkv"], a["D"], True)
    assert size in (0, nat.attn_bwd_workspace_bytes(1000, 8))


def test_forward_workspace():
    size = nat.attn_fwd_workspace_bytes
    for n_q, n_k, hq, hkv, D in ((16, 8016, 32, 8, 128), (2048, 2048, 2, 1, 128), (1, 5000, 4, 4, 64)):
        part = n_q * hq * (D + 2) * 4
        assert any(size(n_q, n_k, 1, hq, hkv, D, True) == (p * part + 255) // 256 * 256 for p in range(2, 17))
    assert size(32768, 32768, 8, 32, 8, 128, True) == 0                             # rows enough
    assert size(16, 400, 1, 8, 8, 64, True) == 0                                    # too few keys to share
    for a in ((16, 8016, 1, 3, 2, 64), (16, 8016, 1, 8, 0, 64), (16, 8016, 1, 8, 8, 96), (-1, 8016, 1, 8, 8, 64), (16, 1 << 40, 1, 8, 8, 64), (16, 8016, 0, 8, 8, 64)):
        assert size(*a, True) == 0


def test_forward_refusals():
    import ctypes
    from paper_2603_06619_amd import binding
    lib, fake = nat.load_library(), 1 << 20
    p = binding._CAttnParams(1, 8, 8, 64, nat.DTYPE_BF16, 1, 0.1, 16, 8016)
    call = lambda **kw: lib.nat_attn_fwd_split(ctypes.byref(p), *(kw.get(n, fake) for n in ("q", "k", "v", "cu_q", "cu_k", "out", "lse", "ws")), 1 << 30, None)
    invalid = lib.nat_attn_fwd(None, fake, fake, fake, fake, fake, fake, fake, None)
    assert invalid != 0
    for n in ("q", "k", "v", "cu_q", "cu_k", "out", "lse"):
        assert call(**{n: None}) == invalid, n
    assert call(ws=fake + 16) == invalid and call(out=fake + 8) == invalid
