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
