"""Host-only: calls that would need more work-items than a launch has room for (2^32) are refused.  Pointers named `fake` are never dereferenced."""
import pytest

from test_host_operators import SHAPE, attn, cache, fake, nat  # noqa: F401 (nat is a fixture)


@pytest.mark.parametrize("entry", ["nat_attn_fwd", "nat_attn_bwd"])
def test_attention_of_very_many_sequences(nat, entry):  # noqa: F811
    call = lambda **kw: attn(nat, entry, **kw)
    for kw in (dict(n_seqs=1 << 23, n_kv_heads=2), dict(n_seqs=1 << 21, n_kv_heads=8), dict(n_seqs=(1 << 24) - 7, n_kv_heads=1), dict(n_seqs=1 << 12, n_q_heads=4096, n_kv_heads=4096),
               dict(n_seqs=1 << 20, n_kv_heads=2, n_k=(1 << 31) - 1)):
        assert call(**kw) == SHAPE, kw


def test_decoding_of_very_many_sequences(nat):  # noqa: F811
    lib = nat.load_library()

    def call(n, hq, width=4, **kw):
        return lib.nat_attn_decode(cache(nat, **kw), fake, 0, n, hq, fake, width, fake, 0.1, fake, 0, fake, fake, 1 << 62, None)
    assert call(1 << 23, 2, n_kv_heads=2) == SHAPE and call(1 << 21, 8, n_kv_heads=8) == SHAPE and call(1 << 22, 256, width=1, n_kv_heads=4) == SHAPE
    assert call(1 << 19, 32, width=1 << 10, n_kv_heads=8) == SHAPE
    for n, hq, hkv, tokens in ((1 << 23, 2, 2, 256), (1 << 19, 32, 8, 1 << 16)):
        assert nat.attn_decode_workspace_bytes(n, hq, hkv, 128, tokens) == 0


def test_the_join_of_many_heads(nat):  # noqa: F811
    """Few key heads of many query heads each, 3 chunks of 4096 tokens: the second kernel, a wavefront per query head, is the larger one."""
    lib, n, hq = nat.load_library(), 300000, 256
    assert n * (hq // 16) * 3 * 256 < 1 << 32 < n * hq * 64
    call = lib.nat_attn_decode(cache(nat, n_kv_heads=1, page_size=256), fake, 0, n, hq, fake, 48, fake, 0.1, fake, 0, fake, fake, 1 << 62, None)
    assert call == SHAPE
