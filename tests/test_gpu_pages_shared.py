"""Rollouts that share the full pages of their prompt: read by all of them, given back by one."""
import pytest
import torch

from nat_testlib import DEV

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_a_prompt_of_several_rollouts():
    from paper_2603_06619_amd.rollout import PagedCache, RolloutStage
    stage, page, width, n_pages, group, hkv, D = RolloutStage(DEV), 16, 6, 12, 3, 2, 64
    g = torch.Generator(device=DEV).manual_seed(1)
    new = lambda *s: torch.randn(s, generator=g, device=DEV).bfloat16()
    cache = PagedCache.empty(n_pages, hkv, page, D, device=DEV, fp4=True)
    table, free, counts = dev([[-1] * width] * group), dev([3, 8, 1, 11, 0, 5, 9, 2, 10, 4, 7, 6]), dev([n_pages, 0])
    # the prompt: two full pages, of the first rollout, and named by the others
    first = stage.reserve(table, dev([0] * group), dev([2 * page, 0, 0]), free, counts, page, 2 * page)
    k, v = new(2 * page, hkv, D), new(2 * page, hkv, D)
    stage.write_cache(cache, k, v, first["slots"])
    shared = table[0, :2].tolist()
    table[1:, :2] = table[0, :2]
    lens, counts = dev([2 * page] * group), first["counts"]
    # their own tokens, in pages of their own
    own = stage.reserve(table, lens, dev([20] * group), free, counts, page, 20 * group)
    mine = table[:, 2:4].flatten().tolist()
    assert own["counts"].tolist() == [n_pages - 2 - 2 * group, 0] and len(set(mine + shared)) == 2 + 2 * group
    k2, v2 = new(20 * group, hkv, D), new(20 * group, hkv, D)
    stage.write_cache(cache, k2, v2, own["slots"])
    # each reads what it would read from a cache of its own
    q = new(group, 4, D)
    out, lse = stage.decode(q, cache, table, own["seq_lens"])
    for i in range(group):
        alone = PagedCache.empty(width, hkv, page, D, device=DEV, fp4=True)
        rows = slice(20 * i, 20 * i + 20)
        stage.write_cache(alone, torch.cat((k, k2[rows])), torch.cat((v, v2[rows])), torch.arange(2 * page + 20, device=DEV))
        ref, ref_lse = stage.decode(q[i:i + 1], alone, torch.arange(width, dtype=torch.int32, device=DEV)[None], own["seq_lens"][i:i + 1])
        assert torch.equal(out[i:i + 1], ref) and torch.equal(lse[i:i + 1], ref_lse)
    # back: the two others first, without the shared pages, which they do not own; then the first
    keep_out = table.clone()
    keep_out[1:, :2] = -1
    lens, counts = stage.release(keep_out, own["seq_lens"], dev([2 * page + 20, 0, 0]), free, own["counts"], page)
    assert lens.tolist() == [2 * page + 20, 0, 0] and counts.tolist() == [n_pages - 4, 0]
    assert not set(free[:n_pages - 4].tolist()) & set(table[0, :4].tolist())
    lens, counts = stage.release(keep_out, lens, dev([0] * group), free, counts, page)
    assert counts.tolist() == [n_pages, 0] and sorted(free.tolist()) == list(range(n_pages))
